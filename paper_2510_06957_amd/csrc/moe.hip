// A mixture-of-experts feed-forward layer for a few tokens (tst_moe): the router, the top experts of each token, and the experts'
// products from 8-bit weights.
//
// Weights meet the matrix cores as bf16, which holds every 8-bit code exactly.  The activations are cut into bf16 planes by cutting
// mantissas off (x = p0 + p1 + p2, p0 the upper 16 bits of x, p1 those of x - p0, ...): one plane holds a bf16 entry, two an fp16
// entry, three an fp32 entry, all exactly, so that products are exact and only the fp32 sums round.
//
// The tokens are the columns of a matrix instruction (16 at a time) and the weights its rows: up to 16 tokens cost the matrix cores the same, and
// a token that has not chosen an expert is a column that is not used (first product) or zero (second).
#include "ops_internal.h"

namespace tst {
namespace {

constexpr int kMaxTokens = 64;   // of one launch; more go in slabs
constexpr int kMaxE = TST_MOE_MAX_EXPERTS, kMaxTop = TST_MOE_MAX_TOP;

struct MoeArgs {
    const void *X;
    int64_t x_stride;
    const void *router;
    const char *gate, *up, *down;
    const float *gate_scale, *up_scale, *down_scale;
    void *Y;
    int32_t *ids;
    float *p;
    int E, D, F, T, top;
    bool normalize;
    // workspace
    float *logits;      // [T][E]
    uint16_t *x;        // [planes][T][D_pad] bf16, zero behind D
    uint16_t *h;        // [h planes][T * top][F_pad] bf16, zero behind F
};

constexpr int planes_of(int type) { return type == TST_F32 ? 3 : type == TST_F16 ? 2 : 1; }
constexpr int h_planes_of(int type) { return type == TST_F32 ? 3 : 2; }
inline __host__ __device__ int pad64(int n) { return (n + 63) & ~63; }

// The upper 16 bits of v, and what is left of v (0 if v is infinite, NaN if it is NaN).
__device__ __forceinline__ uint16_t cut(float &v)
{
    const unsigned u = __float_as_uint(v), hi = u & 0xffff0000u;
    v = (u & 0x7fffffffu) == 0x7f800000u ? 0.f : v - __uint_as_float(hi);
    return (uint16_t)(hi >> 16);
}

__device__ __forceinline__ float wave_sum(float v)
{
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d);
    return v;
}

// ------------------------------------------------------------------------------------------------------------------
// k_moe_router: a wavefront per (token, expert) for the logits, and the planes of X.
constexpr int kRouterWaves = 4;

template <int TYPE>
__global__ void __launch_bounds__(kRouterWaves * 64)
k_moe_router(const MoeArgs a)
{
    typedef Entry<TYPE> E;
    typedef typename E::bits bits;
    const int t = blockIdx.y, lane = threadIdx.x & 63, e = blockIdx.x * kRouterWaves + (threadIdx.x >> 6);
    const bits *x = static_cast<const bits *>(a.X) + t * a.x_stride;
    if (e < a.E) {
        const bits *r = static_cast<const bits *>(a.router) + (size_t)e * a.D;
        float sum = 0.f;
        for (int d = lane; d < a.D; d += 64) sum = fmaf(E::get(x[d]), E::get(r[d]), sum);
        sum = wave_sum(sum);
        if (lane == 0) a.logits[t * a.E + e] = sum;
    }
    const int d_pad = pad64(a.D);
    for (int d = blockIdx.x * kRouterWaves * 64 + threadIdx.x; d < d_pad; d += gridDim.x * kRouterWaves * 64) {
        float v = d < a.D ? E::get(x[d]) : 0.f;
#pragma unroll
        for (int p = 0; p < planes_of(TYPE); ++p) a.x[((size_t)p * a.T + t) * d_pad + d] = cut(v);
    }
}

// ------------------------------------------------------------------------------------------------------------------
// Which tokens chose which expert, in the LDS: place[e][t] = rank of expert e among token t's, or 255.
struct Chosen {
    uint8_t place[kMaxE][kMaxTokens];
    float p[kMaxTokens][kMaxTop];
    uint16_t active[kMaxE];   // experts that some token chose, ascending
    int n_active;
};

// Bits that order as logits do: NaN above everything, -0 as +0.
__device__ __forceinline__ unsigned order_key(float v)
{
    const unsigned u = __float_as_uint(v + 0.f);
    if ((u & 0x7fffffffu) > 0x7f800000u) return 0xffffffffu;
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

__device__ __forceinline__ unsigned long long wave_max64(unsigned long long v)
{
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) {
        const unsigned long long o = ((unsigned long long)(unsigned)__shfl_xor((int)(v >> 32), d) << 32) | (unsigned)__shfl_xor((int)v, d);
        v = v > o ? v : o;
    }
    return v;
}

// A wavefront finds a token's experts: top rounds of the largest of what is left; lane l holds experts l, l + 64, ...
__device__ void choose_experts(const MoeArgs &a, Chosen &c, int t, int lane, bool write)
{
    constexpr int kPer = kMaxE / 64;
    float l[kPer];
    unsigned long long key[kPer];   // logit, then the lower expert first; 0: none (left)
    float most = -INFINITY;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int e = lane + 64 * i;
        l[i] = e < a.E ? a.logits[t * a.E + e] : -INFINITY;
        key[i] = e < a.E ? ((unsigned long long)order_key(l[i]) << 32) | (unsigned)(kMaxE - e) : 0ull;
    }
    float all = 0.f, chosen = 0.f;
    for (int j = 0; j < a.top; ++j) {
        unsigned long long best = 0;
#pragma unroll
        for (int i = 0; i < kPer; ++i) best = best > key[i] ? best : key[i];
        best = wave_max64(best);
        const int e = kMaxE - (int)(unsigned)best;
        float value = 0.f;
#pragma unroll
        for (int i = 0; i < kPer; ++i)
            if (key[i] == best) {
                key[i] = 0;
                value = l[i];
            }
        value = __shfl(value, e & 63);
        if (j == 0) {
            most = value;
#pragma unroll
            for (int i = 0; i < kPer; ++i)
                if (lane + 64 * i < a.E) all += expf(l[i] - most);
            all = wave_sum(all);
        }
        const float w = expf(value - most);
        chosen += w;
        if (lane == 0) {
            c.place[e][t] = (uint8_t)j;
            c.p[t][j] = w;
            if (write) a.ids[t * a.top + j] = e;
        }
    }
    const float total = a.normalize ? chosen : all;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");   // lane 0 wrote what the others read
    if (lane < a.top) {
        const float p = c.p[t][lane] / total;
        c.p[t][lane] = p;
        if (write) a.p[t * a.top + lane] = p;
    }
}

// place[][] from the experts of each token (all threads), and the list of experts in use.
__device__ void list_active(const MoeArgs &a, Chosen &c)
{
    if (threadIdx.x < 64) {   // one wavefront goes through the experts, 64 at a time
        int n = 0;
        for (int e0 = 0; e0 < a.E; e0 += 64) {
            const int e = e0 + threadIdx.x;
            bool any = false;
            if (e < a.E)
                for (int t = 0; t < a.T; ++t) any |= c.place[e][t] != 255;
            const unsigned long long set = __ballot(any);
            if (any) c.active[n + __popcll(set & ((1ull << threadIdx.x) - 1))] = (uint16_t)e;
            n += __popcll(set);
        }
        if (threadIdx.x == 0) c.n_active = n;
    }
    __syncthreads();
}

__device__ __forceinline__ void clear_places(const MoeArgs &a, Chosen &c, int threads)
{
    unsigned *w = reinterpret_cast<unsigned *>(c.place);
    for (int i = threadIdx.x; i < a.E * kMaxTokens / 4; i += threads) w[i] = 0xffffffffu;
    __syncthreads();
}

// Sixteen 8-bit weights of a lane as two operands of the bf16 matrix instruction.
__device__ __forceinline__ void widen(u32x4 w, bf16x8 out[2])
{
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        u32x4 o;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const unsigned v = w[2 * s + i / 2] >> (16 * (i % 2));
            const unsigned lo = __float_as_uint((float)(int)(signed char)(v & 0xff));
            const unsigned hi = __float_as_uint((float)(int)(signed char)((v >> 8) & 0xff));
            o[i] = __builtin_amdgcn_perm(hi, lo, 0x07060302);
        }
        out[s] = __builtin_bit_cast(bf16x8, o);
    }
}

// ------------------------------------------------------------------------------------------------------------------
// k_moe_up: h = silu(x gate) (x up) p for each token and expert it chose, in planes.  Every workgroup finds the experts by itself;
// the first one writes them out.  Work is one expert x 16 columns of its gate and up, for all tokens; wavefronts share D.
constexpr int kUpWaves = 8;

template <int TYPE, int NT>
__global__ void __launch_bounds__(kUpWaves * 64)
k_moe_up(const MoeArgs a)
{
    __shared__ Chosen c;
    __shared__ f32x4 part[kUpWaves][2][NT][64];
    constexpr int P = planes_of(TYPE), PH = h_planes_of(TYPE);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    clear_places(a, c, kUpWaves * 64);
    for (int t = wave; t < a.T; t += kUpWaves) choose_experts(a, c, t, lane, blockIdx.x == 0);
    __syncthreads();
    list_active(a, c);

    const int d_pad = pad64(a.D), f_pad = pad64(a.F);
    const int k_blocks = d_pad / 64, cols = f_pad / 16, real_cols = blocks_of(a.F, kW8Cols);
    const size_t matrix = (size_t)k_blocks * real_cols * kW8Piece;
    for (int item = blockIdx.x; item < c.n_active * cols; item += gridDim.x) {
        const int e = c.active[item / cols], nb = item % cols;
        bool mine[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) mine[t] = 16 * t + (lane & 15) < a.T && c.place[e][16 * t + (lane & 15)] != 255;
        f32x4 acc[2][NT] = {};
        if (nb < real_cols) {
            const size_t at = e * matrix + (size_t)nb * k_blocks * kW8Piece + lane * 16;
            for (int kb = wave; kb < k_blocks; kb += kUpWaves) {
                bf16x8 wg[2], wu[2];
                widen(*reinterpret_cast<const u32x4 *>(a.gate + at + (size_t)kb * kW8Piece), wg);
                widen(*reinterpret_cast<const u32x4 *>(a.up + at + (size_t)kb * kW8Piece), wu);
#pragma unroll
                for (int t = 0; t < NT; ++t) {
#pragma unroll
                    for (int p = 0; p < P; ++p) {
                        const uint16_t *x = a.x + ((size_t)p * a.T + 16 * t + (lane & 15)) * d_pad + kb * 64 + 16 * (lane >> 4);
#pragma unroll
                        for (int s = 0; s < 2; ++s) {
                            u32x4 v = {};
                            if (mine[t]) v = *reinterpret_cast<const u32x4 *>(x + 8 * s);
                            const bf16x8 xf = __builtin_bit_cast(bf16x8, v);
                            acc[0][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wg[s], xf, acc[0][t], 0, 0, 0);
                            acc[1][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wu[s], xf, acc[1][t], 0, 0, 0);
                        }
                    }
                }
            }
        }
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            part[wave][0][t][lane] = acc[0][t];
            part[wave][1][t][lane] = acc[1][t];
        }
        __syncthreads();
        for (int i = threadIdx.x; i < NT * 64; i += kUpWaves * 64) {
            const int t = i >> 6, l = i & 63, token = 16 * t + (l & 15);
            const int place = token < a.T ? c.place[e][token] : 255;
            if (place == 255) continue;
            f32x4 g = part[0][0][t][l], u = part[0][1][t][l];
#pragma unroll
            for (int w = 1; w < kUpWaves; ++w) {
                g += part[w][0][t][l];
                u += part[w][1][t][l];
            }
            const int f = nb * 16 + 4 * (l >> 4);
            uint16_t out[PH][4];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                float h = 0.f;
                if (f + r < a.F) {
                    const float gv = g[r] * a.gate_scale[(size_t)e * a.F + f + r], uv = u[r] * a.up_scale[(size_t)e * a.F + f + r];
                    h = gv / (1.f + expf(-gv)) * uv * c.p[token][place];
                }
#pragma unroll
                for (int p = 0; p < PH; ++p) out[p][r] = p < PH - 1 ? cut(h) : Entry<TST_BF16>::put(h);   // the last one rounds
            }
#pragma unroll
            for (int p = 0; p < PH; ++p)
                *reinterpret_cast<u32x2 *>(a.h + ((size_t)p * a.T * a.top + token * a.top + place) * f_pad + f) =
                    u32x2{out[p][0] | (unsigned)out[p][1] << 16, out[p][2] | (unsigned)out[p][3] << 16};
        }
        __syncthreads();
    }
}

// ------------------------------------------------------------------------------------------------------------------
// k_moe_down: 16 columns of Y for all tokens; the wavefronts share the rows of all experts in use, one after another.  Between
// experts a wavefront scales its sums with the expert's channels and adds them to those of the token.
constexpr int kDownWaves = 8;

template <int TYPE, int NT>
__global__ void __launch_bounds__(kDownWaves * 64)
k_moe_down(const MoeArgs a)
{
    typedef Entry<TYPE> E;
    __shared__ Chosen c;
    __shared__ f32x4 part[kDownWaves][NT][64];
    constexpr int PH = h_planes_of(TYPE);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, nb = blockIdx.x;
    clear_places(a, c, kDownWaves * 64);
    for (int i = threadIdx.x; i < a.T * a.top; i += kDownWaves * 64) c.place[a.ids[i]][i / a.top] = (uint8_t)(i % a.top);
    __syncthreads();
    list_active(a, c);

    const int f_pad = pad64(a.F), k_blocks = f_pad / 64, n_blocks = blocks_of(a.D, kW8Cols);
    const int total = c.n_active * k_blocks, share = blocks_of(total, kDownWaves);
    int at = min(wave * share, total);
    const int end = min(at + share, total);
    f32x4 sum[NT] = {};
    while (at < end) {
        const int e = c.active[at / k_blocks], kb0 = at % k_blocks, kb1 = min(k_blocks, kb0 + end - at);
        at += kb1 - kb0;
        int row[NT];   // of h, or -1
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const int token = 16 * t + (lane & 15);
            const int place = token < a.T ? c.place[e][token] : 255;
            row[t] = place == 255 ? -1 : token * a.top + place;
        }
        const char *w = a.down + ((size_t)e * n_blocks + nb) * k_blocks * kW8Piece + lane * 16;
        f32x4 acc[NT] = {};
        for (int kb = kb0; kb < kb1; ++kb) {
            bf16x8 wd[2];
            widen(*reinterpret_cast<const u32x4 *>(w + (size_t)kb * kW8Piece), wd);
#pragma unroll
            for (int t = 0; t < NT; ++t) {
#pragma unroll
                for (int p = 0; p < PH; ++p) {
#pragma unroll
                    for (int s = 0; s < 2; ++s) {
                        u32x4 v = {};
                        if (row[t] >= 0)
                            v = *reinterpret_cast<const u32x4 *>(a.h + ((size_t)p * a.T * a.top + row[t]) * f_pad + kb * 64 + 16 * (lane >> 4) + 8 * s);
                        acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wd[s], __builtin_bit_cast(bf16x8, v), acc[t], 0, 0, 0);
                    }
                }
            }
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int d = min(nb * 16 + 4 * (lane >> 4) + r, a.D - 1);
            const float scale = a.down_scale[(size_t)e * a.D + d];
#pragma unroll
            for (int t = 0; t < NT; ++t)
                if (row[t] >= 0) sum[t][r] = fmaf(scale, acc[t][r], sum[t][r]);
        }
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) part[wave][t][lane] = sum[t];
    __syncthreads();
    for (int i = threadIdx.x; i < NT * 64; i += kDownWaves * 64) {
        const int t = i >> 6, l = i & 63, token = 16 * t + (l & 15);
        if (token >= a.T) continue;
        f32x4 y = part[0][t][l];
#pragma unroll
        for (int w = 1; w < kDownWaves; ++w) y += part[w][t][l];
        typename E::bits *to = static_cast<typename E::bits *>(a.Y) + (size_t)token * a.D;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int d = nb * 16 + 4 * (l >> 4) + r;
            if (d < a.D) to[d] = E::put(y[r]);
        }
    }
}

struct MoeSpace {
    size_t logits, x, h, total;
};
MoeSpace moe_space(const tst_moe_t &m, int T, int top)
{
    MoeSpace s{};
    if (T > kMaxTokens) T = kMaxTokens;
    size_t at = 0;
    s.logits = at;
    at += round256((size_t)T * m.experts * sizeof(float));
    s.x = at;
    at += round256((size_t)planes_of(m.type) * T * pad64(m.width) * 2);
    s.h = at;
    at += round256((size_t)h_planes_of(m.type) * T * top * pad64(m.inner) * 2);
    s.total = at;
    return s;
}

template <int TYPE, int NT> hipError_t launch_moe_nt(const MoeArgs &a, hipStream_t stream)
{
    k_moe_router<TYPE><<<dim3(blocks_of(a.E, kRouterWaves), a.T), kRouterWaves * 64, 0, stream>>>(a);
    if (hipError_t e = hipGetLastError()) return e;
    const int64_t items = (int64_t)(a.E < a.T * a.top ? a.E : a.T * a.top) * (pad64(a.F) / 16);
    k_moe_up<TYPE, NT><<<(unsigned)(items < 1024 ? items : 1024), kUpWaves * 64, 0, stream>>>(a);
    if (hipError_t e = hipGetLastError()) return e;
    k_moe_down<TYPE, NT><<<blocks_of(a.D, kW8Cols), kDownWaves * 64, 0, stream>>>(a);
    return hipGetLastError();
}

int check_moe(const tst_moe_t *m, int T, int top)
{
    if (!m || m->struct_size != sizeof(tst_moe_t) || !type_ok(m->type) || T < 0) return TSTGEMM_EINVAL;
    if (m->experts < 1 || m->experts > kMaxE || m->width < 1 || m->width > kW8MaxK || m->inner < 1 || m->inner > kW8MaxK)
        return TSTGEMM_EINVAL;
    if (top < 1 || top > kMaxTop || top > m->experts) return TSTGEMM_EINVAL;
    return TSTGEMM_OK;
}

}  // namespace
}  // namespace tst

extern "C" {

int tst_moe_workspace_bytes(const tst_moe_t *moe, int T, int top_k, size_t *bytes)
{
    if (!bytes) return TSTGEMM_EINVAL;
    if (int rc = tst::check_moe(moe, T, top_k)) return rc;
    *bytes = tst::moe_space(*moe, T, top_k).total;
    return TSTGEMM_OK;
}

int tst_moe(const void *X, int64_t x_stride, const tst_moe_t *moe, int top_k, int normalize, void *Y, int32_t *ids, float *p, int T,
            void *workspace, size_t workspace_bytes, void *stream)
{
    if (int rc = tst::check_moe(moe, T, top_k)) return rc;
    if (T == 0) return TSTGEMM_OK;
    const tst_moe_t &m = *moe;
    const size_t entry = tst::type_bytes(m.type);
    if (!X || !Y || !ids || !p || !m.router || !m.gate || !m.up || !m.down || !m.gate_scale || !m.up_scale || !m.down_scale ||
        x_stride < m.width || !tst::aligned(X, entry) || !tst::aligned(Y, entry) || !tst::aligned(m.router, entry) ||
        !tst::aligned(m.gate, 16) || !tst::aligned(m.up, 16) || !tst::aligned(m.down, 16))
        return TSTGEMM_EINVAL;
    const tst::MoeSpace s = tst::moe_space(m, T, top_k);
    if (!workspace || workspace_bytes < s.total) return TSTGEMM_EWORKSPACE;
    if (!tst::aligned(workspace, 256)) return TSTGEMM_EINVAL;
    char *ws = static_cast<char *>(workspace);
    for (int64_t t0 = 0; t0 < T; t0 += tst::kMaxTokens) {
        const int n = (int)(T - t0 < tst::kMaxTokens ? T - t0 : tst::kMaxTokens);
        const tst::MoeArgs a{static_cast<const char *>(X) + t0 * x_stride * entry, x_stride, m.router, static_cast<const char *>(m.gate),
                             static_cast<const char *>(m.up), static_cast<const char *>(m.down), m.gate_scale, m.up_scale, m.down_scale,
                             static_cast<char *>(Y) + t0 * m.width * entry, ids + t0 * top_k, p + t0 * top_k, m.experts, m.width, m.inner, n,
                             top_k, normalize != 0, reinterpret_cast<float *>(ws + s.logits), reinterpret_cast<uint16_t *>(ws + s.x),
                             reinterpret_cast<uint16_t *>(ws + s.h)};
        const hipError_t e = tst::for_type(m.type, [&](auto type) {
            constexpr int TYPE = decltype(type)::value;
            hipStream_t st = static_cast<hipStream_t>(stream);
            return n <= 16 ? tst::launch_moe_nt<TYPE, 1>(a, st) : n <= 32 ? tst::launch_moe_nt<TYPE, 2>(a, st) : tst::launch_moe_nt<TYPE, 4>(a, st);
        });
        if (e != hipSuccess) return TSTGEMM_EHIP;
    }
    return TSTGEMM_OK;
}

}  // extern "C"
