// Causal attention over whole prompts, packed one behind another, with grouped heads (tst_attention).
//
// A workgroup has a tile of rows of one key head, a row being (token, query head of the group), so that the keys and values that it loads serve all heads of
// the group, and goes through the keys from the first to the tile's last, 64 (fp32: 32) at a time, with the running largest logit and sum of each row.  Z^T = K Q^T and
// Y^T = V^T P^T with the 32 x 32 x 16 instructions: a row's logits, weights and sums stay in the lanes with its number (mod 32), and the weights are the second
// product's operand as they come out of the first, since keys may stand in any order there: lanes of half h hold keys 8 (r / 4) + 4 h + r % 4 of 32.
// K and V go through the LDS as rows; the second product's operand, four keys of a channel in a lane, comes out of it by reads that transpose.
//
// fp32 operands are cut into three bf16 planes by cutting mantissas off (exact) and six products of planes are summed: all but 2^-24 of a product.
#include "attention_internal.h"

#include <cmath>

#ifndef V_QB
#define V_QB 1
#define V_NW 8
#define V_OCC 2
#endif
namespace tst {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr float kNan = __builtin_nanf("");
constexpr float kLog2e = 1.44269504088896340736f;

struct PromptArgs {
    Rows q, k, v;
    int q_heads, heads, group, size, sequences, tokens, tiles;
    const int32_t *offsets;
    float scale;   // its magnitude times log2 e; 2^-126 for 0 and less, so that -inf stays what it is
    bool negative;
    void *y;
    bool wide;     // rows of Q, K and V on 16-byte borders, of a multiple of 8 entries
};

// 8 entries of a row as the planes that matrix instructions take, zeros behind its end.
template <int TYPE> struct Planes {
    static constexpr int kCount = TYPE == TST_F32 ? 3 : 1;
    u32x4 p[kCount];
};
// Entries d .. d + 7; raw bits.
template <int TYPE> struct Raw {
    typename Entry<TYPE>::bits e[8];
};
template <int TYPE> __device__ __forceinline__ Raw<TYPE> load_raw(const typename Entry<TYPE>::bits *row, int d, int size, bool there, bool wide)
{
    union {
        Raw<TYPE> r;
        u32x4 v[sizeof(Raw<TYPE>) / 16];
    } u;
#pragma unroll
    for (int i = 0; i < (int)(sizeof(u) / 16); ++i) u.v[i] = u32x4{0, 0, 0, 0};
    if (wide) {
        if (there && d < size) {
#pragma unroll
            for (int i = 0; i < (int)(sizeof(u) / 16); ++i) u.v[i] = reinterpret_cast<const u32x4 *>(row + d)[i];
        }
    } else if (there) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (d + i < size) u.r.e[i] = row[d + i];
    }
    return u.r;
}
template <int TYPE> __device__ __forceinline__ Planes<TYPE> planes_of(const Raw<TYPE> &r)
{
    Planes<TYPE> out;
    if constexpr (TYPE != TST_F32) {
        out.p[0] = __builtin_bit_cast(u32x4, r);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            unsigned w[3] = {0, 0, 0};
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float x = r.e[2 * i + e];
#pragma unroll
                for (int p = 0; p < 3; ++p) {
                    const unsigned b = __float_as_uint(x) & 0xffff0000u;
                    w[p] |= e ? b : b >> 16;
                    x -= __uint_as_float(b);
                }
            }
#pragma unroll
            for (int p = 0; p < 3; ++p) out.p[p][i] = w[p];
        }
    }
    return out;
}

// Two weights as the second product takes them, and their sum.
template <int TYPE> struct Pair;
template <> struct Pair<TST_BF16> {
    typedef __bf16 entry;
    bf16x2 v;
    __device__ __forceinline__ Pair(entry a, entry b) : v{a, b} {}
    __device__ __forceinline__ float added(float sum) const { return __builtin_amdgcn_fdot2_f32_bf16(v, bf16x2{(entry)1.f, (entry)1.f}, sum, false); }
    __device__ __forceinline__ unsigned bits() const { return __builtin_bit_cast(unsigned, v); }
};
template <> struct Pair<TST_F16> {
    typedef _Float16 entry;
    f16x2 v;
    __device__ __forceinline__ Pair(entry a, entry b) : v{a, b} {}
    __device__ __forceinline__ float added(float sum) const { return __builtin_amdgcn_fdot2(v, f16x2{(entry)1.f, (entry)1.f}, sum, false); }
    __device__ __forceinline__ unsigned bits() const { return __builtin_bit_cast(unsigned, v); }
};

template <int TYPE> __device__ __forceinline__ f32x16 product(u32x4 a, u32x4 b, f32x16 c)
{
    if constexpr (TYPE == TST_F16) return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// The largest of a lane's logits, NaN if one is (what does not care for NaN costs an instruction more for each).
__device__ __forceinline__ float largest_of(const f32x16 &z)
{
    float m = z[0];
#pragma unroll
    for (int r = 1; r < 15; r += 2) m = __builtin_elementwise_maximum(__builtin_elementwise_maximum(m, z[r]), z[r + 1]);
    return __builtin_elementwise_maximum(m, z[15]);
}

// The larger of a value and that of the lane 32 away.
__device__ __forceinline__ float across_max(float v)
{
    auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __builtin_elementwise_maximum(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float across_sum(float v)
{
    auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

template <int TYPE, int ROW, int QB, int NW> struct Shape {
    static constexpr int kPlanes = Planes<TYPE>::kCount;
    static constexpr int kRows = NW * QB * 32;             // of a tile
    static constexpr int kKeys = TYPE == TST_F32 ? 32 : 64;
    static constexpr int kBuffers = TYPE == TST_F32 ? 1 : 2;
    // bytes from key to key: 16 rows of keys, and 4 rows of 32 channels of values, fall into different banks
    static constexpr int kStrideK = ROW * 2 + 16, kStrideV = ROW * 2 + (ROW % 128 == 96 ? 0 : 64);
    static constexpr int kPlaneK = kKeys * kStrideK, kPlaneV = kKeys * kStrideV;
    static constexpr int kBuffer = kPlanes * (kPlaneK + kPlaneV);
    static constexpr int kChunks = (kKeys * (ROW / 8) + 64 * NW - 1) / (64 * NW);   // of 8 entries that a thread stages, of K and as many of V
};

// Weights are 2^shift times those relative to the row's base, which the largest logit may pass by 2^kSlack before all is scaled anew: fp16 holds them with 11 bits
// down to 2^-21 of the largest.
constexpr float kSlack = 8.f;
template <int TYPE> constexpr float kShift = TYPE == TST_F16 ? 7.f : 0.f;

template <int TYPE, int ROW, int QB, int NW> __global__ void __launch_bounds__(64 * NW, V_OCC) k_attention(PromptArgs a)
{
    typedef Shape<TYPE, ROW, QB, NW> S;
    typedef typename Entry<TYPE>::bits Bits;
    constexpr int P = S::kPlanes, kSteps = ROW / 16, kTiles = ROW / 32, kSub = S::kKeys / 32;
    __shared__ __attribute__((aligned(16))) char lds[S::kBuffers * S::kBuffer];
    __shared__ int spoilt[ROW];   // the first key whose value of the channel is not finite, among the keys that some of the tile's rows do not see
    __shared__ int any_spoilt;
    const int wave = uniform(threadIdx.x / 64), lane = threadIdx.x % 64, half = lane / 32, col = lane % 32;
    // tiles of sequence i have the numbers from offsets[i] * group / rows + i on; the last tiles, which see most keys, come first
    const int head = blockIdx.x % a.heads, number = a.tiles - 1 - (int)(blockIdx.x / a.heads);
    int seq = 0;
    {
        auto base = [&](int i) { return (int64_t)min(max(a.offsets[i], 0), a.tokens) * a.group / S::kRows + i; };
        int n = a.sequences;
        while (n > 1) {
            const int step = (n + 63) / 64, i = seq + lane * step;
            const bool before = lane * step < n && base(min(i, a.sequences)) <= number;
            const int c = max(__popcll(__ballot(before)), 1) - 1;
            seq += c * step;
            n = min(step, n - c * step);
        }
        seq = uniform(seq);
    }
    const Span rows = span_of(a.offsets, a.tokens, seq);
    const int tile = number - (int)((int64_t)min(max(a.offsets[seq], 0), a.tokens) * a.group / S::kRows + seq);
    if (tile < 0 || (int64_t)tile * S::kRows >= (int64_t)rows.n * a.group) return;

    const int64_t rho0 = (int64_t)tile * S::kRows;
    const int first_token = (int)(rho0 / a.group), last_token = (int)min((rho0 + S::kRows - 1) / a.group, (int64_t)rows.n - 1);
    const int keys = last_token + 1;          // that the tile sees
    const int tiles = (keys + S::kKeys - 1) / S::kKeys;

    for (int d = threadIdx.x; d < ROW; d += 64 * NW) spoilt[d] = 0x7fffffff;
    if (threadIdx.x == 0) any_spoilt = 0;

    u32x4 q[QB][P][kSteps];
    int limit[QB];     // keys that the row sees
    int token[QB], q_head[QB];
    int least = 0x7fffffff, largest = 0;
#pragma unroll
    for (int b = 0; b < QB; ++b) {
        const int64_t rho = rho0 + (wave * QB + b) * 32 + col;
        const bool there = rho < (int64_t)rows.n * a.group;
        token[b] = there ? (int)(rho / a.group) : -1;
        q_head[b] = head * a.group + (there ? (int)(rho - (int64_t)token[b] * a.group) : 0);
        limit[b] = token[b] + 1;
        if (there) least = min(least, limit[b]), largest = max(largest, limit[b]);
        const Bits *row = static_cast<const Bits *>(a.q.data) + (int64_t)(rows.first + max(token[b], 0)) * a.q.token + q_head[b] * a.q.head;
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            Raw<TYPE> raw = load_raw<TYPE>(row, 16 * s + 8 * half, a.size, there, a.wide);
            if (a.negative) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    if constexpr (TYPE == TST_F32) raw.e[e] = -raw.e[e];
                    else raw.e[e] ^= 0x8000;
                }
            }
            const Planes<TYPE> x = planes_of<TYPE>(raw);
#pragma unroll
            for (int p = 0; p < P; ++p) q[b][p][s] = x.p[p];
        }
    }
    for (int d = 1; d < 32; d <<= 1) least = min(least, __shfl_xor(least, d)), largest = max(largest, __shfl_xor(largest, d));
    least = uniform(least), largest = uniform(largest);

    f32x16 o[QB][kTiles];
    float base[QB], sum[QB];     // logits are relative to base, in powers of two
#pragma unroll
    for (int b = 0; b < QB; ++b) {
        base[b] = -INFINITY, sum[b] = 0.f;
#pragma unroll
        for (int t = 0; t < kTiles; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[b][t][r] = 0.f;
    }

    const Bits *k_data = static_cast<const Bits *>(a.k.data) + (int64_t)rows.first * a.k.token + head * a.k.head;
    const Bits *v_data = static_cast<const Bits *>(a.v.data) + (int64_t)rows.first * a.v.token + head * a.v.head;
    Raw<TYPE> k_raw[S::kChunks], v_raw[S::kChunks];
    auto load = [&](int kt) {
#pragma unroll
        for (int i = 0; i < S::kChunks; ++i) {
            const int c = threadIdx.x + 64 * NW * i, key = kt * S::kKeys + c / (ROW / 8), d = c % (ROW / 8) * 8;
            const bool there = key < keys && c < S::kKeys * (ROW / 8);
            k_raw[i] = load_raw<TYPE>(k_data + (int64_t)min(key, keys - 1) * a.k.token, d, a.size, there, a.wide);
            v_raw[i] = load_raw<TYPE>(v_data + (int64_t)min(key, keys - 1) * a.v.token, d, a.size, there, a.wide);
        }
    };
    auto store = [&](int kt) {
        char *buffer = lds + kt % S::kBuffers * S::kBuffer;
        // values that some rows do not see: 0 times an infinity would be a NaN, so what is not finite is a 0 there and remembered
        if ((kt + 1) * S::kKeys > first_token + 1) {
#pragma unroll
            for (int i = 0; i < S::kChunks; ++i) {
                const int c = threadIdx.x + 64 * NW * i, key = kt * S::kKeys + c / (ROW / 8), d = c % (ROW / 8) * 8;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float x = Entry<TYPE>::get(v_raw[i].e[e]);
                    if (!(x - x == 0.f)) {
                        v_raw[i].e[e] = 0;
                        atomicMin(&spoilt[d + e], key);
                        any_spoilt = 1;
                    }
                }
            }
        }
#pragma unroll
        for (int i = 0; i < S::kChunks; ++i) {
            const int c = threadIdx.x + 64 * NW * i, key = c / (ROW / 8), d = c % (ROW / 8) * 8;
            if (key >= S::kKeys) continue;
            const Planes<TYPE> kp = planes_of<TYPE>(k_raw[i]), vp = planes_of<TYPE>(v_raw[i]);
#pragma unroll
            for (int p = 0; p < P; ++p) {
                *reinterpret_cast<u32x4 *>(buffer + p * S::kPlaneK + key * S::kStrideK + d * 2) = kp.p[p];
                *reinterpret_cast<u32x4 *>(buffer + P * S::kPlaneK + p * S::kPlaneV + key * S::kStrideV + d * 2) = vp.p[p];
            }
        }
    };

    __syncthreads();     // spoilt is clear
    load(0);
    store(0);
    __syncthreads();
    for (int kt = 0; kt < tiles; ++kt) {
        if (kt + 1 < tiles) load(kt + 1);
        const char *buffer = lds + kt % S::kBuffers * S::kBuffer;
        if (kt * S::kKeys < largest) {
            f32x16 z[QB][kSub];
#pragma unroll
            for (int s = 0; s < kSub; ++s) {
#pragma unroll
                for (int b = 0; b < QB; ++b)
#pragma unroll
                    for (int r = 0; r < 16; ++r) z[b][s][r] = 0.f;
#pragma unroll
                for (int step = 0; step < kSteps; ++step) {
                    u32x4 k[P];
#pragma unroll
                    for (int p = 0; p < P; ++p)
                        k[p] = *reinterpret_cast<const u32x4 *>(buffer + p * S::kPlaneK + (s * 32 + col) * S::kStrideK + (16 * step + 8 * half) * 2);
#pragma unroll
                    for (int b = 0; b < QB; ++b)
#pragma unroll
                        for (int p = 0; p < P; ++p)
#pragma unroll
                            for (int r = 0; p + r < P; ++r) z[b][s] = product<TYPE>(k[p], q[b][r][step], z[b][s]);
                }
            }
            const bool cut = (kt + 1) * S::kKeys > least;
            u32x4 w[QB][P][kSub][2];
#pragma unroll
            for (int b = 0; b < QB; ++b) {
                if (cut) {
#pragma unroll
                    for (int s = 0; s < kSub; ++s)
#pragma unroll
                        for (int r = 0; r < 16; ++r)
                            if (kt * S::kKeys + s * 32 + 8 * (r / 4) + 4 * half + r % 4 >= limit[b]) z[b][s][r] = -INFINITY;
                }
                float top = largest_of(z[b][0]);
                if constexpr (kSub == 2) top = __builtin_elementwise_maximum(top, largest_of(z[b][kSub - 1]));
                top = across_max(top) * a.scale;
                if (__any(top > base[b] + kSlack)) {
                    const float now = fmaxf(base[b], top), keep = now == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(base[b] - now);
                    base[b] = now;
                    sum[b] *= keep;
#pragma unroll
                    for (int t = 0; t < kTiles; ++t) o[b][t] *= keep;
                }
                const float from = base[b] == -INFINITY ? 0.f : base[b] - kShift<TYPE>;
                float s_all = 0.f;
#pragma unroll
                for (int s = 0; s < kSub; ++s) {
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        z[b][s][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(z[b][s][r], a.scale, -from));
                        if constexpr (TYPE == TST_F32) s_all += z[b][s][r];
                    }
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        if constexpr (TYPE == TST_F32) {
                            Raw<TYPE> x;
#pragma unroll
                            for (int i = 0; i < 8; ++i) x.e[i] = z[b][s][8 * j + i];
                            const Planes<TYPE> px = planes_of<TYPE>(x);
#pragma unroll
                            for (int p = 0; p < P; ++p) w[b][p][s][j] = px.p[p];
                        } else {
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const Pair<TYPE> pair = {(typename Pair<TYPE>::entry)z[b][s][8 * j + 2 * i], (typename Pair<TYPE>::entry)z[b][s][8 * j + 2 * i + 1]};
                                s_all = pair.added(s_all);
                                w[b][0][s][j][i] = pair.bits();
                            }
                        }
                    }
                }
                sum[b] += s_all;
            }
            // four keys of a lane's channel: in each group of 16 lanes, lanes 4 r .. 4 r + 3 point to 16 channels of the r-th key
            const char *v_at = buffer + P * S::kPlaneK + (4 * half + lane % 16 / 4) * S::kStrideV + (col / 16 * 16 + lane % 4 * 4) * 2;
#pragma unroll
            for (int s = 0; s < kSub; ++s)
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int t = 0; t < kTiles; ++t) {
                        u32x4 v[P];
#pragma unroll
                        for (int p = 0; p < P; ++p) {
                            u32x2 part[2];
#pragma unroll
                            for (int i = 0; i < 2; ++i) {
                                const char *at = v_at + p * S::kPlaneV + (s * 32 + 16 * j + 8 * i) * S::kStrideV + t * 64;
                                part[i] = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)at));
                            }
                            v[p] = u32x4{part[0][0], part[0][1], part[1][0], part[1][1]};
                        }
#pragma unroll
                        for (int b = 0; b < QB; ++b)
#pragma unroll
                            for (int p = 0; p < P; ++p)
#pragma unroll
                                for (int r = 0; p + r < P; ++r) o[b][t] = product<TYPE>(v[p], w[b][r][s][j], o[b][t]);
                    }
        }
        if (S::kBuffers == 1) __syncthreads();   // everybody has read the only buffer
        if (kt + 1 < tiles) store(kt + 1);
        __syncthreads();
    }

    const bool bad = any_spoilt;
#pragma unroll
    for (int b = 0; b < QB; ++b) {
        if (token[b] < 0) continue;
        const float inverse = 1.f / across_sum(sum[b]);
        Bits *out = static_cast<Bits *>(a.y) + ((int64_t)(rows.first + token[b]) * a.q_heads + q_head[b]) * a.size;
        const bool whole = (a.size & 3) == 0 && ((uintptr_t)a.y & (4 * sizeof(Bits) - 1)) == 0;
#pragma unroll
        for (int t = 0; t < kTiles; ++t)
#pragma unroll
            for (int r = 0; r < 16; r += 4) {
                const int d = 32 * t + 2 * r + 4 * half;
                Bits four[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) four[e] = Entry<TYPE>::put(bad && spoilt[d + e] < limit[b] ? kNan : o[b][t][r + e] * inverse);
                if (whole) {
                    if (d < a.size) __builtin_memcpy(__builtin_assume_aligned(out + d, 4 * sizeof(Bits)), four, sizeof(four));
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (d + e < a.size) out[d + e] = four[e];
                }
            }
    }
}

bool wide(const Rows &x, int type, int size)
{
    const int64_t per = 16 / (int64_t)type_bytes(type);
    return aligned(x.data, 16) && x.token % per == 0 && x.head % per == 0 && size % 8 == 0;
}

}  // namespace
}  // namespace tst

extern "C" {

int tst_attention(const tst_heads_t *Q, const tst_heads_t *K, const tst_heads_t *V, int type, int q_heads, int heads, int head_size, const int32_t *offsets,
                  int sequences, int tokens, float scale, void *Y, void *stream)
{
    if (!tst::type_ok(type) || heads < 1 || q_heads < heads || q_heads > TST_MAX_HEADS || q_heads % heads || head_size < 1 || head_size > TST_MAX_HEAD_SIZE || sequences < 0 ||
        sequences > TST_MAX_SEQUENCES || tokens < 0 || tokens > TST_MAX_TOKENS || (int64_t)tokens * q_heads > TST_MAX_ROWS || !(scale - scale == 0.f))
        return TSTGEMM_EINVAL;
    if (sequences == 0 || tokens == 0) return TSTGEMM_OK;
    if (!tst::rows_ok(Q, type) || !tst::rows_ok(K, type) || !tst::rows_ok(V, type) || !offsets || !tst::aligned(offsets, 4) || !Y || !tst::aligned(Y, tst::type_bytes(type)))
        return TSTGEMM_EINVAL;
    const int group = q_heads / heads;
    tst::PromptArgs a{tst::rows_of(Q), tst::rows_of(K), tst::rows_of(V), q_heads, heads, group, head_size, sequences, tokens, 0, offsets, std::fmax(std::fabs(scale) * tst::kLog2e, 1.17549435e-38f), scale < 0, Y, false};
    a.wide = tst::wide(a.q, type, head_size) && tst::wide(a.k, type, head_size) && tst::wide(a.v, type, head_size);
    return tst::status(tst::for_type(type, [&](auto t) {
        return tst::for_row(head_size, [&](auto r) {
            constexpr int TYPE = decltype(t)::value, ROW = decltype(r)::value, QB = V_QB, NW = V_NW;
            a.tiles = (int)((int64_t)tokens * group / tst::Shape<TYPE, ROW, QB, NW>::kRows) + sequences;
            tst::k_attention<TYPE, ROW, QB, NW><<<(unsigned)a.tiles * heads, 64 * NW, 0, static_cast<hipStream_t>(stream)>>>(a);
            return hipGetLastError();
        });
    }));
}

}  // extern "C"
