// A mixture-of-experts feed-forward layer for a few tokens (tst_moe): the router, the top experts of each token, and the experts'
// products from 8-bit weights.
//
// Weights meet the matrix cores as bf16, which holds every 8-bit code exactly.  The activations are cut into bf16 planes by cutting
// mantissas off (x = p0 + p1 + p2, p0 the upper 16 bits of x, p1 those of x - p0, ...): one plane holds a bf16 entry, two an fp16
// entry, three an fp32 entry, all exactly, so that products are exact and only the fp32 sums round.
//
// The tokens that chose an expert are the columns of a matrix instruction, 16 at a time, and the weights its rows: up to 16 tokens cost
// the matrix cores the same.  Columns without a token hold anything and are not used; a column's values stay in it.
#include "ops_internal.h"

namespace tst {
namespace {

constexpr int kMaxTokens = 64;   // of one launch; more go in slabs
constexpr int kMaxE = TST_MOE_MAX_EXPERTS, kMaxTop = TST_MOE_MAX_TOP;

// Activations as operands: for each 64 rows of a product and plane two operands of the matrix instruction, in each 16 bytes for a quarter of
// the rows and a token, [block][plane][half][quarter][token][8 bf16], the row being 64 block + 16 quarter + 8 half + i, as in the pieces
// of the weights.  Neighbouring lanes read neighbouring tokens.
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
    bool normalize, wide;   // wide: rows of X and of the router can be loaded 16 bytes at a time
    // workspace
    float *logits;   // [T][E]
    u32x4 *x;        // operands of X, zero behind D
    u32x4 *h;        // operands of h, a row for each token and expert it chose, zero behind F
    int32_t *count;  // experts in use
    int32_t *used;   // they, ascending
    uint16_t *members;   // [nth][16 NT] of the nth expert in use, as in Chosen
    float *partial;  // [split][T][D]
    int splits;
};

constexpr int planes_of(int type) { return type == TST_F32 ? 3 : type == TST_F16 ? 2 : 1; }
// h keeps the 24 bits that it is computed with, whatever the type: with two planes (16 bits) results of 16 bits are off by single last places
// more often than the fp32 sums alone make them.  It costs a token 1 us of 73, 16 tokens 2 of 74, 64 tokens on 8 experts of 4096 x 11008 45 of 389.
constexpr int kHPlanes = 3;
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
// k_moe_router: a wavefront per (token, expert) for the logits, and workgroups behind these for the operands of X.  Bound by latency: 4.6 us for 16 tokens and 64 experts
// of width 2048.
constexpr int kRouterWaves = 4;

template <int TYPE, bool WIDE>
__global__ void __launch_bounds__(kRouterWaves * 64)
k_moe_router(const MoeArgs a)
{
    typedef Entry<TYPE> E;
    typedef typename E::bits bits;
    constexpr int V = WIDE ? 16 / sizeof(bits) : 1;
    typedef bits piece __attribute__((ext_vector_type(V)));
    const int t = blockIdx.y, lane = threadIdx.x & 63, e = blockIdx.x * kRouterWaves + (threadIdx.x >> 6);
    const bits *x = static_cast<const bits *>(a.X) + t * a.x_stride;
    const int logit_groups = blocks_of(a.E, kRouterWaves);
    if ((int)blockIdx.x < logit_groups) {
        if (e >= a.E) return;
        const bits *r = static_cast<const bits *>(a.router) + (size_t)e * a.D;
        float sum = 0.f;
#pragma unroll 8
        for (int d = lane * V; d < a.D; d += 64 * V) {   // (WIDE: D is a multiple of V)
            const piece xv = *reinterpret_cast<const piece *>(x + d), rv = *reinterpret_cast<const piece *>(r + d);
#pragma unroll
            for (int i = 0; i < V; ++i) sum = fmaf(E::get(xv[i]), E::get(rv[i]), sum);
        }
        sum = wave_sum(sum);
        if (lane == 0) a.logits[t * a.E + e] = sum;
        return;
    }
    constexpr int P = planes_of(TYPE);
    const int unit = ((int)blockIdx.x - logit_groups) * kRouterWaves * 64 + threadIdx.x;
    if (unit < pad64(a.D) / 8) {
        const int d = unit * 8, kb = unit >> 3, quarter = (unit >> 1) & 3, half = unit & 1;
        uint16_t out[P][8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float v = d + i < a.D ? E::get(x[d + i]) : 0.f;
#pragma unroll
            for (int p = 0; p < P; ++p) out[p][i] = cut(v);
        }
#pragma unroll
        for (int p = 0; p < P; ++p) {
            u32x4 o;
#pragma unroll
            for (int i = 0; i < 4; ++i) o[i] = out[p][2 * i] | (unsigned)out[p][2 * i + 1] << 16;
            a.x[(size_t)(((kb * P + p) * 2 + half) * 4 + quarter) * a.T + t] = o;
        }
    }
}

// ------------------------------------------------------------------------------------------------------------------
// Which tokens chose which expert, in the LDS behind the workgroup's own: the members of expert e, their tokens ascending, stand in
// of(e, 0), of(e, 1), ... as token | rank of e among the token's << 8, and kNobody behind the last.
constexpr unsigned kNobody = 0xffff;
__device__ __forceinline__ int token_of(unsigned member) { return member & 0xff; }
__device__ __forceinline__ int rank_of(unsigned member) { return member >> 8; }

template <int NT> struct Chosen {
    static constexpr int kTokens = 16 * NT;
    uint16_t *members;  // [E][kTokens]; while they are chosen, entry t is token t's
    float *p;           // [T][top]
    uint16_t *active;   // experts that some token chose, ascending
    __device__ Chosen(char *lds, const MoeArgs &a)
        : members(reinterpret_cast<uint16_t *>(lds)), p(reinterpret_cast<float *>(members + a.E * kTokens)),
          active(reinterpret_cast<uint16_t *>(p + a.T * a.top))
    {
    }
    static size_t bytes(const MoeArgs &a) { return (size_t)a.E * kTokens * sizeof(uint16_t) + (size_t)a.T * a.top * sizeof(float) + (size_t)a.E * sizeof(uint16_t); }
    __device__ unsigned of(int e, int i) const { return members[e * kTokens + i]; }
};

// A wavefront finds a token's experts: top rounds of the largest of what is left; lane l holds experts l, l + 64, ...
template <int PER, int NT>
__device__ void choose_experts(const MoeArgs &a, const Chosen<NT> &c, int t, int lane, bool write)
{
    float l[PER];
    unsigned key[PER];   // 0: none (left)
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int e = lane + 64 * i;
        l[i] = e < a.E ? a.logits[t * a.E + e] : -INFINITY;
        key[i] = e < a.E ? order_bits(l[i]) : 0;
    }
    float most = 0.f, all = 0.f, chosen = 0.f, mine = 0.f;
    for (int j = 0; j < a.top; ++j) {
        unsigned best = key[0];
#pragma unroll
        for (int i = 1; i < PER; ++i) best = max(best, key[i]);
        best = wave_max(best);
        int e = -1;   // the lowest that has it
        float value = 0.f;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const unsigned long long have = __ballot(key[i] == best);
            if (e < 0 && have) {
                const int at = __builtin_ctzll(have);
                e = at + 64 * i;
                value = __uint_as_float(__builtin_amdgcn_readlane((int)__float_as_uint(l[i]), at));
                if (lane == at) key[i] = 0;
            }
        }
        if (j == 0) {
            most = value;
            if (!a.normalize) {
#pragma unroll
                for (int i = 0; i < PER; ++i)
                    if (lane + 64 * i < a.E) all += expf(l[i] - most);
                all = wave_sum(all);
            }
        }
        const float w = expf(value - most);
        chosen += w;
        if (lane == j) mine = w;
        if (lane == 0) {
            c.members[e * c.kTokens + t] = (uint16_t)(t | j << 8);
            if (write) a.ids[t * a.top + j] = e;
        }
    }
    if (lane < a.top) {
        const float p = mine / (a.normalize ? chosen : all);
        c.p[t * a.top + lane] = p;
        if (write) a.p[t * a.top + lane] = p;
    }
}

template <int NT> __device__ __forceinline__ void clear_members(const MoeArgs &a, const Chosen<NT> &c)
{
    unsigned *w = reinterpret_cast<unsigned *>(c.members);
    for (int i = threadIdx.x; i < a.E * c.kTokens / 2; i += blockDim.x) w[i] = 0xffffffffu;
    __syncthreads();
}

// The list of experts in use, which every wavefront counts and the first one writes down, and each expert's members moved together.
template <int NT> __device__ int list_active(const MoeArgs &a, const Chosen<NT> &c)
{
    int n = 0;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    for (int e0 = 0; e0 < a.E; e0 += 64) {
        const int e = e0 + lane;
        bool any = false;
        if (e < a.E) {
            const u32x4 *w = reinterpret_cast<const u32x4 *>(c.members + e * c.kTokens);
#pragma unroll
            for (int i = 0; i < 2 * NT; ++i) any |= (w[i][0] & w[i][1] & w[i][2] & w[i][3]) != 0xffffffffu;
        }
        const unsigned long long set = __ballot(any);
        if (any && wave == 0) c.active[n + __popcll(set & ((1ull << lane) - 1))] = (uint16_t)e;
        n += __popcll(set);
    }
    __syncthreads();
    for (int i = wave; i < n; i += waves) {
        uint16_t *row = c.members + c.active[i] * c.kTokens;
        const unsigned m = lane < c.kTokens ? row[lane] : kNobody;
        const unsigned long long set = __ballot(m != kNobody);
        if (m != kNobody) row[__popcll(set & ((1ull << lane) - 1))] = (uint16_t)m;   // (all have read; never behind where it stood)
        if (lane < c.kTokens && lane >= __popcll(set)) row[lane] = kNobody;
    }
    __syncthreads();
    return n;
}

// Sixteen 8-bit weights of a lane as two operands of the bf16 matrix instruction: 1.5 instructions a weight.
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

// A meeting of the workgroup that orders the LDS alone: loads on their way stay there.
__device__ __forceinline__ void meet()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// ------------------------------------------------------------------------------------------------------------------
// k_moe_up: h = silu(x gate) (x up) p for each token and expert it chose, as operands.  Every workgroup finds the experts by itself;
// the first one writes them out.  An item of work is one expert x 16 columns of its gate and up, for all tokens; wavefronts share D
// and hold U blocks of it on the way: a block's registers are loaded again, for the round or the item to come, as soon as it is used.
// Bound by the weights' bytes: one token, two experts of 4096 x 11008 (180 MB) 36.2 us, 5.0 TB/s; 16 tokens, 64 experts of 2048 x 1024, 4
// each (some 170 MB) 36.  More tokens are not: 64 of them on all 64 experts (268 MB) 98 us, in fp32 on 128 of 2048 x 768 (403 MB) 262: every workgroup
// chooses for all tokens before it asks for a weight, and tiles of members behind the second ask for X when they need it.
constexpr int kUpWaves = 8;

template <int TYPE, int NT>
__global__ void __launch_bounds__(kUpWaves * 64, NT == 1 || planes_of(TYPE) == 1 ? 4 : 2)
k_moe_up(const MoeArgs a)
{
    constexpr int P = planes_of(TYPE), PH = kHPlanes;
    constexpr int AHEAD = NT == 1 ? 1 : 2;   // tiles of members whose X is requested ahead; few experts have more
    constexpr int U = NT == 1 ? (P == 1 ? 4 : 2) : NT == 4 && P == 1 ? 2 : 3;
    __shared__ f32x4 part[2][kUpWaves][2][64];
    extern __shared__ u32x4 lds_behind[];
    const Chosen<NT> c(reinterpret_cast<char *>(lds_behind), a);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    clear_members(a, c);
    for (int t = wave; t < a.T; t += kUpWaves) {
        if (a.E <= 64) choose_experts<1>(a, c, t, lane, blockIdx.x == 0);
        else choose_experts<kMaxE / 64>(a, c, t, lane, blockIdx.x == 0);
    }
    __syncthreads();
    const int k_blocks = pad64(a.D) / 64, cols = pad64(a.F) / 16, real_cols = blocks_of(a.F, kW8Cols);
    const int n_active = list_active(a, c), items = n_active * cols, rounds = blocks_of(k_blocks, kUpWaves * U);
    const unsigned column = k_blocks * kW8Piece;

    struct Block {
        u32x4 gate, up, x[P][2][AHEAD];
    } block[U];
    // Block u of a round of an item; blocks that are not there (behind D, of padded columns, of no item) are left as they are
    // and not multiplied.
    auto there = [&](int item, int round, int u) {
        return item < items && item % cols < real_cols && (round * U + u) * kUpWaves + wave < k_blocks;
    };
    auto operand = [&](int kb, int p, int s, unsigned m) { return a.x[(size_t)(((kb * P + p) * 2 + s) * 4 + (lane >> 4)) * a.T + token_of(m)]; };
    auto load = [&](int item, int round, int u, Block &b) {
        if (!there(item, round, u)) return;
        const int e = __builtin_amdgcn_readfirstlane(c.active[item / cols]), kb = (round * U + u) * kUpWaves + wave;
        const size_t at = ((size_t)e * real_cols + item % cols) * column + (size_t)kb * kW8Piece + lane * 16;
        b.gate = *reinterpret_cast<const u32x4 *>(a.gate + at);
        b.up = *reinterpret_cast<const u32x4 *>(a.up + at);
#pragma unroll
        for (int t = 0; t < AHEAD; ++t) {
            const unsigned m = c.of(e, 16 * t + (lane & 15));
#pragma unroll
            for (int p = 0; p < P; ++p)
#pragma unroll
                for (int s = 0; s < 2; ++s)
                    if (m != kNobody) b.x[p][s][t] = operand(kb, p, s, m);   // the other columns are not used, whatever they hold
        }
    };
#pragma unroll
    for (int u = 0; u < U; ++u) {
        block[u] = Block{};
        load(blockIdx.x, 0, u, block[u]);
    }
    if (blockIdx.x == gridDim.x - 1) {   // for k_moe_down
        if (threadIdx.x == 0) *a.count = n_active;
        for (int i = threadIdx.x; i < n_active; i += kUpWaves * 64) a.used[i] = c.active[i];
        for (int i = threadIdx.x; i < n_active * c.kTokens; i += kUpWaves * 64) a.members[i] = (uint16_t)c.of(c.active[i / c.kTokens], i % c.kTokens);
    }
    // h of a tile of members and an item, from the sums of the wavefronts.
    auto finish = [&](int item, int t, int buffer) {
        const int e = c.active[item / cols], nb = item % cols;
        const unsigned m = c.of(e, 16 * t + (lane & 15));
        if (m == kNobody) return;
        const int row = token_of(m) * a.top + rank_of(m);
        f32x4 g = part[buffer][0][0][lane], u = part[buffer][0][1][lane];
#pragma unroll
        for (int w = 1; w < kUpWaves; ++w) {
            g += part[buffer][w][0][lane];
            u += part[buffer][w][1][lane];
        }
        const int f = nb * 16 + 4 * (lane >> 4);
        uint16_t out[PH][4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            float h = 0.f;
            if (f + r < a.F) {
                const float gv = g[r] * a.gate_scale[(size_t)e * a.F + f + r], uv = u[r] * a.up_scale[(size_t)e * a.F + f + r];
                h = gv / (1.f + expf(-gv)) * uv * c.p[row];
            }
#pragma unroll
            for (int p = 0; p < PH; ++p) out[p][r] = p < PH - 1 ? cut(h) : Entry<TST_BF16>::put(h);   // the last one rounds
        }
        const int kb = f >> 6, quarter = (f >> 4) & 3, half = (f >> 3) & 1;
#pragma unroll
        for (int p = 0; p < PH; ++p) {
            u32x4 *to = a.h + (size_t)(((kb * PH + p) * 2 + half) * 4 + quarter) * (a.T * a.top) + row;
            reinterpret_cast<u32x2 *>(to)[(f >> 2) & 1] = u32x2{out[p][0] | (unsigned)out[p][1] << 16, out[p][2] | (unsigned)out[p][3] << 16};
        }
    };
    int buffer = 0;
    for (int item = blockIdx.x; item < items; item += gridDim.x) {
        f32x4 acc[2][NT] = {};
        int tiles = 1;   // of 16 members
#pragma unroll
        for (int t = 1; t < NT; ++t)
            if (__builtin_amdgcn_readfirstlane((int)c.of(c.active[item / cols], 16 * t)) != (int)kNobody) tiles = t + 1;
        for (int round = 0; round < rounds; ++round) {
            const bool last = round == rounds - 1;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                Block &b = block[u];
                if (there(item, round, u)) {
                    bf16x8 wg[2], wu[2];
                    widen(b.gate, wg);
                    widen(b.up, wu);
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        if (t >= tiles) break;
                        const unsigned m = t < AHEAD ? 0 : c.of(c.active[item / cols], 16 * t + (lane & 15));
#pragma unroll
                        for (int p = 0; p < P; ++p)
#pragma unroll
                            for (int s = 0; s < 2; ++s) {
                                u32x4 x = {};
                                if (t < AHEAD) x = b.x[p][s][t < AHEAD ? t : 0];
                                else if (m != kNobody) x = operand((round * U + u) * kUpWaves + wave, p, s, m);
                                const bf16x8 xf = __builtin_bit_cast(bf16x8, x);
                                acc[0][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wg[s], xf, acc[0][t], 0, 0, 0);
                                acc[1][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wu[s], xf, acc[1][t], 0, 0, 0);
                            }
                    }
                }
                load(last ? item + gridDim.x : item, last ? 0 : round + 1, u, b);
            }
        }
#pragma unroll
        for (int t = 0; t < NT; ++t) {   // a tile of members after another, through two buffers: what stands in one was read before the
            if (t >= tiles) break;       // meeting that lets the other be read
            part[buffer][wave][0][lane] = acc[0][t];
            part[buffer][wave][1][lane] = acc[1][t];
            meet();
            if (wave == 0) finish(item, t, buffer);
            buffer ^= 1;
        }
    }
}

// ------------------------------------------------------------------------------------------------------------------
// k_moe_down: 64 columns of Y for all tokens.  The blocks of all experts in use, one expert behind another, are shared by the workgroups of
// a split and their wavefronts, each with a run of them and U on the way.  Four pieces of weights use one operand of h, which
// comes from the L2: with 16 columns the registers of h on its way left too few for the weights (86 MB of weights 41 us; now 20.7, 4.2 TB/s).
// 64 tokens: 134 MB 52 us, 361 MB (8 experts of 4096 x 11008) 194.
// Between experts a wavefront scales its sums with the expert's channels and adds them to those of the token.
constexpr int kDownCols = 4;   // pieces of 16
constexpr int kDownWaves = 8;

template <int TYPE, int NT>
__global__ void __launch_bounds__(kDownWaves * 64, 2)
k_moe_down(const MoeArgs a)
{
    typedef Entry<TYPE> E;
    constexpr int PH = kHPlanes, U = NT == 1 ? 3 : NT == 2 ? 2 : 1;
    constexpr int AHEAD = NT > 1 ? 2 : 1;   // tiles of members whose h is requested ahead; few experts have more
    __shared__ f32x4 part[kDownWaves][kDownCols][NT][64];   // of the experts that a wavefront is done with
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int split = blockIdx.y, nb0 = blockIdx.x * kDownCols;
    const int k_blocks = pad64(a.F) / 64, n_blocks = blocks_of(a.D, kW8Cols);
    const int total = *a.count * k_blocks, share = blocks_of(total, kDownWaves * a.splits);
    const int begin = min((split * kDownWaves + wave) * share, total), end = min(begin + share, total);

    struct Block {
        u32x4 w[kDownCols], h[PH][2][AHEAD];
        int kb;
    } block[U];
    int e = 0, kb = 0, next = begin, row[AHEAD];   // of the block to be requested next; row: of h, or -1
    auto enter = [&](int nth) {
        e = __builtin_amdgcn_readfirstlane(a.used[nth]);
#pragma unroll
        for (int t = 0; t < AHEAD; ++t) {
            const unsigned m = a.members[nth * 16 * NT + 16 * t + (lane & 15)];
            row[t] = m == kNobody ? -1 : token_of(m) * a.top + rank_of(m);
        }
    };
    auto operand = [&](int kb, int p, int s, int row) { return a.h[(size_t)(((kb * PH + p) * 2 + s) * 4 + (lane >> 4)) * (a.T * a.top) + row]; };
    auto load = [&](Block &b) {
        if (next >= end) return;
#pragma unroll
        for (int j = 0; j < kDownCols; ++j)
            b.w[j] = *reinterpret_cast<const u32x4 *>(a.down + (((size_t)e * n_blocks + min(nb0 + j, n_blocks - 1)) * k_blocks + kb) * kW8Piece + lane * 16);
        b.kb = kb;
#pragma unroll
        for (int t = 0; t < AHEAD; ++t)
#pragma unroll
            for (int p = 0; p < PH; ++p)
#pragma unroll
                for (int s = 0; s < 2; ++s)
                    if (row[t] >= 0) b.h[p][s][t] = operand(kb, p, s, row[t]);
        ++next;
        if (++kb == k_blocks && next < end) {
            kb = 0;
            enter(next / k_blocks);
        }
    };
    f32x4 acc[kDownCols][NT] = {};
    int left = 0, nth = 0, tiles = 1;   // the expert whose sums are in acc: its blocks to come, its tiles of 16 members
    auto count_tiles = [&]() {
        tiles = 1;
#pragma unroll
        for (int t = 1; t < NT; ++t)
            if (a.members[(nth * NT + t) * 16] != kNobody) tiles = t + 1;
    };
    if (begin < end) {
        nth = begin / k_blocks;
        kb = begin % k_blocks;
        left = k_blocks - kb;
        enter(nth);
        count_tiles();
    }
    auto settle = [&]() {
        order_wave();   // a token's sums were written by the lane that had its column before
        const float *scale = a.down_scale + (size_t)a.used[nth] * a.D;
#pragma unroll
        for (int j = 0; j < kDownCols; ++j) {
            float by[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) by[r] = scale[min((nb0 + j) * 16 + 4 * (lane >> 4) + r, a.D - 1)];
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                if (t >= tiles) break;
                const unsigned m = a.members[nth * 16 * NT + 16 * t + (lane & 15)];
                if (m != kNobody) {
                    f32x4 &v = part[wave][j][token_of(m) >> 4][(lane & 48) | (token_of(m) & 15)];
#pragma unroll
                    for (int r = 0; r < 4; ++r) v[r] = fmaf(by[r], acc[j][t][r], v[r]);
                }
                acc[j][t] = f32x4{};
            }
        }
    };
#pragma unroll
    for (int j = 0; j < kDownCols; ++j)
#pragma unroll
        for (int t = 0; t < NT; ++t) part[wave][j][t][lane] = f32x4{};
#pragma unroll
    for (int u = 0; u < U; ++u) load(block[u]);
    for (int at = begin; at < end; at += U) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            Block &b = block[u];
            if (at + u >= end) break;
            bf16x8 wd[kDownCols][2];
#pragma unroll
            for (int j = 0; j < kDownCols; ++j) widen(b.w[j], wd[j]);
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                if (t >= tiles) break;
                const unsigned m = t < AHEAD ? 0 : a.members[nth * 16 * NT + 16 * t + (lane & 15)];
#pragma unroll
                for (int p = 0; p < PH; ++p)
#pragma unroll
                    for (int s = 0; s < 2; ++s) {
                        u32x4 h = {};
                        if (t < AHEAD) h = b.h[p][s][t < AHEAD ? t : 0];
                        else if (m != kNobody) h = operand(b.kb, p, s, token_of(m) * a.top + rank_of(m));
#pragma unroll
                        for (int j = 0; j < kDownCols; ++j)
                            acc[j][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wd[j][s], __builtin_bit_cast(bf16x8, h), acc[j][t], 0, 0, 0);
                    }
            }
            load(b);
            if (--left == 0) {
                settle();
                left = k_blocks;
                if (at + u + 1 < end) {
                    ++nth;
                    count_tiles();
                }
            }
        }
    }
    if (begin < end && left != k_blocks) settle();   // an expert that others go on with
    __syncthreads();
    for (int i = threadIdx.x; i < kDownCols * NT * 64; i += kDownWaves * 64) {
        const int l = i & 63, t = (i >> 6) % NT, j = (i >> 6) / NT, token = 16 * t + (l & 15);
        if (token >= a.T) continue;
        f32x4 y = part[0][j][t][l];
#pragma unroll
        for (int w = 1; w < kDownWaves; ++w) y += part[w][j][t][l];
        const int d = (nb0 + j) * 16 + 4 * (l >> 4);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            if (d + r >= a.D) continue;
            if (a.splits == 1) static_cast<typename E::bits *>(a.Y)[(size_t)token * a.D + d + r] = E::put(y[r]);
            else a.partial[((size_t)split * a.T + token) * a.D + d + r] = y[r];
        }
    }
}

// k_moe_join: the sums of the splits, in their order (4.7 us, latency; without splits a quarter of the compute units would do the second
// product).
constexpr int kJoinThreads = 256;

template <int TYPE>
__global__ void __launch_bounds__(kJoinThreads)
k_moe_join(const MoeArgs a)
{
    typedef Entry<TYPE> E;
    const int i = blockIdx.x * kJoinThreads + threadIdx.x, n = a.T * a.D;   // (T <= 64, D < 2^17)
    if (i >= n) return;
    float y = a.partial[i];
#pragma unroll 16
    for (int s = 1; s < a.splits; ++s) y += a.partial[(size_t)s * n + i];
    static_cast<typename E::bits *>(a.Y)[i] = E::put(y);
}

// Workgroups that share the experts of a column tile, so that every compute unit has one where D reaches 1024 (kMaxSplits); each has at least one
// block for a wavefront.  us of whole calls as chosen, with one and with 4, bf16: one token, 2 of 8 experts 4096 x 11008 72 90 73; 16 tokens,
// 4 of 64 experts 2048 x 1024 74 133 81; 4 tokens, 6 of 64 42 67 44; 16 tokens, 2 of 16 experts 1024 x 4096 68 165 84.
constexpr int kMaxSplits = 16;
int most_splits(int D)
{
    const int wanted = blocks_of(compute_units(), blocks_of(D, 16 * kDownCols));
    return wanted < kMaxSplits ? wanted : kMaxSplits;
}
int down_splits(int T, int D, int F, int top)
{
    const int64_t blocks = (int64_t)blocks_of(F, 64) * (T < 4 ? top : 2 * top);   // (experts in use are not known here)
    const int64_t useful = (blocks + kDownWaves - 1) / kDownWaves;
    return useful < most_splits(D) ? (int)useful : most_splits(D);
}

struct MoeSpace {
    size_t logits, x, h, count, used, members, partial, total;
};
MoeSpace moe_space(const tst_moe_t &m, int T, int top)
{
    MoeSpace s{};
    if (T > kMaxTokens) T = kMaxTokens;
    auto take = [&](size_t &at, size_t bytes) {
        at = s.total;
        s.total += round256(bytes);
    };
    const size_t in_use = (size_t)m.experts < (size_t)T * top ? m.experts : (size_t)T * top;
    take(s.logits, (size_t)T * m.experts * sizeof(float));
    take(s.x, (size_t)planes_of(m.type) * T * pad64(m.width) * 2);
    take(s.h, (size_t)kHPlanes * T * top * pad64(m.inner) * 2);
    take(s.count, sizeof(int32_t));
    take(s.used, in_use * sizeof(int32_t));
    take(s.members, in_use * kMaxTokens * sizeof(uint16_t));
    take(s.partial, most_splits(m.width) > 1 ? (size_t)most_splits(m.width) * T * m.width * sizeof(float) : 0);
    return s;
}

template <int TYPE, int NT> hipError_t launch_moe_nt(const MoeArgs &a, hipStream_t stream)
{
    const dim3 router(blocks_of(a.E, kRouterWaves) + blocks_of(pad64(a.D) / 8, kRouterWaves * 64), a.T);
    if (a.wide) k_moe_router<TYPE, true><<<router, kRouterWaves * 64, 0, stream>>>(a);
    else k_moe_router<TYPE, false><<<router, kRouterWaves * 64, 0, stream>>>(a);
    if (hipError_t e = hipGetLastError()) return e;
    // Two workgroups of k_moe_up for each compute unit, also where registers (16 tokens and more in fp32 or fp16) or the LDS (hundreds of experts) hold
    // one: the others start when the first are done.
    const size_t lds = Chosen<NT>::bytes(a);
    const int64_t items = (int64_t)(a.E < a.T * a.top ? a.E : a.T * a.top) * (pad64(a.F) / 16), groups = 2 * (int64_t)compute_units();
    k_moe_up<TYPE, NT><<<(unsigned)(items < groups ? items : groups), kUpWaves * 64, lds, stream>>>(a);
    if (hipError_t e = hipGetLastError()) return e;
    k_moe_down<TYPE, NT><<<dim3(blocks_of(a.D, 16 * kDownCols), a.splits), kDownWaves * 64, 0, stream>>>(a);
    if (a.splits > 1) {
        if (hipError_t e = hipGetLastError()) return e;
        k_moe_join<TYPE><<<blocks_of(a.T * a.D, kJoinThreads), kJoinThreads, 0, stream>>>(a);
    }
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
    const int piece = (int)(16 / entry);
    const bool wide = tst::aligned(X, 16) && tst::aligned(m.router, 16) && x_stride % piece == 0 && m.width % piece == 0;
    for (int64_t t0 = 0; t0 < T; t0 += tst::kMaxTokens) {
        const int n = (int)(T - t0 < tst::kMaxTokens ? T - t0 : tst::kMaxTokens);
        const tst::MoeArgs a{static_cast<const char *>(X) + t0 * x_stride * entry, x_stride, m.router, static_cast<const char *>(m.gate),
                             static_cast<const char *>(m.up), static_cast<const char *>(m.down), m.gate_scale, m.up_scale, m.down_scale,
                             static_cast<char *>(Y) + t0 * m.width * entry, ids + t0 * top_k, p + t0 * top_k, m.experts, m.width, m.inner, n,
                             top_k, normalize != 0, wide, reinterpret_cast<float *>(ws + s.logits), reinterpret_cast<tst::u32x4 *>(ws + s.x),
                             reinterpret_cast<tst::u32x4 *>(ws + s.h), reinterpret_cast<int32_t *>(ws + s.count), reinterpret_cast<int32_t *>(ws + s.used),
                             reinterpret_cast<uint16_t *>(ws + s.members), reinterpret_cast<float *>(ws + s.partial),
                             tst::down_splits(n, m.width, m.inner, top_k)};
        const hipError_t e = tst::for_type(m.type, [&](auto type) {
            constexpr int TYPE = decltype(type)::value;
            hipStream_t st = static_cast<hipStream_t>(stream);
            // tiles of tokens: 16 tokens with 1, 2 and 4 of them 74 75 79 us (bf16, 4 of 64 experts 2048 x 1024) and 85 104 106 (fp32), 32 tokens with
            // 2 and 4 115 and 118, 170 and 172
            return n <= 16 ? tst::launch_moe_nt<TYPE, 1>(a, st) : n <= 32 ? tst::launch_moe_nt<TYPE, 2>(a, st) : tst::launch_moe_nt<TYPE, 4>(a, st);
        });
        if (e != hipSuccess) return TSTGEMM_EHIP;
    }
    return TSTGEMM_OK;
}

}  // extern "C"
