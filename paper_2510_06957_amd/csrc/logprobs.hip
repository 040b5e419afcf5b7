// Log probabilities of given tokens, entropy and the top alternatives of rows of logits (tst_logprobs).
//
// One pass over the logits.  A row, or a split of one where there are few rows, belongs to a workgroup, whose wavefronts take it in chunks
// that their lanes hold in registers, each for itself: nobody waits for anybody before the end.  A lane keeps a running maximum m,
// sum e^(z - m) and sum e^(z - m) (z - m).  The alternatives come from the same registers: of the lanes' maxima of a chunk, the n-th
// largest is a lower bound of the row's n-th largest logit, so only what reaches it (seldom much more than n) goes into a list in the
// LDS, with its place; a member's rank is the number of members before it.
//
// Bound by memory and, about as much, by the exponentials: 1024 x 131072 bf16 with one alternative 55 us, 4.9 TB/s.  With 20 of them it takes
// 92, and 700 x 30000 35: the wavefronts learn their bounds each for itself.  Rows off 16-byte borders go an entry at a time: 1024 x 131071
// 132 us.  Few rows are bound by latency: 1 x 131072 with 20 alternatives 10.5 us and 5.2 for joining the splits.
// Entries that are infinite or the type's lowest value are known for masked ones and skipped; masks of other values (-1e9) tie like any logits,
// and a row that has hardly any others takes about twice as long (1024 x 131072 bf16 with 20 alternatives 209 us in place of 108).
#include "ops_internal.h"

namespace tst {
namespace {

struct LogArgs {
    const void *z;
    int64_t stride;
    const void *tokens;
    int token_bytes, C, top;
    float *of_token, *entropy;
    int32_t *top_ids;
    float *of_top;
    int V;
    bool wide;            // rows on 16-byte borders
    int splits, length;   // of a row, and logits of each
    float4 *states;       // [R][splits]: most, sum, weighted
    unsigned long long *keys;   // [R][splits][top], 0 behind the last
};

// What is sorted: the logit, then the lower token first.  0 is below every key.
__device__ __forceinline__ unsigned long long key_of(float v, int token) { return (unsigned long long)order_bits(v) << 32 | (unsigned)~token; }
__device__ __forceinline__ int token_of(unsigned long long key) { return (int)~(unsigned)key; }

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kVectors = 4, kFewVectors = 2;   // 16 bytes each, of a chunk for a lane: of whole rows, of splits
constexpr int kMaxTop = TST_LOGPROBS_MAX_TOP;
// A wavefront's list is kept under kShort.  Rising logits fill it with all that 64 lanes hold in one vector.
constexpr int kShort = 192, kRoom = kMaxTop + 64 * 8;
constexpr float kNan = __builtin_nanf("");
typedef unsigned long long Key;

// e^d below is 2^fl32(d log2 e), off by up to 2^-24 of d log2 e.  With the exponent's rounding put back by an fma the results' errors against 64 bits
// are the same (1024 x 131072 bf16: 5 to 8e-8, both ways) and the kernel takes 70 us in place of 60.
struct Shared {
    Key list[kWaves][kRoom], best[kWaves][kMaxTop], sorted[kMaxTop];
    float sums[3][kWaves], lost[kWaves];
    int counts[kWaves], flags[kWaves];
};

// The n largest of list[0 .. count), largest first, into sorted; 0 behind the last.  `threads` threads that have met, t of them this one.
__device__ __forceinline__ void rank_keys(const Key *list, int count, Key *sorted, int n, int t, int threads)
{
    for (int i = t; i < count; i += threads) {
        const Key mine = list[i];
        int rank = 0;
#pragma unroll 4
        for (int j = 0; j < count; ++j) rank += list[j] > mine;   // (keys differ: each holds its token)
        if (rank < n) sorted[rank] = mine;
    }
}

template <typename F> __device__ __forceinline__ float over_waves(float v, float *part, F f)
{
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) v = f(v, __shfl_xor(v, d));
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    v = part[0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) v = f(v, part[w]);
    return v;
}

// The n-th largest of the lanes' values (n <= 64).
__device__ __forceinline__ float nth_of_lanes(float mine, int n)
{
    unsigned left = order_bits(mine), least = 0;
    for (int j = 0; j < n; ++j) {
        least = wave_max(left);
        const unsigned long long have = __ballot(left == least);
        if ((int)(threadIdx.x & 63) == __builtin_ctzll(have)) left = 0;
    }
    return from_order_bits(least);
}

// Alternatives of a row (split) that has NaN, or whose lists did not have the room: n rounds over it.
template <int TYPE> __device__ void sort_slowly(const typename Entry<TYPE>::bits *z, int begin, int end, int n, Shared &s)
{
    typedef Entry<TYPE> E;
    Key last = 0;
    for (int j = 0; j < n; ++j) {
        Key mine = 0;
        for (int v = begin + threadIdx.x; v < end; v += kThreads) {
            const Key key = key_of(E::get(z[v]), v);
            if ((j == 0 || key < last) && key > mine) mine = key;   // (a NaN at token 0 has the largest key there is)
        }
        __syncthreads();
        s.list[0][threadIdx.x] = mine;
        __syncthreads();
        for (int half = kThreads / 2; half > 0; half /= 2) {
            if ((int)threadIdx.x < half && s.list[0][threadIdx.x + half] > s.list[0][threadIdx.x]) s.list[0][threadIdx.x] = s.list[0][threadIdx.x + half];
            __syncthreads();
        }
        last = s.list[0][0];
        if (threadIdx.x == 0) s.sorted[j] = last;
    }
    __syncthreads();
}

// The last step: results of a row from its state and its alternatives in sorted[].
template <int TYPE> __device__ void finish(const LogArgs &a, int64_t r, float most, float sum, float weighted, const Key *sorted)
{
    typedef Entry<TYPE> E;
    const typename E::bits *z = static_cast<const typename E::bits *>(a.z) + r * a.stride;
    // a sum of NaN: NaN or +infinity in the row; of 0: nothing but -infinity
    const float log_sum = sum > 0.f ? logf(sum) : kNan;
    if (threadIdx.x == 0 && a.entropy) a.entropy[r] = log_sum - weighted / sum;
    if ((int)threadIdx.x < a.C) {
        const int64_t i = r * a.C + threadIdx.x;
        const int64_t token = a.token_bytes == 8 ? static_cast<const int64_t *>(a.tokens)[i] : static_cast<const int32_t *>(a.tokens)[i];
        a.of_token[i] = token < 0 || token >= a.V ? kNan : E::get(z[token]) - most - log_sum;
    }
    if ((int)threadIdx.x < a.top) {
        const int token = token_of(sorted[threadIdx.x]);   // of the row, there being as many keys as alternatives (top <= V); -1 of no key
        a.top_ids[r * a.top + threadIdx.x] = token;
        a.of_top[r * a.top + threadIdx.x] = token < 0 ? kNan : E::get(z[token]) - most - log_sum;
    }
}

template <int TYPE, bool TOP, int VECTORS>
__global__ void __launch_bounds__(kThreads, 4)
k_logprobs(const LogArgs a)
{
    typedef Entry<TYPE> E;
    typedef typename E::bits bits;
    constexpr int V = 16 / sizeof(bits), kChunk = 64 * V * VECTORS;
    typedef bits piece __attribute__((ext_vector_type(V)));
    __shared__ Shared s;
    const int64_t r = blockIdx.x;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int split = blockIdx.y, begin = split * a.length, end = min(begin + a.length, a.V), n = min(a.top, end - begin);
    const bits *z = static_cast<const bits *>(a.z) + r * a.stride;
    const bits nothing = E::put(-INFINITY);
    const float lowest = TYPE == TST_F16 ? -65504.f : TYPE == TST_BF16 ? -0x1.fep127f : -0x1.fffffep127f;   // of the type

    float most = -INFINITY, sum = 0.f, weighted = 0.f;   // of the lane
    // Of the wavefront: n of its logits at least reach the bound (or all it has had); closed: the list has n that do.  What is larger
    // than `lost` and belongs to its n largest is in the list, what is equal to it may not be, if any is lost.
    float bound = -INFINITY, lost = -INFINITY;
    bool closed = false, any_lost = false, slow = false;
    int count = 0;   // of the list
    Key *const list = s.list[wave];

    auto load = [&](int v0, piece (&to)[VECTORS]) {
        if (a.wide && v0 + kChunk <= end) {
#pragma unroll
            for (int i = 0; i < VECTORS; ++i) to[i] = *reinterpret_cast<const piece *>(z + v0 + (i * 64 + lane) * V);
        } else {
#pragma unroll
            for (int i = 0; i < VECTORS; ++i)
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const int v = v0 + (i * 64 + lane) * V + j;
                    to[i][j] = v < end ? z[v] : nothing;
                }
        }
    };
    piece x[VECTORS], next[VECTORS];
    int v0 = begin + wave * kChunk;
    if (v0 < end) load(v0, x);
    for (; v0 < end; v0 += kWaves * kChunk) {
        if (v0 + kWaves * kChunk < end) load(v0 + kWaves * kChunk, next);
        __builtin_amdgcn_sched_barrier(0);   // or the compiler moves the loads behind the work that hides them
        float of_vector[VECTORS], here = -INFINITY;
#pragma unroll
        for (int i = 0; i < VECTORS; ++i) {
            of_vector[i] = E::get(x[i][0]);
#pragma unroll
            for (int j = 1; j < V; ++j) of_vector[i] = fmaxf(of_vector[i], E::get(x[i][j]));
            here = fmaxf(here, of_vector[i]);
        }
        if (here > most) {
            const float d = most - here;   // -infinity at first: nothing to move
            const float f = __builtin_amdgcn_exp2f(d * 1.44269504f);
            weighted = f > 0.f ? (weighted + d * sum) * f : 0.f;
            sum *= f;
            most = here;
        }
        const float from = most > -INFINITY ? most : 0.f;
#pragma unroll
        for (int i = 0; i < VECTORS; ++i)
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float d = E::get(x[i][j]) - from, f = __builtin_amdgcn_exp2f(d * 1.44269504f);   // NaN, +infinity: NaN
                sum += f;
                weighted = fmaf(f, fmaxf(d, -150.f), weighted);   // e^-150 is 0 here; -infinity would make 0 times it NaN
            }
        if constexpr (TOP) {
            auto collect = [&](bool strict) {
#pragma unroll
                for (int i = 0; i < VECTORS; ++i) {
                    if (__ballot(of_vector[i] >= bound) == 0) continue;
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        const float y = E::get(x[i][j]);
                        const int v = v0 + (i * 64 + lane) * V + j;
                        const bool take = (strict ? y > bound : y >= bound) && v < end;
                        const unsigned long long set = __ballot(take);
                        if (set == 0) continue;
                        const int at = count + __popcll(set & ((1ull << lane) - 1));
                        if (take && at < kRoom) list[at] = key_of(y, v);
                        count += __popcll(set);
                    }
                }
            };
            auto keep_largest = [&](int of) {   // of the list's first
                order_wave();
                rank_keys(list, of, s.best[wave], n, lane, 64);
                order_wave();
                count = min(of, n);
                if (lane < count) list[lane] = s.best[wave][lane];
            };
            // Few lanes reach what the list holds: that goes into it.  Else what n lanes of this chunk reach is a better bound.
            const int reach = closed ? __popcll(__ballot(here > bound)) : 64;
            if (reach > n) {
                const float better = nth_of_lanes(here, n);
                if (!closed || better > bound) {
                    bound = fmaxf(bound, better);
                    closed = false;
                }
            }
            if (reach > 0) {
                const bool masked = bound <= lowest && !closed;   // most of the chunk is: none of that goes into the list
                const int held = count;
                collect(closed || masked);
                if (masked) {
                    lost = bound;
                    any_lost = true;
                }
                if (count > kShort) {
                    // Too many: logits that tie at the bound, or rising ones.  Of this chunk the list takes what passes the n-th largest
                    // of the lanes' maxima; what is equal to it is lost for now.
                    keep_largest(held);
                    bound = fmaxf(bound, nth_of_lanes(here, n));
                    closed = false;
                    collect(true);
                    if (!any_lost || bound > lost) lost = bound;
                    any_lost = true;
                    if (count > kRoom) {
                        slow = true;
                        count = 0;
                    }
                }
                if (count > n + 16 || (count >= n && !closed)) {
                    keep_largest(count);
                    const float nth = from_order_bits((unsigned)(s.best[wave][n - 1] >> 32));
                    if (nth >= bound) {
                        bound = nth;
                        closed = true;   // what comes later in the row and is equal to it comes behind it
                    }
                }
            }
        }
#pragma unroll
        for (int i = 0; i < VECTORS; ++i) x[i] = next[i];
    }
    const float all = over_waves(most, s.sums[0], [](float x, float y) { return fmaxf(x, y); });
    const float d = most - all, f = most > -INFINITY ? __builtin_amdgcn_exp2f(d * 1.44269504f) : 0.f;
    const bool spoilt = sum != sum;
    weighted = f > 0.f ? (weighted + d * sum) * f : 0.f;
    sum = spoilt ? kNan : f > 0.f ? sum * f : 0.f;
    if constexpr (TOP) {
        order_wave();
        if (lane < n) s.best[wave][lane] = 0;
        order_wave();
        rank_keys(list, count, s.best[wave], n, lane, 64);
        if (lane == 0) {
            s.lost[wave] = lost;
            s.flags[wave] = (any_lost ? 1 : 0) | (slow ? 2 : 0);
        }
    }
    sum = over_waves(sum, s.sums[1], [](float x, float y) { return x + y; });
    weighted = over_waves(weighted, s.sums[2], [](float x, float y) { return x + y; });
    if constexpr (TOP) {
        int flags = 0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            flags |= s.flags[w];
            if (s.flags[w] & 1) lost = fmaxf(lost, s.lost[w]);
        }
        if (sum != sum || (flags & 2)) {
            sort_slowly<TYPE>(z, begin, end, n, s);
        } else {
            // the wavefronts' n largest behind one another
            __syncthreads();
            Key *const together = s.list[0];
            if ((int)threadIdx.x < n) s.sorted[threadIdx.x] = 0;
            if (lane < n) together[wave * n + lane] = s.best[wave][lane];
            __syncthreads();
            const Key mine = (int)threadIdx.x < kWaves * n ? together[threadIdx.x] : 0;
            if (mine) {
                int rank = 0;
#pragma unroll 4
                for (int j = 0; j < kWaves * n; ++j) rank += together[j] > mine;
                if (rank < n) s.sorted[rank] = mine;
            }
            __syncthreads();
            // What was lost counts if fewer than n lie above it: then the lowest tokens with that logit follow them.
            if (flags & 1) {
                const unsigned edge = order_bits(lost);
                int found = __syncthreads_count((int)threadIdx.x < n && (unsigned)(s.sorted[threadIdx.x] >> 32) > edge);
                for (int t0 = begin; t0 < end && found < n; t0 += kThreads) {
                    const int v = t0 + threadIdx.x;
                    const bool tie = v < end && E::get(z[v]) == lost;
                    const unsigned long long set = __ballot(tie);
                    __syncthreads();
                    if (lane == 0) s.counts[wave] = __popcll(set);
                    __syncthreads();
                    int before = found + __popcll(set & ((1ull << lane) - 1));
                    for (int w = 0; w < kWaves; ++w) {
                        if (w < wave) before += s.counts[w];
                        found += s.counts[w];
                    }
                    if (tie && before < n) s.sorted[before] = key_of(lost, v);
                }
                __syncthreads();
            }
        }
    }
    if (a.splits == 1) {
        finish<TYPE>(a, r, all, sum, weighted, s.sorted);
        return;
    }
    const int64_t part = r * a.splits + split;
    if (threadIdx.x == 0) a.states[part] = make_float4(all, sum, weighted, 0.f);
    if (TOP && (int)threadIdx.x < a.top) a.keys[part * a.top + threadIdx.x] = (int)threadIdx.x < n ? s.sorted[threadIdx.x] : 0;
}

// k_logprobs_join: a row from its splits.  Each brings its alternatives in order: of the first ceil(top / splits) of each, the top-th
// largest is a bound again, and only what reaches it is sorted.
constexpr int kMaxSplits = 32;

template <int TYPE>
__global__ void __launch_bounds__(kThreads)
k_logprobs_join(const LogArgs a)
{
    __shared__ Key list[kMaxSplits * kMaxTop], sorted[kMaxTop];
    __shared__ int count;
    const int64_t r = blockIdx.x;
    const int lane = threadIdx.x & 63;
    float most = -INFINITY, sum = 0.f, weighted = 0.f;
    if (lane < a.splits) {   // (every wavefront for itself)
        const float4 v = a.states[r * a.splits + lane];
        most = v.x;
        sum = v.y;
        weighted = v.z;
    }
    float all = most;
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) all = fmaxf(all, __shfl_xor(all, d));
    const float d = most - all, f = most > -INFINITY ? __builtin_amdgcn_exp2f(d * 1.44269504f) : 0.f;
    weighted = f > 0.f ? (weighted + d * sum) * f : 0.f;
    sum = sum != sum ? kNan : f > 0.f ? sum * f : 0.f;
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) {
        sum += __shfl_xor(sum, d);
        weighted += __shfl_xor(weighted, d);
    }
    if (a.top > 0) {
        const Key *keys = a.keys + r * a.splits * a.top;
        const int heads = blocks_of(a.top, a.splits), n = heads * a.splits;   // (below top + splits)
        if ((int)threadIdx.x < n) list[threadIdx.x] = keys[threadIdx.x / heads * a.top + threadIdx.x % heads];
        if ((int)threadIdx.x < a.top) sorted[threadIdx.x] = 0;
        if (threadIdx.x == 0) count = 0;
        __syncthreads();
        rank_keys(list, n, sorted, a.top, threadIdx.x, kThreads);
        __syncthreads();
        const Key bound = sorted[a.top - 1];   // 0: some splits hold fewer
        __syncthreads();
        for (int i = threadIdx.x; i < a.splits * a.top; i += kThreads) {
            const Key key = keys[i];
            if (key && key >= bound) list[atomicAdd(&count, 1)] = key;   // (in any order: they are sorted)
        }
        __syncthreads();
        rank_keys(list, count, sorted, a.top, threadIdx.x, kThreads);
        __syncthreads();
    }
    finish<TYPE>(a, r, all, sum, weighted, sorted);
}

// Splits of a row: while there are fewer than two workgroups for a compute unit, of a chunk for each wavefront at least.  us from Python in splits and
// as whole rows, bf16, with 1 and 20 alternatives: 1 x 131072 10.7 16.2 and 21 56, 128 x 131072 20.9 38.3 and 29.0 62.0, 256 x 131072 30.0 55.6 and
// 30.0 62.3, 400 x 131072 35.9 64.0 and 34.0 69.7; 64 x 32000 10.9 16.1 and 12.2 28.1, 256 x 32000 15.6 28.0 and 12.9 29.2, 400 x 32000 18.6 33.9
// and 15.2 31.8: where two splits are all, they pay for long rows and many alternatives alone.
int splits_of(int R, int V, int type)
{
    const int64_t least = (int64_t)kThreads * kFewVectors * (16 / type_bytes(type));
    const int64_t wanted = blocks_of(2 * compute_units(), R), useful = (V + least - 1) / least;
    const int64_t n = wanted < useful ? wanted : useful;
    return (int)(n < kMaxSplits ? n : kMaxSplits);
}

struct LogSpace {
    size_t keys, total;
};
LogSpace log_space(int R, int top)   // for the most splits there can be
{
    const size_t parts = (size_t)R * kMaxSplits < (size_t)4 * compute_units() ? (size_t)R * kMaxSplits : (size_t)4 * compute_units();
    const size_t keys = round256(parts * sizeof(float4));
    return LogSpace{keys, keys + round256(parts * top * sizeof(unsigned long long))};
}

}  // namespace
}  // namespace tst

extern "C" {

int tst_logprobs_workspace_bytes(int R, int V, int top, size_t *bytes)
{
    if (!bytes || R < 0 || V < 1 || V > 1 << 30 || top < 0 || top > V || top > TST_LOGPROBS_MAX_TOP) return TSTGEMM_EINVAL;
    *bytes = R > 0 && tst::splits_of(R, V, TST_F32) > 1 ? tst::log_space(R, top).total : 0;   // (fp32 rows are split first)
    return TSTGEMM_OK;
}

int tst_logprobs(const void *logits, int type, int64_t stride, const void *tokens, int token_bytes, int C, int top, float *of_token,
                 float *entropy, int32_t *top_ids, float *of_top, int R, int V, void *workspace, size_t workspace_bytes, void *stream)
{
    size_t need = 0;
    if (int rc = tst_logprobs_workspace_bytes(R, V, top, &need)) return rc;
    if (!tst::type_ok(type) || C < 0 || C > TST_LOGPROBS_MAX_TOKENS || (token_bytes != 4 && token_bytes != 8) || stride < V) return TSTGEMM_EINVAL;
    if (R == 0) return TSTGEMM_OK;
    const size_t entry = tst::type_bytes(type);
    if (!logits || !tst::aligned(logits, entry) || (C && (!tokens || !of_token)) || (top && (!top_ids || !of_top))) return TSTGEMM_EINVAL;
    if (need && (!workspace || workspace_bytes < need)) return TSTGEMM_EWORKSPACE;
    if (need && !tst::aligned(workspace, 256)) return TSTGEMM_EINVAL;
    const int per = (int)(16 / entry), splits = tst::splits_of(R, V, type);
    const int length = tst::blocks_of(tst::blocks_of(V, splits), per) * per;   // splits begin on borders of vectors
    tst::LogArgs a{logits, stride, tokens, token_bytes, C, top, of_token, entropy, top_ids, of_top, V,
                   tst::aligned(logits, 16) && stride % per == 0, tst::blocks_of(V, length), length, static_cast<float4 *>(workspace),
                   reinterpret_cast<unsigned long long *>(static_cast<char *>(workspace) + tst::log_space(R, top).keys)};
    return tst::status(tst::for_type(type, [&](auto t) {
        constexpr int T = decltype(t)::value;
        hipStream_t st = static_cast<hipStream_t>(stream);
        for (int64_t r = 0;;) {   // (rows of which there are many are not split)
            const int rows = (int)(R - r < tst::kLaunchRows ? R - r : tst::kLaunchRows);
            const dim3 grid(rows, a.splits);
            if (top > 0 && a.splits == 1) tst::k_logprobs<T, true, tst::kVectors><<<grid, tst::kThreads, 0, st>>>(a);
            else if (top > 0) tst::k_logprobs<T, true, tst::kFewVectors><<<grid, tst::kThreads, 0, st>>>(a);
            else if (a.splits == 1) tst::k_logprobs<T, false, tst::kVectors><<<grid, tst::kThreads, 0, st>>>(a);
            else tst::k_logprobs<T, false, tst::kFewVectors><<<grid, tst::kThreads, 0, st>>>(a);
            if (a.splits > 1) {
                if (hipError_t e = hipGetLastError()) return e;
                tst::k_logprobs_join<T><<<rows, tst::kThreads, 0, st>>>(a);
            }
            if (hipError_t e = hipGetLastError()) return e;
            r += rows;
            if (r == R) return hipSuccess;
            a.z = static_cast<const char *>(a.z) + rows * stride * (int64_t)entry;
            if (C) a.tokens = static_cast<const char *>(a.tokens) + (int64_t)rows * C * token_bytes;
            if (C) a.of_token += (int64_t)rows * C;
            if (a.entropy) a.entropy += rows;
            if (top) a.top_ids += (int64_t)rows * top;
            if (top) a.of_top += (int64_t)rows * top;
        }
    }));
}

}  // extern "C"
