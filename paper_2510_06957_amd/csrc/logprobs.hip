// Log probabilities of given tokens, entropy and the top alternatives of rows of logits (tst_logprobs).
//
// One pass over the logits.  A row, or a split of one where there are few rows, belongs to a workgroup, which takes it in chunks that its
// threads hold in registers; a thread keeps a running maximum m, sum e^(z - m) and sum e^(z - m) (z - m).  The alternatives
// come from the same registers: of the threads' maxima of a chunk, the n-th largest is a lower bound of the row's n-th largest
// logit, so only what reaches it (seldom much more than n) goes into a list in the LDS, with its place; a member's rank is the number
// of members before it.
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
constexpr int kVectors = 8, kFewVectors = 2;   // 16 bytes each, of a chunk for a thread: of whole rows, of splits
// The list.  It is kept short; it has room for what is left of earlier chunks (at most `top`) and all that `top` threads hold of one.
constexpr int kShort = 256, kList = TST_LOGPROBS_MAX_TOP + TST_LOGPROBS_MAX_TOP * kVectors * 8;
constexpr float kNan = __builtin_nanf("");

struct Shared {
    unsigned long long list[kList], sorted[TST_LOGPROBS_MAX_TOP];
    __align__(16) float most[kThreads];
    float sums[2][kWaves], bounds[kWaves];
    int count, counts[kWaves];
    float bound;
};

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

// The n largest keys of list[0 .. count), largest first, into sorted[]; 0 behind the last.  All threads; the list is as it was.
__device__ void sort_top(Shared &s, int count, int n)
{
    __syncthreads();
    if ((int)threadIdx.x < n) s.sorted[threadIdx.x] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < count; i += kThreads) {
        const unsigned long long mine = s.list[i];
        int rank = 0;
#pragma unroll 4
        for (int j = 0; j < count; ++j) rank += s.list[j] > mine;   // (keys differ: each holds its token)
        if (rank < n) s.sorted[rank] = mine;
    }
    __syncthreads();
}

// The n-th largest of the threads' values (n <= kThreads).
__device__ float nth_most(Shared &s, float mine, int n)
{
    __syncthreads();
    s.most[threadIdx.x] = mine;
    __syncthreads();
    int above = 0, same = 0;
#pragma unroll 4
    for (int j = 0; j < kThreads; j += 4) {
        const float4 v = *reinterpret_cast<const float4 *>(s.most + j);
        above += (v.x > mine) + (v.y > mine) + (v.z > mine) + (v.w > mine);
        same += (v.x == mine) + (v.y == mine) + (v.z == mine) + (v.w == mine);
    }
    if (above < n && n <= above + same) s.bound = mine;   // every thread that gets here has the same value
    __syncthreads();
    return s.bound;
}

// A value that n of the threads' values reach at least, and seldom many more: of the n / 4-th largest of each wavefront the least.
__device__ float reached_by(Shared &s, float mine, int n)
{
    unsigned left = order_bits(mine), least = 0;
    for (int j = 0; j < n; j += kWaves) {
        least = wave_max(left);
        const unsigned long long have = __ballot(left == least);
        if ((int)(threadIdx.x & 63) == __builtin_ctzll(have)) left = 0;
    }
    __syncthreads();
    if ((threadIdx.x & 63) == 0) s.bounds[threadIdx.x >> 6] = from_order_bits(least);
    __syncthreads();
    float v = s.bounds[0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) v = fminf(v, s.bounds[w]);
    return v;
}

// Alternatives of a row (split) that has NaN: n rounds over it.
template <int TYPE> __device__ void sort_slowly(const LogArgs &a, const typename Entry<TYPE>::bits *z, int begin, int end, int n, Shared &s)
{
    typedef Entry<TYPE> E;
    unsigned long long last = ~0ull;
    for (int j = 0; j < n; ++j) {
        unsigned long long mine = 0;
        for (int v = begin + threadIdx.x; v < end; v += kThreads) {
            const unsigned long long key = key_of(E::get(z[v]), v);
            if (key < last && key > mine) mine = key;
        }
        __syncthreads();
        s.list[threadIdx.x] = mine;
        __syncthreads();
        for (int half = kThreads / 2; half > 0; half /= 2) {
            if ((int)threadIdx.x < half && s.list[threadIdx.x + half] > s.list[threadIdx.x]) s.list[threadIdx.x] = s.list[threadIdx.x + half];
            __syncthreads();
        }
        last = s.list[0];
        if (threadIdx.x == 0) s.sorted[j] = last;
    }
    __syncthreads();
}

// The last step: results of a row from its state and its alternatives in sorted[].
template <int TYPE> __device__ void finish(const LogArgs &a, int64_t r, float most, float sum, float weighted, const Shared &s)
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
        const int token = token_of(s.sorted[threadIdx.x]);
        a.top_ids[r * a.top + threadIdx.x] = token;
        a.of_top[r * a.top + threadIdx.x] = E::get(z[token]) - most - log_sum;
    }
}

template <int TYPE, bool TOP, int VECTORS>
__global__ void __launch_bounds__(kThreads, 4)
k_logprobs(const LogArgs a)
{
    typedef Entry<TYPE> E;
    typedef typename E::bits bits;
    constexpr int V = 16 / sizeof(bits);
    typedef bits piece __attribute__((ext_vector_type(V)));
    __shared__ Shared s;
    const int64_t r = blockIdx.x;
    const int split = blockIdx.y, begin = split * a.length, end = min(begin + a.length, a.V), n = min(a.top, end - begin);
    const bits *z = static_cast<const bits *>(a.z) + r * a.stride;
    const bits nothing = E::put(-INFINITY);
    if (TOP && threadIdx.x == 0) s.count = 0;

    float most = -INFINITY, sum = 0.f, weighted = 0.f;   // of the thread
    float bound = -INFINITY;                             // n logits at least reach it (or all there were)
    float lost = -INFINITY;                              // some that are equal to this are not in the list ...
    bool any_lost = false;                               // ... if this is set
    bool first = true;
    for (int v0 = begin; v0 < end; v0 += kThreads * V * VECTORS) {
        piece x[VECTORS];
        auto place = [&](int i) { return v0 + (i * kThreads + (int)threadIdx.x) * V; };
#pragma unroll
        for (int i = 0; i < VECTORS; ++i) {
            const int v = place(i);
            if (a.wide && v + V <= end) {
                x[i] = *reinterpret_cast<const piece *>(z + v);
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j) x[i][j] = v + j < end ? z[v + j] : nothing;
            }
        }
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
            // Few threads reach the bound of earlier chunks: what they have goes into the list.  Else a bound of this one's.
            if (first || __syncthreads_count(here >= bound) > n) bound = fmaxf(bound, reached_by(s, here, n));
            first = false;
            // Few vectors reach the bound; they are read again, from the L2, rather than looked for in the registers.
            auto collect = [&](bool strict) {
                if (here < bound) return;
#pragma unroll
                for (int i = 0; i < VECTORS; ++i)
                    if (of_vector[i] >= bound)
                        for (int j = 0, v = place(i); j < V && v < end; ++j, ++v) {
                            const float y = E::get(z[v]);
                            if (strict ? y > bound : y >= bound) {
                                const int at = atomicAdd(&s.count, 1);
                                if (at < kList) s.list[at] = key_of(y, v);
                            }
                        }
            };
            const int held = s.count;
            __syncthreads();
            collect(false);
            __syncthreads();
            if (s.count > kShort) {
                // Too many: logits that tie at the bound (masked ones above all), a bound too low, or much from earlier chunks.  The list
                // keeps its `n` largest, and of this chunk all that pass the n-th largest of the threads' maxima; fewer than n threads
                // have any.  What is equal to it is lost for now.
                sort_top(s, held, n);
                if ((int)threadIdx.x < n) s.list[threadIdx.x] = s.sorted[threadIdx.x];
                if (threadIdx.x == 0) s.count = min(held, n);
                bound = fmaxf(bound, nth_most(s, here, n));   // (meets)
                collect(true);
                __syncthreads();
                if (!any_lost || bound > lost) lost = bound;
                any_lost = true;
            }
        }
    }
    const float all = over_waves(most, s.sums[0], [](float x, float y) { return fmaxf(x, y); });
    const float d = most - all, f = most > -INFINITY ? __builtin_amdgcn_exp2f(d * 1.44269504f) : 0.f;
    const bool spoilt = sum != sum;
    weighted = f > 0.f ? (weighted + d * sum) * f : 0.f;
    sum = spoilt ? kNan : f > 0.f ? sum * f : 0.f;
    __syncthreads();
    sum = over_waves(sum, s.sums[0], [](float x, float y) { return x + y; });
    weighted = over_waves(weighted, s.sums[1], [](float x, float y) { return x + y; });
    if constexpr (TOP) {
        if (sum != sum) {
            sort_slowly<TYPE>(a, z, begin, end, n, s);
        } else {
            sort_top(s, s.count, n);
            // What was lost counts if fewer than n lie above it: then the lowest tokens with that logit follow them.
            if (any_lost) {
                const unsigned edge = order_bits(lost);
                int found = __syncthreads_count((int)threadIdx.x < n && (unsigned)(s.sorted[threadIdx.x] >> 32) > edge);
                for (int v0 = begin; v0 < end && found < n; v0 += kThreads) {
                    const int v = v0 + threadIdx.x;
                    const bool tie = v < end && E::get(z[v]) == lost;
                    const unsigned long long set = __ballot(tie);
                    __syncthreads();
                    if ((threadIdx.x & 63) == 0) s.counts[threadIdx.x >> 6] = __popcll(set);
                    __syncthreads();
                    int before = found + __popcll(set & ((1ull << (threadIdx.x & 63)) - 1));
                    for (int w = 0; w < kWaves; ++w) {
                        if (w < (int)(threadIdx.x >> 6)) before += s.counts[w];
                        found += s.counts[w];
                    }
                    if (tie && before < n) s.sorted[before] = key_of(lost, v);
                }
                __syncthreads();
            }
        }
    }
    if (a.splits == 1) {
        finish<TYPE>(a, r, all, sum, weighted, s);
        return;
    }
    const int64_t part = r * a.splits + split;
    if (threadIdx.x == 0) a.states[part] = make_float4(all, sum, weighted, 0.f);
    if (TOP && (int)threadIdx.x < a.top) a.keys[part * a.top + threadIdx.x] = (int)threadIdx.x < n ? s.sorted[threadIdx.x] : 0;
}

// k_logprobs_join: a row from its splits.  Each brings its alternatives in order: of the first ceil(top / splits) of each, the top-th
// largest is a bound again, and only what reaches it is sorted.
template <int TYPE>
__global__ void __launch_bounds__(kThreads)
k_logprobs_join(const LogArgs a)
{
    __shared__ Shared s;
    const int64_t r = blockIdx.x;
    const int lane = threadIdx.x & 63;
    float most = -INFINITY, sum = 0.f, weighted = 0.f;
    if (lane < a.splits) {   // (every wavefront for itself; at most 32 splits)
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
        const unsigned long long *keys = a.keys + r * a.splits * a.top;
        const int heads = blocks_of(a.top, a.splits), n = heads * a.splits;   // (below top + splits)
        if ((int)threadIdx.x < n) s.list[threadIdx.x] = keys[threadIdx.x / heads * a.top + threadIdx.x % heads];
        sort_top(s, n, a.top);
        const unsigned long long bound = s.sorted[a.top - 1];   // 0: some splits hold fewer
        if (threadIdx.x == 0) s.count = 0;
        __syncthreads();
        for (int i = threadIdx.x; i < a.splits * a.top; i += kThreads) {
            const unsigned long long key = keys[i];
            if (key && key >= bound) s.list[atomicAdd(&s.count, 1)] = key;
        }
        __syncthreads();
        sort_top(s, s.count, a.top);
    }
    finish<TYPE>(a, r, all, sum, weighted, s);
}

// Splits of a row: while there are fewer than two workgroups for a compute unit, of a chunk at least.
constexpr int kMaxSplits = 32;
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
    if (!bytes || R < 0 || V < 1 || top < 0 || top > V || top > TST_LOGPROBS_MAX_TOP) return TSTGEMM_EINVAL;
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
    const tst::LogArgs a{logits, stride, tokens, token_bytes, C, top, of_token, entropy, top_ids, of_top, V,
                         tst::aligned(logits, 16) && stride % per == 0, tst::blocks_of(V, length), length, static_cast<float4 *>(workspace),
                         reinterpret_cast<unsigned long long *>(static_cast<char *>(workspace) + tst::log_space(R, top).keys)};
    return tst::status(tst::for_type(type, [&](auto t) {
        constexpr int T = decltype(t)::value;
        hipStream_t st = static_cast<hipStream_t>(stream);
        const dim3 grid(R, a.splits);
        if (top > 0 && a.splits == 1) tst::k_logprobs<T, true, tst::kVectors><<<grid, tst::kThreads, 0, st>>>(a);
        else if (top > 0) tst::k_logprobs<T, true, tst::kFewVectors><<<grid, tst::kThreads, 0, st>>>(a);
        else if (a.splits == 1) tst::k_logprobs<T, false, tst::kVectors><<<grid, tst::kThreads, 0, st>>>(a);
        else tst::k_logprobs<T, false, tst::kFewVectors><<<grid, tst::kThreads, 0, st>>>(a);
        if (a.splits > 1) {
            if (hipError_t e = hipGetLastError()) return e;
            tst::k_logprobs_join<T><<<R, tst::kThreads, 0, st>>>(a);
        }
        return hipGetLastError();
    }));
}

}  // extern "C"
