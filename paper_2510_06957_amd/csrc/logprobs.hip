// Log probabilities of given tokens, entropy and the top alternatives of rows of logits (tst_logprobs).
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
};

// Bits that order as logits do: NaN above everything, -0 as +0.  0 is below every logit.
__device__ __forceinline__ unsigned order_key(float v)
{
    const unsigned u = __float_as_uint(v + 0.f);
    if ((u & 0x7fffffffu) > 0x7f800000u) return 0xffffffffu;
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// The running state of a softmax: most = max z, sum = sum e^(z - most), weighted = sum e^(z - most) (z - most).
struct Running {
    float most, sum, weighted;
};

// One state of two.  Moving a state from `from` to a larger `to` by d = from - to: sum e^d and (weighted + d sum) e^d.
__device__ __forceinline__ Running join(Running x, Running y)
{
    const float most = fmaxf(x.most, y.most);
    Running r{most, 0.f, 0.f};
    auto add = [&](const Running &s) {
        const float d = s.most - most, f = expf(d);
        if (!(f > 0.f) && d == d) return;   // nothing of it is left (also: an empty state against a real one)
        r.sum += s.sum * f;
        r.weighted += (s.weighted + (d == 0.f ? 0.f : d * s.sum)) * f;
    };
    if (x.sum != 0.f) add(x);
    if (y.sum != 0.f) add(y);
    return r;
}

constexpr int kLogThreads = 1024;

// k_logprobs: a workgroup per row.
template <int TYPE>
__global__ void __launch_bounds__(kLogThreads)
k_logprobs(const LogArgs a)
{
    typedef Entry<TYPE> E;
    __shared__ Running part[kLogThreads / 64];
    __shared__ unsigned long long best[kLogThreads / 64];
    const int64_t r = blockIdx.x;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const typename E::bits *z = static_cast<const typename E::bits *>(a.z) + r * a.stride;
    bool broken = false;   // NaN or +infinity
    float most = -INFINITY;
    for (int v = threadIdx.x; v < a.V; v += kLogThreads) {
        const float x = E::get(z[v]);
        broken |= !(x < INFINITY);
        most = fmaxf(most, x);
    }
    Running s{most, 0.f, 0.f};
    if (most > -INFINITY)
        for (int v = threadIdx.x; v < a.V; v += kLogThreads) {
            const float d = E::get(z[v]) - most, f = expf(d);
            s.sum += f;
            if (f > 0.f) s.weighted += f * d;
        }
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) s = join(s, Running{__shfl_xor(s.most, d), __shfl_xor(s.sum, d), __shfl_xor(s.weighted, d)});
    if (lane == 0) part[wave] = s;
    broken = __syncthreads_or(broken);
    s = part[0];
#pragma unroll
    for (int w = 1; w < kLogThreads / 64; ++w) s = join(s, part[w]);
    const bool none = broken || !(s.most > -INFINITY);
    const float nan = __uint_as_float(0x7fc00000u), log_sum = none ? nan : logf(s.sum);
    if (threadIdx.x == 0 && a.entropy) a.entropy[r] = none ? nan : log_sum - s.weighted / s.sum;
    if ((int)threadIdx.x < a.C) {
        const int64_t i = r * a.C + threadIdx.x;
        const int64_t token = a.token_bytes == 8 ? static_cast<const int64_t *>(a.tokens)[i] : static_cast<const int32_t *>(a.tokens)[i];
        a.of_token[i] = token < 0 || token >= a.V ? nan : E::get(z[token]) - s.most - log_sum;
    }
    unsigned long long last = ~0ull;   // of the alternatives found: logit, then the lower token first
    for (int j = 0; j < a.top; ++j) {
        unsigned long long mine = 0;
        for (int v = threadIdx.x; v < a.V; v += kLogThreads) {
            const unsigned long long key = ((unsigned long long)order_key(E::get(z[v])) << 32) | (unsigned)~v;
            if (key < last && key > mine) mine = key;
        }
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) {
            const unsigned long long o = ((unsigned long long)(unsigned)__shfl_xor((int)(mine >> 32), d) << 32) | (unsigned)__shfl_xor((int)mine, d);
            mine = mine > o ? mine : o;
        }
        __syncthreads();
        if (lane == 0) best[wave] = mine;
        __syncthreads();
        last = best[0];
#pragma unroll
        for (int w = 1; w < kLogThreads / 64; ++w) last = last > best[w] ? last : best[w];
        if (threadIdx.x == 0) {
            const int token = (int)~(unsigned)last;
            a.top_ids[r * a.top + j] = token;
            a.of_top[r * a.top + j] = E::get(z[token]) - s.most - log_sum;
        }
    }
}

}  // namespace
}  // namespace tst

extern "C" {

int tst_logprobs_workspace_bytes(int R, int V, int top, size_t *bytes)
{
    if (!bytes || R < 0 || V < 1 || top < 0 || top > V || top > TST_LOGPROBS_MAX_TOP) return TSTGEMM_EINVAL;
    *bytes = 0;
    return TSTGEMM_OK;
}

int tst_logprobs(const void *logits, int type, int64_t stride, const void *tokens, int token_bytes, int C, int top, float *of_token,
                 float *entropy, int32_t *top_ids, float *of_top, int R, int V, void *workspace, size_t workspace_bytes, void *stream)
{
    size_t need = 0;
    if (int rc = tst_logprobs_workspace_bytes(R, V, top, &need)) return rc;
    if (!tst::type_ok(type) || C < 0 || C > TST_LOGPROBS_MAX_TOKENS || (token_bytes != 4 && token_bytes != 8) || stride < V) return TSTGEMM_EINVAL;
    if (R == 0) return TSTGEMM_OK;
    if (!logits || !tst::aligned(logits, tst::type_bytes(type)) || (C && (!tokens || !of_token)) || (top && (!top_ids || !of_top)))
        return TSTGEMM_EINVAL;
    if (need && (!workspace || workspace_bytes < need)) return TSTGEMM_EWORKSPACE;
    if (need && !tst::aligned(workspace, 256)) return TSTGEMM_EINVAL;
    const tst::LogArgs a{logits, stride, tokens, token_bytes, C, top, of_token, entropy, top_ids, of_top, V};
    return tst::status(tst::for_type(type, [&](auto t) {
        tst::k_logprobs<decltype(t)::value><<<R, tst::kLogThreads, 0, static_cast<hipStream_t>(stream)>>>(a);
        return hipGetLastError();
    }));
}

}  // extern "C"
