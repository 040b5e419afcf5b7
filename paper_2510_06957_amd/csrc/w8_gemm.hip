// Layers in 8 bits: quantisation of tokens, the packed form of the weights, and the product
//   Y[m][n] = scale[m] w_scale[n] sum_k Q[m][k] W[k][n] + b[n].
#include "ops_internal.h"

namespace tst {
namespace {

// ------------------------------------------------------------------------------------------------------------------
// k_quantize: one workgroup per row; the row's largest magnitude, then its codes.  Magnitudes are compared as integers: of
// non-negative floats the bits order as the values do, with infinity and NaN above every number.
constexpr int kQuantThreads = 256;

__device__ __forceinline__ unsigned wave_max(unsigned v)
{
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) v = max(v, (unsigned)__shfl_xor((int)v, d));
    return v;
}

template <int TYPE>
__global__ void __launch_bounds__(kQuantThreads)
k_quantize(const typename Entry<TYPE>::bits *X, int64_t x_stride, int8_t *Q, int64_t q_stride, float *scale, int K)
{
    typedef Entry<TYPE> E;
    __shared__ unsigned most[kQuantThreads / 64];
    const int64_t m = blockIdx.x;
    const typename E::bits *x = X + m * x_stride;
    unsigned a = 0;
    for (int k = threadIdx.x; k < K; k += kQuantThreads) a = max(a, __float_as_uint(E::get(x[k])) & 0x7fffffffu);
    a = wave_max(a);
    if ((threadIdx.x & 63) == 0) most[threadIdx.x >> 6] = a;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kQuantThreads / 64; ++w) a = max(a, most[w]);
    const bool finite = a < 0x7f800000u;
    const float f = __uint_as_float(a);
    const float r = fminf(127.f / f, 3.402823466e38f);   // a = 0: 0 * FLT_MAX = 0
    if (threadIdx.x == 0) scale[m] = finite ? f / 127.f : __uint_as_float(0x7fc00000u);
    int8_t *q = Q + m * q_stride;
    for (int k = threadIdx.x; k < K; k += kQuantThreads) q[k] = finite ? (int8_t)(int)rintf(E::get(x[k]) * r) : (int8_t)0;
}

// ------------------------------------------------------------------------------------------------------------------
// k_w8_pack: one wavefront per piece; lane l holds column l % 16, rows 16 (l / 16) .. + 15 of it, in 16 bytes.
__global__ void __launch_bounds__(64)
k_w8_pack(const int8_t *W, char *packed, int K, int N, int k_blocks, int n_blocks)
{
    const int kb = blockIdx.x % k_blocks, nb = blockIdx.x / k_blocks;
    const int n = nb * kW8Cols + (threadIdx.x & 15), k0 = kb * kW8Rows + 16 * (threadIdx.x >> 4);
    const int8_t *w = W + (size_t)blockIdx.y * K * N;
    unsigned v[4] = {};
#pragma unroll
    for (int i = 0; i < 16; ++i)
        if (n < N && k0 + i < K) v[i / 4] |= (unsigned)(uint8_t)w[(size_t)(k0 + i) * N + n] << (8 * (i % 4));
    char *to = packed + (((size_t)blockIdx.y * n_blocks + nb) * k_blocks + kb) * kW8Piece;
    reinterpret_cast<u32x4 *>(to)[threadIdx.x] = u32x4{v[0], v[1], v[2], v[3]};
}

// ------------------------------------------------------------------------------------------------------------------
// k_w8_rows: 16 MT rows x 16 columns of Y for a workgroup; its wavefronts share K, block by block, and add their sums in the LDS.
// W is the first operand of the matrix instruction, so that a lane ends with four neighbouring columns of one row of Y.
struct GemmArgs {
    const int8_t *Q;
    int64_t q_stride;
    const float *scale;
    const char *packed;
    const float *w_scale, *b;
    void *Y;
    int M, K, N;
    bool wide;   // four neighbouring results can be stored at once
};

template <int TYPE>
__device__ __forceinline__ void store4(const GemmArgs &a, int m, int n, i32x4 sum)
{
    typedef Entry<TYPE> E;
    typedef typename E::bits bits;
    typedef bits bits4 __attribute__((ext_vector_type(4)));
    if (m >= a.M) return;
    const float s = a.scale[m];
    bits *y = static_cast<bits *>(a.Y) + (size_t)m * a.N + n;
    bits4 out;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int c = min(n + i, a.N - 1);
        float v = (float)sum[i] * s * a.w_scale[c];
        if (a.b) v += a.b[c];
        out[i] = E::put(v);
    }
    if (a.wide && n + 4 <= a.N) {
        *reinterpret_cast<bits4 *>(y) = out;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (n + i < a.N) y[i] = out[i];
    }
}

constexpr int kRowsWaves = 8;

template <int TYPE, int MT>
__global__ void __launch_bounds__(kRowsWaves * 64)
k_w8_rows(const GemmArgs a)
{
    __shared__ i32x4 part[kRowsWaves][MT][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int nb = blockIdx.x, m0 = blockIdx.y * 16 * MT;
    const int k_blocks = blocks_of(a.K, kW8Rows);
    const char *w = a.packed + (size_t)nb * k_blocks * kW8Piece + lane * 16;
    const int8_t *x[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) x[t] = a.Q + (int64_t)min(m0 + 16 * t + (lane & 15), a.M - 1) * a.q_stride;
    i32x4 acc[MT] = {};
    for (int kb = wave; kb < k_blocks; kb += kRowsWaves) {
        const i32x4 wf = *reinterpret_cast<const i32x4 *>(w + (size_t)kb * kW8Piece);
        const int k = kb * kW8Rows + 16 * (lane >> 4);
#pragma unroll
        for (int t = 0; t < MT; ++t) {
            i32x4 xf = {};
            if (k < a.K) xf = *reinterpret_cast<const i32x4 *>(x[t] + k);   // what lies behind K meets weights of 0
            acc[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wf, xf, acc[t], 0, 0, 0);
        }
    }
#pragma unroll
    for (int t = 0; t < MT; ++t) part[wave][t][lane] = acc[t];
    __syncthreads();
    for (int i = threadIdx.x; i < MT * 64; i += kRowsWaves * 64) {
        const int t = i >> 6, l = i & 63;
        i32x4 sum = part[0][t][l];
#pragma unroll
        for (int v = 1; v < kRowsWaves; ++v) sum += part[v][t][l];
        store4<TYPE>(a, m0 + 16 * t + (l & 15), nb * kW8Cols + 4 * (l >> 4), sum);
    }
}

hipError_t launch_gemm(const GemmArgs &a, int y_type, hipStream_t stream)
{
    return for_type(y_type, [&](auto type) {
        constexpr int T = decltype(type)::value;
        const unsigned cols = blocks_of(a.N, kW8Cols);
        if (a.M <= 16) k_w8_rows<T, 1><<<dim3(cols, 1), kRowsWaves * 64, 0, stream>>>(a);
        else k_w8_rows<T, 4><<<dim3(cols, blocks_of(a.M, 64)), kRowsWaves * 64, 0, stream>>>(a);
        return hipGetLastError();
    });
}

hipError_t launch_quantize(const void *X, int type, int64_t x_stride, int8_t *Q, int64_t q_stride, float *scale, int M, int K,
                           hipStream_t stream)
{
    return for_type(type, [&](auto t) {
        typedef typename Entry<decltype(t)::value>::bits bits;
        k_quantize<decltype(t)::value><<<M, kQuantThreads, 0, stream>>>(static_cast<const bits *>(X), x_stride, Q, q_stride, scale, K);
        return hipGetLastError();
    });
}

// the most rows of 64 that a grid's second dimension holds
constexpr int kMaxRows = 65535 * 64;

int check_gemm(const void *X, const void *packed, const float *w_scale, const void *Y, int type, int M, int K, int N)
{
    if (!type_ok(type) || M < 0 || M > kMaxRows || K < 1 || K > kW8MaxK || N < 1 || N > INT32_MAX - 64) return TSTGEMM_EINVAL;
    if (M > 0 && (!X || !packed || !w_scale || !Y || !aligned(packed, 16) || !aligned(Y, type_bytes(type)))) return TSTGEMM_EINVAL;
    return TSTGEMM_OK;
}

GemmArgs gemm_args(const int8_t *Q, int64_t q_stride, const float *scale, const void *packed, const float *w_scale, const float *b,
                   void *Y, int y_type, int M, int K, int N)
{
    return GemmArgs{Q, q_stride, scale, static_cast<const char *>(packed), w_scale, b, Y, M, K, N,
                    N % 4 == 0 && aligned(Y, 4 * type_bytes(y_type))};
}

}  // namespace
}  // namespace tst

extern "C" {

int tst_quantize(const void *X, int type, int64_t x_stride, int8_t *Q, int64_t q_stride, float *scale, int M, int K, void *stream)
{
    if (!tst::type_ok(type) || M < 0 || K < 1 || x_stride < K || q_stride < K) return TSTGEMM_EINVAL;
    if (M == 0) return TSTGEMM_OK;
    if (!X || !Q || !scale || !tst::aligned(X, tst::type_bytes(type)) || !tst::aligned(scale, 4)) return TSTGEMM_EINVAL;
    return tst::status(tst::launch_quantize(X, type, x_stride, Q, q_stride, scale, M, K, static_cast<hipStream_t>(stream)));
}

int tst_w8_bytes(int K, int N, size_t *bytes)
{
    if (!bytes || K < 1 || K > tst::kW8MaxK || N < 1) return TSTGEMM_EINVAL;
    *bytes = tst::w8_bytes(K, N);
    return TSTGEMM_OK;
}

int tst_w8_pack(const int8_t *W, int count, int K, int N, void *packed, void *stream)
{
    if (!W || !packed || count < 1 || count > 65535 || K < 1 || K > tst::kW8MaxK || N < 1 || !tst::aligned(packed, 16)) return TSTGEMM_EINVAL;
    const int k_blocks = tst::blocks_of(K, tst::kW8Rows), n_blocks = tst::blocks_of(N, tst::kW8Cols);
    if ((int64_t)k_blocks * n_blocks > INT32_MAX) return TSTGEMM_ETOOBIG;
    tst::k_w8_pack<<<dim3(k_blocks * n_blocks, count), 64, 0, static_cast<hipStream_t>(stream)>>>(W, static_cast<char *>(packed), K, N,
                                                                                                 k_blocks, n_blocks);
    return tst::status(hipGetLastError());
}

int tst_w8_gemm(const int8_t *Q, int64_t q_stride, const float *scale, const void *packed, const float *w_scale, const float *b,
                void *Y, int y_type, int M, int K, int N, void *stream)
{
    if (int rc = tst::check_gemm(Q, packed, w_scale, Y, y_type, M, K, N)) return rc;
    if (M == 0) return TSTGEMM_OK;
    if (!scale || !tst::aligned(Q, 16) || (M > 1 && (q_stride < K || q_stride % 16))) return TSTGEMM_EINVAL;
    return tst::status(tst::launch_gemm(tst::gemm_args(Q, q_stride, scale, packed, w_scale, b, Y, y_type, M, K, N), y_type,
                                        static_cast<hipStream_t>(stream)));
}

int tst_w8_linear_workspace_bytes(int M, int K, size_t *bytes)
{
    if (!bytes || M < 0 || K < 1 || K > tst::kW8MaxK) return TSTGEMM_EINVAL;
    *bytes = tst::round256((size_t)M * tst::blocks_of(K, 64) * 64) + tst::round256((size_t)M * sizeof(float));
    return TSTGEMM_OK;
}

int tst_w8_linear(const void *X, int type, int64_t x_stride, const void *packed, const float *w_scale, const float *b, void *Y,
                  int M, int K, int N, void *workspace, size_t workspace_bytes, void *stream)
{
    if (int rc = tst::check_gemm(X, packed, w_scale, Y, type, M, K, N)) return rc;
    if (M == 0) return TSTGEMM_OK;
    if (x_stride < K || !tst::aligned(X, tst::type_bytes(type))) return TSTGEMM_EINVAL;
    size_t need = 0;
    tst_w8_linear_workspace_bytes(M, K, &need);
    if (!workspace || workspace_bytes < need) return TSTGEMM_EWORKSPACE;
    if (!tst::aligned(workspace, 256)) return TSTGEMM_EINVAL;
    const int64_t q_stride = (int64_t)tst::blocks_of(K, 64) * 64;
    int8_t *Q = static_cast<int8_t *>(workspace);
    float *scale = reinterpret_cast<float *>(Q + tst::round256((size_t)M * q_stride));
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (hipError_t e = tst::launch_quantize(X, type, x_stride, Q, q_stride, scale, M, K, s)) return tst::status(e);
    return tst::status(tst::launch_gemm(tst::gemm_args(Q, q_stride, scale, packed, w_scale, b, Y, type, M, K, N), type, s));
}

}  // extern "C"
