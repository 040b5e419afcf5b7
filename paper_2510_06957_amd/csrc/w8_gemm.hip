// Layers in 8 bits: quantisation of tokens, the packed form of the weights, and the product
//   Y[m][n] = scale[m] w_scale[n] sum_k Q[m][k] W[k][n] + b[n].
#include "ops_internal.h"
#include "w8_choice.h"

namespace tst {
namespace {

// ------------------------------------------------------------------------------------------------------------------
// k_quantize: one workgroup per row; the row's largest magnitude, then its codes.  Magnitudes are compared as integers: of
// non-negative floats the bits order as the values do, with infinity and NaN above every number.  2048 x 4096 bf16 7.0 us, 3.6 TB/s read and
// written where a large copy reaches 5.2: a workgroup has two loads a thread on the way, a meeting behind them, then the stores, and is done.
// Few rows are bound by latency (37 x 2053 fp16 4.7 us).
// The row stays in the registers on the way if it fits (64 bytes for a thread), else it is read twice.
constexpr int kQuantBytes = 64;

// What a row's codes are made with, from the bits of its largest magnitude.
struct Scaling {
    bool finite;
    float factor, scale;
    __device__ explicit Scaling(unsigned most)
    {
        finite = most < 0x7f800000u;
        const float a = __uint_as_float(most);
        factor = fminf(127.f / a, 3.402823466e38f);   // a = 0: 0 * FLT_MAX = 0
        scale = finite ? a / 127.f : __uint_as_float(0x7fc00000u);
    }
    __device__ __forceinline__ unsigned code(float x) const { return finite ? (unsigned)(int)rintf(x * factor) & 0xffu : 0u; }
};

// WIDE: rows of X on 16-byte borders, rows of Q on borders of a piece's codes, K a multiple of a piece; else an entry at a time.
template <int TYPE, bool WIDE, int THREADS>
__global__ void __launch_bounds__(THREADS)
k_quantize(const typename Entry<TYPE>::bits *X, int64_t x_stride, int8_t *Q, int64_t q_stride, float *scale, int K)
{
    typedef Entry<TYPE> E;
    typedef typename E::bits bits;
    constexpr int V = WIDE ? 16 / sizeof(bits) : 1, kPieces = kQuantBytes / sizeof(bits) / V;
    typedef bits piece __attribute__((ext_vector_type(V)));
    __shared__ unsigned most[THREADS / 64];
    const int64_t m = blockIdx.x;
    const bits *x = X + m * x_stride;
    int8_t *q = Q + m * q_stride;
    piece v[kPieces];
    auto load = [&](int k0) {
#pragma unroll
        for (int p = 0; p < kPieces; ++p) {
            const int k = k0 + (p * THREADS + threadIdx.x) * V;
            v[p] = piece{};
            if (k < K) v[p] = *reinterpret_cast<const piece *>(x + k);
        }
    };
    constexpr int kRound = kPieces * THREADS * V;
    unsigned a = 0;
    for (int k0 = 0; k0 < K; k0 += kRound) {
        load(k0);
#pragma unroll
        for (int p = 0; p < kPieces; ++p)
#pragma unroll
            for (int i = 0; i < V; ++i) a = max(a, __float_as_uint(E::get(v[p][i])) & 0x7fffffffu);
    }
    a = wave_max(a);
    if ((threadIdx.x & 63) == 0) most[threadIdx.x >> 6] = a;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) a = max(a, most[w]);
    const Scaling by(a);
    if (threadIdx.x == 0) scale[m] = by.scale;
    for (int k0 = 0; k0 < K; k0 += kRound) {
        if (K > kRound) load(k0);
#pragma unroll
        for (int p = 0; p < kPieces; ++p) {
            const int k = k0 + (p * THREADS + threadIdx.x) * V;
            if (k >= K) continue;
            if constexpr (V == 1) {
                q[k] = (int8_t)by.code(E::get(v[p][0]));
            } else {
                unsigned out[V / 4] = {};
#pragma unroll
                for (int i = 0; i < V; ++i) out[i / 4] |= by.code(E::get(v[p][i])) << (8 * (i % 4));
                if constexpr (V == 8) *reinterpret_cast<u32x2 *>(q + k) = u32x2{out[0], out[1]};
                else *reinterpret_cast<unsigned *>(q + k) = out[0];
            }
        }
    }
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

// Four neighbouring results of row m from column n on.
template <int TYPE>
__device__ __forceinline__ void store4(const GemmArgs &a, int m, int n, i32x4 sum, float s, const float (&t)[4], const float (&b)[4])
{
    typedef Entry<TYPE> E;
    typedef typename E::bits bits;
    typedef bits bits4 __attribute__((ext_vector_type(4)));
    bits *y = static_cast<bits *>(a.Y) + (size_t)m * a.N + n;
    bits4 out;
#pragma unroll
    for (int r = 0; r < 4; ++r) out[r] = E::put((float)sum[r] * s * t[r] + b[r]);
    if (a.wide) {   // N is a multiple of 4: all four or none
        if (n < a.N) *reinterpret_cast<bits4 *>(y) = out;
    } else {
#pragma unroll
        for (int r = 0; r < 4; ++r)
            if (n + r < a.N) y[r] = out[r];
    }
}

constexpr int kBufferFlags = 0x00027000;       // untyped, out of bounds by the byte
constexpr unsigned kOutside = 0x80000000u;     // of every buffer, also with the lane offsets that are added to it

// bytes from `at` on, both the same for all lanes (kept in scalar registers)
__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer(const void *at, unsigned bytes)
{
    const uint64_t p = reinterpret_cast<uint64_t>(at);
    const uint64_t uniform = (uint64_t)(unsigned)__builtin_amdgcn_readfirstlane((int)(p >> 32)) << 32 | (unsigned)__builtin_amdgcn_readfirstlane((int)p);
    return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void *>(uniform), 0, __builtin_amdgcn_readfirstlane((int)bytes), kBufferFlags);
}

// 16 bytes; 0 where lane_offset lies outside the buffer (`offset`, the same for all lanes, never leads there)
__device__ __forceinline__ i32x4 load16(__amdgpu_buffer_rsrc_t from, unsigned lane_offset, unsigned offset)
{
    return __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(from, lane_offset, offset, 0));
}

// 16 MT rows x 16 NT columns of Y for a workgroup; its wavefronts share K, 128 at a time, and add their sums in the LDS at the end.
// W comes from memory straight into the registers (a piece of the packed form is an operand of the matrix instruction).  X goes through a
// part of the LDS that belongs to the wavefront: an operand wants row l % 16 in lane l, and loads whose neighbouring lanes lie in different
// rows take the address unit a cycle for each lane (64 x 16384 x 4096: 35 us in place of 18), so 8 lanes load 128 bytes of a row together.
// Chunk c of 8 of a row stands in slot (row % 16) ^ c, which makes both the writes (8 chunks of a row together) and the reads (16 rows
// of a chunk together) free of bank conflicts.  64 x 16384 x 4096 16.4 us (67 MB of weights at 4.1 TB/s), 256 x 4096 x 4096 11.6.
constexpr int kRowsWaves = 8, kRowsThreads = kRowsWaves * 64;

template <int TYPE, int MT, int NT>
__global__ void __launch_bounds__(kRowsThreads, 2)
k_w8_rows(const GemmArgs a)
{
    constexpr int kPieces = 2 * MT;   // 16-byte pieces of X for a lane and step
    constexpr int kStage = 16 * MT * 8, kPart = MT * NT * 64;   // 16 bytes each, for a wavefront
    __shared__ i32x4 lds[kRowsWaves * (kStage > kPart ? kStage : kPart)];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int nb0 = blockIdx.x * NT, m0 = blockIdx.y * 16 * MT;
    const int k_blocks = blocks_of(a.K, kW8Rows), steps = (k_blocks + 1) / 2, n_blocks = blocks_of(a.N, kW8Cols);
    const unsigned column = k_blocks * kW8Piece, q_stride = (unsigned)a.q_stride;
    const auto w = buffer(a.packed + (size_t)nb0 * column, min(NT, n_blocks - nb0) * column);
    const auto x = buffer(a.Q + m0 * a.q_stride, (min(16 * MT, a.M - m0) - 1) * q_stride + ((a.K + 15) & ~15));
    const int c = lane & 7, r0 = lane >> 3;   // a lane's pieces: chunk c of rows r0, r0 + 8, ...
    i32x4 *const stage = lds + wave * kStage;
    i32x4 acc[MT][NT] = {}, xr[kPieces], wr[2][NT], wn[2][NT];
    auto load_x = [&](int step) {
        const unsigned k = step * kStepK + c * 16, at = k < (unsigned)a.K ? r0 * q_stride + k : kOutside;
#pragma unroll
        for (int p = 0; p < kPieces; ++p) xr[p] = load16(x, at + p * 8 * q_stride, 0);
    };
    auto load_w = [&](int step, i32x4 (&to)[2][NT]) {
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int j = 0; j < NT; ++j) to[s][j] = load16(w, min(2 * step + s, k_blocks - 1) * kW8Piece + j * column + lane * 16, 0);
    };
    auto store_x = [&]() {
#pragma unroll
        for (int p = 0; p < kPieces; ++p) {
            const int row = p * 8 + r0;
            stage[((row >> 4) * 8 + c) * 16 + ((row & 15) ^ c)] = xr[p];
        }
    };
    load_x(wave);
    load_w(wave, wr);
    for (int step = wave; step < steps; step += kRowsWaves) {
        store_x();
        order_wave();
        load_x(step + kRowsWaves);   // behind the last step: X reads as 0
        load_w(step + kRowsWaves, wn);
        __builtin_amdgcn_sched_barrier(0);   // or the compiler moves the loads to where they are used
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int t = 0; t < MT; ++t) {
                const int chunk = 4 * s + (lane >> 4);
                const i32x4 xf = stage[(t * 8 + chunk) * 16 + ((lane & 15) ^ chunk)];
#pragma unroll
                for (int j = 0; j < NT; ++j) acc[t][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wr[s][j], xf, acc[t][j], 0, 0, 0);
            }
        order_wave();
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int j = 0; j < NT; ++j) wr[s][j] = wn[s][j];
    }
    __syncthreads();
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int j = 0; j < NT; ++j) lds[(wave * MT * NT + t * NT + j) * 64 + lane] = acc[t][j];
    __syncthreads();
    for (int i = threadIdx.x; i < MT * NT * 64; i += kRowsThreads) {
        const int l = i & 63, t = (i >> 6) / NT, j = (i >> 6) % NT;
        i32x4 sum = lds[i];
#pragma unroll
        for (int v = 1; v < kRowsWaves; ++v) sum += lds[v * kPart + i];
        const int m = m0 + 16 * t + (l & 15), n = (nb0 + j) * kW8Cols + 4 * (l >> 4);
        float ws[4], b[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            ws[r] = a.w_scale[min(n + r, a.N - 1)];
            b[r] = a.b ? a.b[min(n + r, a.N - 1)] : 0.f;
        }
        if (m < a.M) store4<TYPE>(a, m, n, sum, a.scale[m], ws, b);
    }
}

// ------------------------------------------------------------------------------------------------------------------
// k_w8_few: tst_w8_linear() for a token or a few in one launch: every workgroup quantises them by itself, while its first weights are on
// their way, keeps the codes in the LDS, and goes on as k_w8_rows with one row tile and one column tile.  Bound by the weights: 1 x 4096 x
// 11008 7.6 us on the GPU, 5.9 TB/s (two column tiles 8.8).  us from Python, and of the two launches of other calls, bf16, 1 to 4 rows:
// 4096 x 11008 8.8 9.8 11.3 12.6 and 12.5 12.7 12.4 12.7, 4096 x 4096 5.3 6.3 5.8 7.7 and 9.4 9.6 9.3 9.4, 1024 x 4096 5.3 and 9.7 each,
// 8192 x 4096 8.2 9.7 and 10.4 10.5, 16384 x 4096 13.7 and 14.6: what a further row costs is what every workgroup quantises again, and
// with kFewCodes codes in all it comes to the launch that it saves.
constexpr int kFewRows = 4, kFewCodes = 16384;   // rows, and rows x (K padded to kStepK), at most

template <int TYPE>
__global__ void __launch_bounds__(kRowsThreads, 4)
k_w8_few(const GemmArgs a, const typename Entry<TYPE>::bits *X, int64_t x_stride, bool wide)
{
    typedef Entry<TYPE> E;
    typedef typename E::bits bits;
    constexpr int V = 16 / sizeof(bits);
    typedef bits piece __attribute__((ext_vector_type(V)));
    __shared__ i32x4 codes[kFewCodes / 16];
    __shared__ i32x4 part[kRowsWaves * 64];
    __shared__ unsigned most[kFewRows][kRowsWaves];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), nb = blockIdx.x;
    const int k_blocks = blocks_of(a.K, kW8Rows), steps = (k_blocks + 1) / 2, row_codes = steps * kStepK;
    const unsigned column = k_blocks * kW8Piece;
    const auto w = buffer(a.packed + (size_t)nb * column, column);
    i32x4 acc = {}, w0[2], w1[2];
    auto load_w = [&](int step, i32x4 (&to)[2]) {
#pragma unroll
        for (int s = 0; s < 2; ++s) to[s] = load16(w, min(2 * step + s, k_blocks - 1) * kW8Piece + lane * 16, 0);
    };
    load_w(wave, w0);
    load_w(wave + kRowsWaves, w1);

    for (int m = 0; m < a.M; ++m) {
        const bits *x = X + m * x_stride;
        unsigned v = 0;
        if (wide) {
            for (int k = threadIdx.x * V; k < a.K; k += kRowsThreads * V) {   // K is a multiple of V
                const piece p = *reinterpret_cast<const piece *>(x + k);
#pragma unroll
                for (int i = 0; i < V; ++i) v = max(v, __float_as_uint(E::get(p[i])) & 0x7fffffffu);
            }
        } else {
#pragma unroll 4
            for (int k = threadIdx.x; k < a.K; k += kRowsThreads) v = max(v, __float_as_uint(E::get(x[k])) & 0x7fffffffu);
        }
        v = wave_max(v);
        if (lane == 0) most[m][wave] = v;
    }
    __syncthreads();
    auto scaling = [&](int m) {
        unsigned v = most[m][0];
#pragma unroll
        for (int i = 1; i < kRowsWaves; ++i) v = max(v, most[m][i]);
        return Scaling(v);
    };
    char *const bytes = reinterpret_cast<char *>(codes);
    for (int m = 0; m < a.M; ++m) {   // from the L2; 0 behind K
        const bits *x = X + m * x_stride;
        const Scaling by = scaling(m);
        if (wide) {
            for (int k = threadIdx.x * V; k < row_codes; k += kRowsThreads * V) {
                unsigned out[V / 4] = {};
                if (k < a.K) {
                    const piece p = *reinterpret_cast<const piece *>(x + k);
#pragma unroll
                    for (int i = 0; i < V; ++i) out[i / 4] |= by.code(E::get(p[i])) << (8 * (i % 4));
                }
#pragma unroll
                for (int i = 0; i < V / 4; ++i) reinterpret_cast<unsigned *>(bytes + m * row_codes + k)[i] = out[i];
            }
        } else {
#pragma unroll 4
            for (int k = threadIdx.x; k < row_codes; k += kRowsThreads) bytes[m * row_codes + k] = k < a.K ? (char)by.code(E::get(x[k])) : 0;
        }
    }
    __syncthreads();
    const char *const mine = bytes + min(lane & 15, a.M - 1) * row_codes + 16 * (lane >> 4);   // columns of rows that are not there are not used
    auto multiply = [&](int step, const i32x4 (&ws)[2]) {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const i32x4 xf = *reinterpret_cast<const i32x4 *>(mine + step * kStepK + 64 * s);
            acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(ws[s], xf, acc, 0, 0, 0);
        }
    };
    for (int step = wave; step < steps;) {
        multiply(step, w0);
        load_w(step + 2 * kRowsWaves, w0);
        step += kRowsWaves;
        if (step >= steps) break;
        multiply(step, w1);
        load_w(step + 2 * kRowsWaves, w1);
        step += kRowsWaves;
    }
    part[wave * 64 + lane] = acc;
    __syncthreads();
    const int i = threadIdx.x, m = i & 15, n = nb * kW8Cols + 4 * (i >> 4);
    if (i < 64 && m < a.M) {
        i32x4 sum = part[i];
#pragma unroll
        for (int v = 1; v < kRowsWaves; ++v) sum += part[v * 64 + i];
        float ws[4], b[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            ws[r] = a.w_scale[min(n + r, a.N - 1)];
            b[r] = a.b ? a.b[min(n + r, a.N - 1)] : 0.f;
        }
        store4<TYPE>(a, m, n, sum, scaling(m).scale, ws, b);
    }
}

// ------------------------------------------------------------------------------------------------------------------
// k_w8_tiles: 256 columns x 16 MF rows of Y for a workgroup of four wavefronts, 64 columns x all its rows each.  What a wavefront
// takes of W nobody else in the workgroup needs, so it goes from memory straight into the registers (a piece of the packed form is an
// operand of the matrix instruction); X goes through the LDS, 128 of K at a time in two buffers, in slots as in k_w8_rows.  Bound by its
// loads: 48 KiB a step for 256 x 128 results.  4096 x 8192 x 8192 217 us, 2.53 POP/s (a library's product of this size 236;
// instructions of 32 x 32 x 32 9 % slower; a tile of 256 x 256 does not fit the registers of four wavefronts), 2048 x 4096 x 4096 38 us.
constexpr int kTileThreads = 256, kTileCols = 256;

template <int TYPE, int MF>
__global__ void __launch_bounds__(kTileThreads, 2)
k_w8_tiles(const GemmArgs a, int m_tiles, int n_tiles)
{
    constexpr int kRows = 16 * MF, kPieces = MF / 2;   // 16-byte pieces of X for a thread and step
    __shared__ i32x4 xs[2][kRows * 8];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // tiles that follow one another share rows or columns and run on one XCD (workgroups go to the eight XCDs in turn)
    const int total = m_tiles * n_tiles, per = total / 8, id = blockIdx.x;
    const int tile = id < per * 8 ? (id % 8) * per + id / 8 : id;
    constexpr int kGroup = 32 / MF;   // row tiles that go through the columns together: 512 rows
    const int group = tile / (kGroup * n_tiles), rest = tile % (kGroup * n_tiles);
    const int height = min(kGroup, m_tiles - group * kGroup);
    const int m0 = __builtin_amdgcn_readfirstlane((group * kGroup + rest % height) * kRows);
    const int nb0 = __builtin_amdgcn_readfirstlane(rest / height * (kTileCols / 16) + wave * 4);

    // Rows behind M, and chunks of X behind K, read as 0 by the hardware's bounds; what of W has no counterpart there does not matter, and
    // is read from the last block or column that there is.
    const int k_blocks = blocks_of(a.K, kW8Rows), n_blocks = blocks_of(a.N, kW8Cols), steps = (k_blocks + 1) / 2;
    const unsigned column = k_blocks * kW8Piece, q_stride = (unsigned)a.q_stride;   // (launch_gemm() sees to it that offsets fit)
    const int first = min(nb0, n_blocks - 1), more = min(3, n_blocks - 1 - first);
    const auto w = buffer(a.packed + (size_t)first * column, (more + 1) * column);
    const auto x = buffer(a.Q + m0 * a.q_stride, (min(kRows, a.M - m0) - 1) * q_stride + ((a.K + 15) & ~15));
    const int c = threadIdx.x & 7, r0 = threadIdx.x >> 3;   // a thread's pieces: chunk c of rows r0, r0 + 32, ...
    const unsigned x_at = r0 * q_stride + c * 16;
    const int slot = ((r0 >> 4) * 8 + c) * 16 + ((r0 & 15) ^ c);
    i32x4 xr[kPieces], w0[2][4], w1[2][4], acc[4][MF] = {};
    auto load_x = [&](int step) {
        const unsigned at = step * kStepK + c * 16 < a.K ? x_at + step * kStepK : kOutside;
#pragma unroll
        for (int p = 0; p < kPieces; ++p) xr[p] = load16(x, at + p * 32 * q_stride, 0);
    };
    auto store_x = [&](int step) {
#pragma unroll
        for (int p = 0; p < kPieces; ++p) xs[step & 1][slot + p * 256] = xr[p];
    };
    auto load_w = [&](int step, int s, i32x4 (&to)[4]) {
#pragma unroll
        for (int j = 0; j < 4; ++j) to[j] = load16(w, lane * 16, min(j, more) * column + min(2 * step + s, k_blocks - 1) * kW8Piece);
    };
    auto meet = [&]() {
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
    };
    // One step.  As soon as a half of its W has been multiplied, the same registers are loaded for the step after the next.  X of
    // the next step, requested a step ago, goes into the other buffer, which was read in the step before; everybody has met since.
    auto compute = [&](int step, i32x4 (&wr)[2][4]) {
        const i32x4 *const from = xs[step & 1];
#pragma unroll
        for (int q = 0; q < 2 * MF; ++q) {
            const int s = q / MF, i = q % MF, chunk = 4 * s + (lane >> 4);
            const i32x4 xf = from[(i * 8 + chunk) * 16 + ((lane & 15) ^ chunk)];
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[j][i] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wr[s][j], xf, acc[j][i], 0, 0, 0);
            if (q == MF - 1) {
                load_w(step + 2, 0, wr[0]);
                store_x(step + 1);
                load_x(step + 2);
            }
        }
        load_w(step + 2, 1, wr[1]);
        // the order of issue: reads of X three ahead of their products; loads and stores between the products
        __builtin_amdgcn_sched_group_barrier(0x100, 3, 0);
#pragma unroll
        for (int q = 0; q < 2 * MF; ++q) {
            __builtin_amdgcn_sched_group_barrier(0x008, 2, 0);
            if (q >= MF && q < MF + kPieces) __builtin_amdgcn_sched_group_barrier(0x200, 1, 0);
            if (q >= MF && q < MF + 4) __builtin_amdgcn_sched_group_barrier(0x020, 2, 0);
            __builtin_amdgcn_sched_group_barrier(0x008, 2, 0);
            if (q < 2 * MF - 3) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
        meet();
    };
    load_x(0);
    load_w(0, 0, w0[0]);
    load_w(0, 1, w0[1]);
    store_x(0);
    load_x(1);
    load_w(1, 0, w1[0]);
    load_w(1, 1, w1[1]);
    meet();
    for (int step = 0;;) {   // (left, not skipped over: waits are counted along the paths there are)
        compute(step, w0);
        if (++step >= steps) break;
        compute(step, w1);
        if (++step >= steps) break;
    }

    float t[4][4], b[4][4];
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int n = min((nb0 + j) * 16 + 4 * (lane >> 4) + r, a.N - 1);
            t[j][r] = a.w_scale[n];
            b[j][r] = a.b ? a.b[n] : 0.f;
        }
#pragma unroll
    for (int i = 0; i < MF; ++i) {
        const int m = m0 + 16 * i + (lane & 15);
        const float s = a.scale[min(m, a.M - 1)];
        if (m < a.M) {
#pragma unroll
            for (int j = 0; j < 4; ++j) store4<TYPE>(a, m, (nb0 + j) * 16 + 4 * (lane >> 4), acc[j][i], s, t[j], b[j]);
        }
    }
}

hipError_t launch_gemm(const GemmArgs &a, int y_type, hipStream_t stream)
{
    const GemmTile tile = choose_tile(a.M, a.K, a.N, compute_units());
    const int m = blocks_of(a.M, 16 * tile.mt), n = blocks_of(a.N, 16 * tile.nt);
    return for_type(y_type, [&](auto type) {
        constexpr int T = decltype(type)::value;
        const dim3 grid(n, m);
        if (!tile.rows) {
            if (tile.mt == 4) k_w8_tiles<T, 4><<<m * n, kTileThreads, 0, stream>>>(a, m, n);
            else k_w8_tiles<T, 8><<<m * n, kTileThreads, 0, stream>>>(a, m, n);
        } else if (tile.nt == 1) {
            k_w8_rows<T, 1, 1><<<grid, kRowsThreads, 0, stream>>>(a);
        } else if (tile.nt == 4) {
            k_w8_rows<T, 4, 4><<<grid, kRowsThreads, 0, stream>>>(a);
        } else if (tile.mt == 1) {
            k_w8_rows<T, 1, 2><<<grid, kRowsThreads, 0, stream>>>(a);
        } else if (tile.mt == 2) {
            k_w8_rows<T, 2, 2><<<grid, kRowsThreads, 0, stream>>>(a);
        } else {
            k_w8_rows<T, 4, 2><<<grid, kRowsThreads, 0, stream>>>(a);
        }
        return hipGetLastError();
    });
}

hipError_t launch_quantize(const void *X, int type, int64_t x_stride, int8_t *Q, int64_t q_stride, float *scale, int M, int K,
                           hipStream_t stream)
{
    return for_type(type, [&](auto t) {
        typedef typename Entry<decltype(t)::value>::bits bits;
        constexpr int T = decltype(t)::value, V = 16 / sizeof(bits);
        const bool wide = aligned(X, 16) && K % V == 0 && x_stride % V == 0 && aligned(Q, V) && q_stride % V == 0;
        const bits *x = static_cast<const bits *>(X);
        // Few rows get more threads each.  With rows off 16-byte borders, an entry a load, 16 to 300 rows of 16384 bf16 take 8.6 us with 1024 threads
        // and 14 with 256, 1024 rows of 4096 11.1 and 8.9 (from Python); on borders the two differ by less than a call's own time.
        const bool few = M < compute_units();
        if (wide && few) k_quantize<T, true, 1024><<<M, 1024, 0, stream>>>(x, x_stride, Q, q_stride, scale, K);
        else if (few) k_quantize<T, false, 1024><<<M, 1024, 0, stream>>>(x, x_stride, Q, q_stride, scale, K);
        else
            for (int64_t m = 0; m < M; m += kLaunchRows) {
                const int rows = (int)(M - m < kLaunchRows ? M - m : kLaunchRows);
                if (wide) k_quantize<T, true, 256><<<rows, 256, 0, stream>>>(x + m * x_stride, x_stride, Q + m * q_stride, q_stride, scale + m, K);
                else k_quantize<T, false, 256><<<rows, 256, 0, stream>>>(x + m * x_stride, x_stride, Q + m * q_stride, q_stride, scale + m, K);
                if (hipError_t e = hipGetLastError()) return e;
            }
        return hipGetLastError();
    });
}

template <int TYPE>
hipError_t launch_few(const GemmArgs &a, const void *X, int64_t x_stride, hipStream_t stream)
{
    typedef typename Entry<TYPE>::bits bits;
    constexpr int V = 16 / sizeof(bits);
    const bits *x = static_cast<const bits *>(X);
    const bool wide = aligned(X, 16) && a.K % V == 0 && (a.M == 1 || x_stride % V == 0);
    k_w8_few<TYPE><<<blocks_of(a.N, kW8Cols), kRowsThreads, 0, stream>>>(a, x, x_stride, wide);
    return hipGetLastError();
}

// the most rows that a grid's second dimension holds with the smallest tile, and bytes between rows whose offsets in a tile fit 31 bits
constexpr int kMaxRows = 65535 * 16, kMaxStride = 1 << 22;
// the most columns: k_w8_rows and k_w8_few have 512 threads for 16 of them, and a dimension of a grid fewer than 2^32
constexpr int kMaxColumns = (1 << 27) - 16;

int check_gemm(const void *X, const void *packed, const float *w_scale, const void *Y, int type, int M, int K, int N)
{
    if (!type_ok(type) || M < 0 || M > kMaxRows || K < 1 || K > kW8MaxK || N < 1 || N > kMaxColumns) return TSTGEMM_EINVAL;
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
    if (!tst::type_ok(type) || M < 0 || K < 1 || K > 1 << 30 || x_stride < K || q_stride < K) return TSTGEMM_EINVAL;
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
    if ((int64_t)k_blocks * n_blocks * 64 > UINT32_MAX) return TSTGEMM_ETOOBIG;   // threads of a dimension of the grid
    tst::k_w8_pack<<<dim3(k_blocks * n_blocks, count), 64, 0, static_cast<hipStream_t>(stream)>>>(W, static_cast<char *>(packed), K, N,
                                                                                                 k_blocks, n_blocks);
    return tst::status(hipGetLastError());
}

int tst_w8_gemm(const int8_t *Q, int64_t q_stride, const float *scale, const void *packed, const float *w_scale, const float *b,
                void *Y, int y_type, int M, int K, int N, void *stream)
{
    if (int rc = tst::check_gemm(Q, packed, w_scale, Y, y_type, M, K, N)) return rc;
    if (M == 0) return TSTGEMM_OK;
    if (!scale || !tst::aligned(Q, 16) || (M > 1 && (q_stride < K || q_stride % 16 || q_stride > tst::kMaxStride))) return TSTGEMM_EINVAL;
    if (M == 1) q_stride = 0;
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
    if (M <= tst::kFewRows && (int64_t)M * tst::blocks_of(K, tst::kStepK) * tst::kStepK <= tst::kFewCodes)
        return tst::status(tst::for_type(type, [&](auto t) {
            return tst::launch_few<decltype(t)::value>(tst::gemm_args(nullptr, 0, nullptr, packed, w_scale, b, Y, type, M, K, N), X, x_stride,
                                                       static_cast<hipStream_t>(stream));
        }));
    const int64_t q_stride = (int64_t)tst::blocks_of(K, 64) * 64;
    int8_t *Q = static_cast<int8_t *>(workspace);
    float *scale = reinterpret_cast<float *>(Q + tst::round256((size_t)M * q_stride));
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (hipError_t e = tst::launch_quantize(X, type, x_stride, Q, q_stride, scale, M, K, s)) return tst::status(e);
    return tst::status(tst::launch_gemm(tst::gemm_args(Q, q_stride, scale, packed, w_scale, b, Y, type, M, K, N), type, s));
}

}  // extern "C"
