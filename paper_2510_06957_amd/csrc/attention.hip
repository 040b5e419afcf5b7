// Causal attention over whole prompts, packed one behind another, with grouped heads (tst_attention).
//
// A workgroup has a tile of rows of one key head, a row being (token, query head of the group), so that the keys and values that it loads serve all heads of
// the group, and goes through the keys from the first to the tile's last, 32 to 128 at a time, with the running largest logit and sum of each row.  Z^T = K Q^T and
// Y^T = V^T P^T with the 32 x 32 x 16 instructions: a row's logits, weights and sums stay in the lanes with its number (mod 32), and the weights are the second
// product's operand as they come out of the first, since keys may stand in any order there: lanes of half h hold keys 8 (r / 4) + 4 h + r % 4 of 32.
// K and V go through the LDS as rows; the second product's operand, four keys of a channel in a lane, comes out of it by reads that transpose.
//
// fp32 operands are cut into three bf16 planes by cutting mantissas off (exact) and six products of planes are summed: all but 2^-24 of a product.
//
// Matrix cores and vector units share the time: a weight costs 6 vector instructions (largest, exponential, sum, rounding, operands) beside 256 multiplications of heads of 128.  In bf16 the next 32 keys'
// logits are therefore made beside the weights of these.  8192 tokens, 32 query and 8 key heads of 128: 549 GFLOP in 548 to 555 us (1.0 PFLOP/s, matrix cores busy 44 % of the cycles; matrix
// instructions and barriers alone 287 us); heads of 64 321 to 333, 4096 tokens of 256 487, 24 prompts of up to 2048 264 to 268; 2048 tokens of fp32, 16 query heads, 153.
#include "attention_internal.h"

#include <cmath>

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
    float scale;   // its magnitude times log2 e; 2^-149 for 0, so that -inf stays what it is (and others are below 2^-21)
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

// How rows are read and dealt: anywhere, an entry at a time; on 16-byte borders; so, and few of them, in tiles of half the rows; so few that several wavefronts share
// the keys of the same rows and join their sums at the end.
enum Way { kAny, kFast, kFew, kShared };
template <int TYPE, int ROW, int WAY> struct Shape {
    static constexpr int kPlanes = Planes<TYPE>::kCount;
    static constexpr bool kAhead = (WAY == kFast || WAY == kFew) && TYPE != TST_F32;      // the next keys' logits beside these keys' weights
    static constexpr int kGroups = WAY != kShared ? 1 : TYPE == TST_F32 ? 2 : 4;           // wavefronts that share the keys of 32 rows
    static constexpr int kWaves = (kAhead && WAY == kFast && ROW <= 128) || (WAY == kShared && TYPE != TST_F32) ? 8 : 4;   // two for a SIMD where their registers fit
    static constexpr int kOccupancy = kAhead && ROW <= 64 ? 4 : (kAhead || (WAY == kShared && TYPE != TST_F32)) && ROW <= 128 ? 2 : 1;
    static constexpr int kThreads = 64 * kWaves, kRows = 32 * (kWaves / kGroups);          // of a tile
    static constexpr int kKeys = kAhead && WAY == kFast && ROW <= 128 ? 64 : 32 * kGroups;  // of a tile in the LDS
    // (kAhead: K's next tile is read while another wavefront still reads this one, and K is stored a tile ahead)
    static constexpr int kOfPlain = ROW <= 128 && (kGroups == 1 || TYPE != TST_F32) ? 2 : 1, kBuffersK = kAhead ? 3 : kOfPlain, kBuffersV = kAhead ? 2 : kOfPlain;
    // bytes from key to key: 16 rows of keys, and 4 rows of 32 channels of values, fall into different banks
    static constexpr int kStrideK = ROW * 2 + 16, kStrideV = ROW * 2 + (ROW % 128 == 96 ? 0 : 64);
    static constexpr int kPlaneK = kKeys * kStrideK, kPlaneV = kKeys * kStrideV;
    static constexpr int kBufferK = kPlanes * kPlaneK, kBufferV = kPlanes * kPlaneV;
    // results of a wavefront's 32 rows go through the LDS, where the tiles were, and out as rows
    static constexpr bool kByRows = kAhead;
    static constexpr int kStrideRow = ROW * 2 + 16, kRowsBytes = 32 * kStrideRow;
    static_assert(!kByRows || kWaves * kRowsBytes <= kBuffersK * kBufferK + kBuffersV * kBufferV, "rows fit where tiles were");
    static constexpr int kChunks = (kKeys * (ROW / 8) + kThreads - 1) / kThreads;   // of 8 entries that a thread stages, of K and as many of V
};

// Weights are 2^shift times those relative to the row's base, which the largest logit may pass by 2^kSlack before all is scaled anew: fp16 holds them with 11 bits
// down to 2^-21 of the largest.
constexpr float kSlack = 8.f;
template <int TYPE> constexpr float kShift = TYPE == TST_F16 ? 7.f : 0.f;
// Sums of up to 2^22 values with weights of up to 2^kSlack can pass 2^128 in bf16 and fp32 where their mean does not.  A tile with results that are not finite therefore goes through
// its keys again, with values 2^-32 times as large, and the rows that those results are of take what comes of that: the same bits, but for values below 2^-94.  (fp16 has no such values.)
constexpr float kLess = 0x1p-32f, kLargest = 3.402823466e38f;
template <int TYPE> constexpr bool kMayPass = TYPE != TST_F16;

// The tile of rows that workgroups of a number have, -1: none.  A sequence's tiles come one after another, since they read the same keys and values, the last,
// which sees most of them, first.  Of up to 64 sequences the shortest come first: what is left at the end are then the shortest tiles of the longest (4096 and 1024 tokens, 32
// heads of 128: 182 us, 190 the other way round); of more, the last.
struct Place {
    int first, n, tile;   // of the sequence: its first row and how many it has; tokens * query heads <= 2^27, so rows of tiles have 32 bits
};
__device__ __forceinline__ Place place_of(const PromptArgs &a, int rows, int number)
{
    const int lane = threadIdx.x % 64;
    if (a.sequences <= 64) {
        const Span span = lane < a.sequences ? span_of(a.offsets, a.tokens, lane) : Span{0, 0};
        const int mine = (span.n * a.group + rows - 1) / rows;
        int before = 0;     // tiles of shorter sequences
        for (int i = 0; i < a.sequences; ++i) {
            const int other = __builtin_amdgcn_readlane(mine, i);
            before += other < mine || (other == mine && i > lane) ? other : 0;
        }
        const int at = number - before;
        const unsigned long long here = __ballot(at >= 0 && at < mine);
        if (!here) return Place{0, 0, -1};
        const int seq = __ffsll(here) - 1;
        return Place{__builtin_amdgcn_readlane(span.first, seq), __builtin_amdgcn_readlane(span.n, seq), __builtin_amdgcn_readlane(mine - 1 - at, seq)};
    }
    // tiles of sequence i have the numbers from offsets[i] * group / rows + i on
    auto base = [&](int i) { return min(max(a.offsets[i], 0), a.tokens) * a.group / rows + i; };
    const int at = a.tiles - 1 - number;
    int seq = 0, n = a.sequences;
    while (n > 1) {
        const int step = (n + 63) / 64, i = seq + lane * step;
        const bool before = lane * step < n && base(min(i, a.sequences)) <= at;
        const int c = max(__popcll(__ballot(before)), 1) - 1;
        seq += c * step;
        n = min(step, n - c * step);
    }
    seq = uniform(seq);
    const Span span = span_of(a.offsets, a.tokens, seq);
    const int tile = at - base(seq);
    return Place{span.first, span.n, tile >= 0 && tile * (int64_t)rows < span.n * a.group ? tile : -1};
}

// A tile of keys or values on its way from memory to the LDS: 8 entries a chunk.
template <int TYPE, int ROW, int WAY> struct Staged {
    typedef Shape<TYPE, ROW, WAY> S;
    Raw<TYPE> raw[S::kChunks];
    const unsigned thread;
    __device__ __forceinline__ explicit Staged(unsigned t) : thread(t) {}
    __device__ __forceinline__ int key_of(int i) const { return (thread + S::kThreads * i) / (ROW / 8); }
    __device__ __forceinline__ int channel_of(int i) const { return (thread + S::kThreads * i) % (ROW / 8) * 8; }

    // the tile's keys; zeros behind `keys`
    __device__ __forceinline__ void load(const typename Entry<TYPE>::bits *data, int64_t stride, int tile, int keys, int size, bool wide)
    {
        const typename Entry<TYPE>::bits *at = data + (int64_t)tile * S::kKeys * stride;
        const int left = keys - tile * S::kKeys;
#pragma unroll
        for (int i = 0; i < S::kChunks; ++i) {
            const bool there = key_of(i) < min(left, S::kKeys);
            if constexpr (WAY != kAny) {
                // from somewhere in the tile whatever it is (zeros come in store()): a load that depends on the lane would have to be waited for
                // before the next.  (offsets within a tile have 32 bits)
                const int key = min(key_of(i), left - 1), channel = channel_of(i) < size ? channel_of(i) : 0;
                union {
                    u32x4 v[sizeof(Raw<TYPE>) / 16];
                    Raw<TYPE> r;
                } u;
#pragma unroll
                for (int w = 0; w < (int)(sizeof(u) / 16); ++w) u.v[w] = reinterpret_cast<const u32x4 *>(at + ((unsigned)key * (unsigned)stride + (unsigned)channel))[w];
                raw[i] = u.r;
            } else raw[i] = load_raw<TYPE>(at + key_of(i) * stride, channel_of(i), size, there, wide);
        }
    }
    // Values that some rows of the tile do not see: 0 times an infinity would be a NaN, so what is not finite becomes a 0, and the first such key of the channel
    // is remembered.
    __device__ __forceinline__ void mend(int tile, int *spoilt, int &any)
    {
        // whether there is one at all, by the largest bits without sign: a branch for each entry takes longer than the rest of the tile's way into the LDS (128 prompts of up to 128 tokens
        // 38.0 us, so 36.2; 24 of up to 2048 275.6 and 273.2)
        if constexpr (TYPE == TST_F32) {
            unsigned most = 0;
#pragma unroll
            for (int i = 0; i < S::kChunks; ++i)
#pragma unroll
                for (int e = 0; e < 8; ++e) most = max(most, __float_as_uint(raw[i].e[e]) & 0x7fffffffu);
            if (most < 0x7f800000u) return;
        } else {
            typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
            u16x2 most = {0, 0};
#pragma unroll
            for (int i = 0; i < S::kChunks; ++i) {
                unsigned two[4];
                __builtin_memcpy(two, raw[i].e, 16);
#pragma unroll
                for (int e = 0; e < 4; ++e) most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, two[e] & 0x7fff7fffu));
            }
            if (max(most[0], most[1]) < (TYPE == TST_BF16 ? 0x7f80 : 0x7c00)) return;
        }
#pragma unroll
        for (int i = 0; i < S::kChunks; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float x = Entry<TYPE>::get(raw[i].e[e]);
                if (!(x - x == 0.f)) {
                    raw[i].e[e] = 0;
                    atomicMin(&spoilt[channel_of(i) + e], tile * S::kKeys + key_of(i));
                    any = 1;
                }
            }
    }
    __device__ __forceinline__ void shrink()
    {
#pragma unroll
        for (int i = 0; i < S::kChunks; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) raw[i].e[e] = Entry<TYPE>::put(Entry<TYPE>::get(raw[i].e[e]) * kLess);
    }
    __device__ __forceinline__ void store(char *to, int stride, int plane, int left, int size)
    {
        if (WAY != kAny && (left < S::kKeys || size < ROW)) {
#pragma unroll
            for (int i = 0; i < S::kChunks; ++i)
                if (key_of(i) >= left || channel_of(i) >= size) raw[i] = Raw<TYPE>{};
        }
#pragma unroll
        for (int i = 0; i < S::kChunks; ++i) {
            if (key_of(i) >= S::kKeys) continue;
            const Planes<TYPE> x = planes_of<TYPE>(raw[i]);
#pragma unroll
            for (int p = 0; p < S::kPlanes; ++p) *reinterpret_cast<u32x4 *>(to + p * plane + key_of(i) * stride + channel_of(i) * 2) = x.p[p];
        }
    }
};

template <int TYPE, int ROW, int WAY> struct Shared {
    typedef Shape<TYPE, ROW, WAY> S;
    __attribute__((aligned(16))) char tiles[S::kBuffersK * S::kBufferK + S::kBuffersV * S::kBufferV];
    int spoilt[ROW];   // the first key whose value of the channel is not finite, among the keys that some of the tile's rows do not see
    int any_spoilt, any_passed;
};

// The results of a tile's rows; of those alone that `mine` says.  LESS: by values kLess times as large.  Whether the lane's row has results that are not finite, by values that it sees all of.
template <int TYPE, int ROW, int WAY, bool LESS> __device__ __forceinline__ bool attend(const PromptArgs &a, int tile, int n, int first, int head, Shared<TYPE, ROW, WAY> &shared, bool mine)
{
    typedef Shape<TYPE, ROW, WAY> S;
    typedef typename Entry<TYPE>::bits Bits;
    constexpr int P = S::kPlanes, kSteps = ROW / 16, kTiles = ROW / 32, kSub = S::kKeys / 32;   // 32 keys at a time
    char *const lds_k = shared.tiles, *const lds_v = lds_k + S::kBuffersK * S::kBufferK;
    int *const spoilt = shared.spoilt, &any_spoilt = shared.any_spoilt;
    unsigned thread = threadIdx.x;
    if constexpr (LESS) asm volatile("" : "+v"(thread));     // (or the compiler keeps what goes by it from the first time on)
    const int wave = uniform(thread / 64) % (S::kWaves / S::kGroups), sharer = uniform(thread / 64) / (S::kWaves / S::kGroups);   // of its rows; of those with the same
    const int lane = thread % 64, half = lane / 32, col = lane % 32;

    const unsigned group = a.group, rho0 = tile * S::kRows;
    const int first_token = rho0 / group, last_token = min((int)((rho0 + S::kRows - 1) / group), n - 1);
    const int keys = last_token + 1;          // that the tile sees
    const int tiles = (keys + S::kKeys - 1) / S::kKeys;

    const Bits *k_data = static_cast<const Bits *>(a.k.data) + (int64_t)first * a.k.token + head * a.k.head;
    const Bits *v_data = static_cast<const Bits *>(a.v.data) + (int64_t)first * a.v.token + head * a.v.head;
    Staged<TYPE, ROW, WAY> k_tile(thread), v_tile(thread), k_next(thread);
    auto load_k = [&](int kt) { k_tile.load(k_data, a.k.token, kt, keys, a.size, WAY != kAny || a.wide); };
    auto load_v = [&](int kt) { v_tile.load(v_data, a.v.token, kt, keys, a.size, WAY != kAny || a.wide); };
    load_k(0), load_v(0);
    if (S::kAhead && tiles > 1) k_next.load(k_data, a.k.token, 1, keys, a.size, true);

    for (int d = thread; d < ROW; d += S::kThreads) spoilt[d] = 0x7fffffff;
    if (thread == 0) any_spoilt = 0;

    u32x4 q[P][kSteps];
    const unsigned rho = rho0 + wave * 32 + col;
    const bool there = rho < (unsigned)n * group;
    const int token = there ? (int)(rho / group) : -1;
    const int q_head = head * a.group + (there ? (int)(rho - token * group) : 0);
    const int limit = token + 1;              // keys that the row sees
    {
        const Bits *row = static_cast<const Bits *>(a.q.data) + (int64_t)(first + max(token, 0)) * a.q.token + q_head * a.q.head;
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            Raw<TYPE> raw = load_raw<TYPE>(row, 16 * s + 8 * half, a.size, there, WAY != kAny || a.wide);
            if (a.negative) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    if constexpr (TYPE == TST_F32) raw.e[e] = -raw.e[e];
                    else raw.e[e] ^= 0x8000;
                }
            }
            const Planes<TYPE> x = planes_of<TYPE>(raw);
#pragma unroll
            for (int p = 0; p < P; ++p) q[p][s] = x.p[p];
        }
    }
    int least = there ? limit : 0x7fffffff, largest = limit;
    for (int d = 1; d < 32; d <<= 1) least = min(least, __shfl_xor(least, d)), largest = max(largest, __shfl_xor(largest, d));
    least = uniform(least) == 0x7fffffff ? 0 : uniform(least);
    const int own = (uniform(largest) + 31) / 32;   // times 32 keys that the wavefront's rows see

    f32x16 o[kTiles];
    float base = -INFINITY, sum = 0.f;     // logits are relative to base, in powers of two
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[t][r] = 0.f;

    auto store_k = [&](int kt) { k_tile.store(lds_k + kt % S::kBuffersK * S::kBufferK, S::kStrideK, S::kPlaneK, keys - kt * S::kKeys, a.size); };
    auto store_v = [&](int kt) {
        if ((kt + 1) * S::kKeys > first_token + 1) v_tile.mend(kt, spoilt, any_spoilt);
        if constexpr (LESS) v_tile.shrink();
        v_tile.store(lds_v + kt % S::kBuffersV * S::kBufferV, S::kStrideV, S::kPlaneV, keys - kt * S::kKeys, a.size);
    };

    typedef u32x4 Weights[P][2];
    auto first_product = [&](int sub, f32x16 &z) {
        const char *at = lds_k + sub / kSub % S::kBuffersK * S::kBufferK + (sub % kSub * 32 + col) * S::kStrideK + half * 16;
#pragma unroll
        for (int r = 0; r < 16; ++r) z[r] = 0.f;
#pragma unroll
        for (int step = 0; step < kSteps; ++step) {
            u32x4 k[P];
#pragma unroll
            for (int p = 0; p < P; ++p) k[p] = *reinterpret_cast<const u32x4 *>(at + p * S::kPlaneK + step * 32);
#pragma unroll
            for (int p = 0; p < P; ++p)
#pragma unroll
                for (int r = 0; p + r < P; ++r) z = product<TYPE>(k[p], q[r][step], z);
        }
    };
    auto mask = [&](int sub, f32x16 &z) {
        if ((sub + 1) * 32 > least) {
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if (sub * 32 + 8 * (r / 4) + 4 * half + r % 4 >= limit) z[r] = -INFINITY;
        }
    };
    auto rebase = [&](const f32x16 &z) {
        const float top = across_max(largest_of(z)) * a.scale;
        if (__any(top > base + kSlack)) {
            const float now = top > base + kSlack ? top : base, keep =   // (by the row itself alone)
                now == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(base - now);
            base = now;
            sum *= keep;
#pragma unroll
            for (int t = 0; t < kTiles; ++t) o[t] *= keep;
        }
    };
    auto weights = [&](const f32x16 &z, Weights &w) {
        const float from = base == -INFINITY ? 0.f : base - kShift<TYPE>;
        float p[16];
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            p[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(z[r], a.scale, -from));
            if constexpr (TYPE == TST_F32) sum += p[r];
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            if constexpr (TYPE == TST_F32) {
                Raw<TYPE> x;
#pragma unroll
                for (int i = 0; i < 8; ++i) x.e[i] = p[8 * j + i];
                const Planes<TYPE> px = planes_of<TYPE>(x);
#pragma unroll
                for (int q = 0; q < P; ++q) w[q][j] = px.p[q];
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const Pair<TYPE> pair = {(typename Pair<TYPE>::entry)p[8 * j + 2 * i], (typename Pair<TYPE>::entry)p[8 * j + 2 * i + 1]};
                    sum = pair.added(sum);
                    w[0][j][i] = pair.bits();
                }
            }
        }
    };
    auto second_product = [&](int sub, const Weights &w) {
        // four keys of a lane's channel: in each group of 16 lanes, lanes 4 r .. 4 r + 3 point to 16 channels of the r-th key
        const char *from = lds_v + sub / kSub % S::kBuffersV * S::kBufferV + (sub % kSub * 32 + 4 * half + lane % 16 / 4) * S::kStrideV + (col / 16 * 16 + lane % 4 * 4) * 2;
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
                        const char *at = from + p * S::kPlaneV + (16 * j + 8 * i) * S::kStrideV + t * 64;
                        part[i] = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)at));
                    }
                    v[p] = u32x4{part[0][0], part[0][1], part[1][0], part[1][1]};
                }
#pragma unroll
                for (int p = 0; p < P; ++p)
#pragma unroll
                    for (int r = 0; p + r < P; ++r) o[t] = product<TYPE>(v[p], w[r][j], o[t]);
            }
    };

    __syncthreads();     // spoilt is clear
    if constexpr (!S::kAhead) {
        store_k(0), store_v(0);
        __syncthreads();
        for (int kt = 0; kt < tiles; ++kt) {
            if (kt + 1 < tiles) load_k(kt + 1), load_v(kt + 1);
#pragma unroll
            for (int s = 0; s < kSub / S::kGroups; ++s) {
                const int sub = kt * kSub + s * S::kGroups + sharer;
                if (sub < own) {
                    f32x16 z;
                    Weights w;
                    first_product(sub, z);
                    mask(sub, z);
                    rebase(z);
                    weights(z, w);
                    second_product(sub, w);
                }
            }
            if (S::kBuffersK == 1) __syncthreads();     // everybody has read the only buffer
            if (kt + 1 < tiles) store_k(kt + 1), store_v(kt + 1);
            __syncthreads();
        }
    } else {
        // While the matrix cores work on the next 32 keys' logits, the other units make the weights of these, which they then take.  K is a tile ahead of V.
        f32x16 z[2];
        store_k(0), store_v(0);
        if (tiles > 1) k_next.store(lds_k + S::kBufferK, S::kStrideK, S::kPlaneK, keys - S::kKeys, a.size);
        __syncthreads();
        if (own > 0) {
            first_product(0, z[0]);
            mask(0, z[0]);
            rebase(z[0]);
        }
        auto inner = [&](int sub, f32x16 &now, f32x16 &next) {     // all rows see the next 32 keys
            Weights w;
            first_product(sub + 1, next);
            weights(now, w);
            __builtin_amdgcn_sched_barrier(0);
            second_product(sub, w);
            rebase(next);
        };
        auto last = [&](int sub, f32x16 &now, f32x16 &next) {      // some do not, or there are none
            if (sub >= own) return;
            Weights w;
            weights(now, w);
            second_product(sub, w);
            if (sub + 1 >= own) return;
            first_product(sub + 1, next);
            mask(sub + 1, next);
            rebase(next);
        };
        auto tile_step = [&](int kt, auto step, f32x16 &first, f32x16 &second) {
            if (kt + 2 < tiles) load_k(kt + 2);
            if (kt + 1 < tiles) load_v(kt + 1);
            step(kt * kSub, first, second);
            if constexpr (kSub == 2) step(kt * kSub + 1, second, first);
            if (kt + 2 < tiles) store_k(kt + 2);
            if (kt + 1 < tiles) store_v(kt + 1);
            __syncthreads();
        };
        int kt = 0;
        if constexpr (kSub == 2) {
            const int whole = (least / 32 - 1) / 2;
            for (; kt < whole; ++kt) tile_step(kt, inner, z[0], z[1]);
            for (; kt < tiles; ++kt) tile_step(kt, last, z[0], z[1]);
        } else {
            const int whole = (least / 32 - 1) / 2 * 2;
            for (; kt < whole; kt += 2) {
                tile_step(kt, inner, z[0], z[1]);
                tile_step(kt + 1, inner, z[1], z[0]);
            }
            for (; kt < tiles; kt += 2) {
                tile_step(kt, last, z[0], z[1]);
                if (kt + 1 < tiles) tile_step(kt + 1, last, z[1], z[0]);
            }
        }
    }

    sum = across_sum(sum);
    if constexpr (S::kGroups > 1) {
        // sharers' sums, relative to their own bases, through the LDS that held the tiles
        constexpr int kOthers = (S::kGroups - 1) * (S::kWaves / S::kGroups);
        static_assert(kOthers * 64 * (kTiles * 64 + 8) <= (int)sizeof(shared.tiles), "sums fit where tiles were");
        f32x4 *sums = reinterpret_cast<f32x4 *>(lds_k);
        float2 *states = reinterpret_cast<float2 *>(sums + kOthers * kTiles * 4 * 64);
        if (sharer > 0) {
            const int slot = (sharer - 1) * (S::kWaves / S::kGroups) + wave;
#pragma unroll
            for (int t = 0; t < kTiles; ++t)
#pragma unroll
                for (int r = 0; r < 16; r += 4) sums[((slot * kTiles + t) * 4 + r / 4) * 64 + lane] = f32x4{o[t][r], o[t][r + 1], o[t][r + 2], o[t][r + 3]};
            states[slot * 64 + lane] = float2{base, sum};
        }
        __syncthreads();
        if (sharer > 0) return false;
        float all = base;
#pragma unroll
        for (int i = 1; i < S::kGroups; ++i) all = fmaxf(all, states[((i - 1) * (S::kWaves / S::kGroups) + wave) * 64 + lane].x);
        const float from = all == -INFINITY ? 0.f : all, mine = __builtin_amdgcn_exp2f(base - from);
        sum *= mine;
#pragma unroll
        for (int t = 0; t < kTiles; ++t) o[t] *= mine;
#pragma unroll
        for (int i = 1; i < S::kGroups; ++i) {
            const int slot = (i - 1) * (S::kWaves / S::kGroups) + wave;
            const float2 state = states[slot * 64 + lane];
            const float w = __builtin_amdgcn_exp2f(state.x - from);
            sum += w * state.y;
#pragma unroll
            for (int t = 0; t < kTiles; ++t)
#pragma unroll
                for (int r = 0; r < 16; r += 4) {
                    const f32x4 v = sums[((slot * kTiles + t) * 4 + r / 4) * 64 + lane];
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[t][r + e] += w * v[e];
                }
        }
    }
    const float inverse = 1.f / sum;
    float most = 0.f;
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            float x = o[t][r] * inverse;
            asm("" : "+v"(x));     // rounded to fp32 however it is stored (else to fp16 at once where the compiler sees that)
            if constexpr (LESS)      // a mean is no larger than what it is of, however its last bits are rounded
                if (__builtin_fabsf(x) <= kLargest) x = fminf(fmaxf(x * (1.f / kLess), -kLargest), kLargest);
            if constexpr (kMayPass<TYPE>) most = __builtin_elementwise_maximum(most, __builtin_fabsf(x));
            o[t][r] = x;
        }
    const bool passed = kMayPass<TYPE> && !LESS && mine && there && !(across_max(most) <= kLargest);
    if (uniform(any_spoilt)) {     // (asked once: asked for each result, it took as long as the stores)
#pragma unroll
        for (int t = 0; t < kTiles; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if (spoilt[32 * t + 8 * (r / 4) + 4 * half + r % 4] < limit) o[t][r] = kNan;
    }
    if constexpr (S::kByRows) {
        // From the lanes as they are, 8 bytes of each of 32 rows, results took 2.6 us of every workgroup's (128 prompts of up to 128 tokens 42.6 us, so 37.3; 24 of up to 2048 276 and
        // 268).  In fp32 a lane has 16 bytes of a row, and it is the other way round (2048 tokens 215 and 219).
        if (((uintptr_t)a.y & 15) == 0) {
            constexpr int per = ROW * (int)sizeof(Bits) / 16, each = 16 / (int)sizeof(Bits);
            char *rows = lds_k + wave * S::kRowsBytes;
#pragma unroll
            for (int t = 0; t < kTiles; ++t)
#pragma unroll
                for (int r = 0; r < 16; r += 4) {
                    const int d = 32 * t + 2 * r + 4 * half;
                    Bits four[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) four[e] = Entry<TYPE>::put(o[t][r + e]);
                    __builtin_memcpy(__builtin_assume_aligned(rows + col * S::kStrideRow + d * (int)sizeof(Bits), 4 * sizeof(Bits)), four, sizeof(four));
                }
            order_wave();
            const int at = mine && there ? (first + token) * a.q_heads + q_head : -1;     // rows * query heads <= 2^27
#pragma unroll
            for (int i = 0; i < 32 * per / 64; ++i) {
                const int r = (lane + 64 * i) / per, d = (lane + 64 * i) % per * each, to = __shfl(at, r);
                const u32x4 v = *reinterpret_cast<const u32x4 *>(rows + r * S::kStrideRow + d * (int)sizeof(Bits));
                if (to >= 0 && d < a.size) *reinterpret_cast<u32x4 *>(static_cast<Bits *>(a.y) + (int64_t)to * a.size + d) = v;
            }
            return passed;
        }
    }
    if (!there || !mine) return false;
    Bits *out = static_cast<Bits *>(a.y) + ((int64_t)(first + token) * a.q_heads + q_head) * a.size;
    const bool whole = (a.size & 3) == 0 && ((uintptr_t)a.y & (4 * sizeof(Bits) - 1)) == 0;
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
            const int d = 32 * t + 2 * r + 4 * half;
            Bits four[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) four[e] = Entry<TYPE>::put(o[t][r + e]);
            if (whole) {
                if (d < a.size) __builtin_memcpy(__builtin_assume_aligned(out + d, 4 * sizeof(Bits)), four, sizeof(four));
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (d + e < a.size) out[d + e] = four[e];
            }
        }
    return passed;
}

template <int TYPE, int ROW, int WAY> __global__ void __launch_bounds__((Shape<TYPE, ROW, WAY>::kThreads), (Shape<TYPE, ROW, WAY>::kOccupancy)) k_attention(PromptArgs a)
{
    const int head = blockIdx.x % a.heads;
    const Place place = place_of(a, Shape<TYPE, ROW, WAY>::kRows, (int)(blockIdx.x / a.heads));
    if (place.tile < 0) return;
    const int tile = uniform(place.tile), n = uniform(place.n), first = uniform(place.first);
    __shared__ Shared<TYPE, ROW, WAY> shared;
    if (threadIdx.x == 0) shared.any_passed = 0;     // (seen by all behind the workgroup's first meeting)
    const bool passed = attend<TYPE, ROW, WAY, false>(a, tile, n, first, head, shared, true);
    if constexpr (kMayPass<TYPE>) {
        if (passed) shared.any_passed = 1;
        __syncthreads();
        if (uniform(shared.any_passed)) attend<TYPE, ROW, WAY, true>(a, tile, n, first, head, shared, passed);
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
        sequences > TST_MAX_SEQUENCES || tokens < 0 || tokens > TST_MAX_TOKENS || (int64_t)tokens * q_heads > TST_MAX_ROWS || (int64_t)sequences * heads > TST_MAX_SEQUENCE_HEADS || !tst::scale_ok(scale))
        return TSTGEMM_EINVAL;
    if (sequences == 0 || tokens == 0) return TSTGEMM_OK;
    if (!tst::rows_ok(Q, type) || !tst::rows_ok(K, type) || !tst::rows_ok(V, type) || !offsets || !tst::aligned(offsets, 4) || !Y || !tst::aligned(Y, tst::type_bytes(type)))
        return TSTGEMM_EINVAL;
    const int group = q_heads / heads;
    tst::PromptArgs a{tst::rows_of(Q), tst::rows_of(K), tst::rows_of(V), q_heads, heads, group, head_size, sequences, tokens, 0, offsets, std::fmax(std::fabs(scale) * tst::kLog2e, 0x1p-149f), scale < 0, Y, false};
    a.wide = tst::wide(a.q, type, head_size) && tst::wide(a.k, type, head_size) && tst::wide(a.v, type, head_size);
    return tst::status(tst::for_type(type, [&](auto t) {
        return tst::for_row(head_size, [&](auto r) {
            constexpr int TYPE = decltype(t)::value, ROW = decltype(r)::value;
            hipStream_t st = static_cast<hipStream_t>(stream);
            auto launch = [&](auto way) {
                constexpr int WAY = decltype(way)::value;
                typedef tst::Shape<TYPE, ROW, WAY> S;
                a.tiles = (int)((int64_t)tokens * group / S::kRows) + sequences;
                tst::k_attention<TYPE, ROW, WAY><<<(unsigned)a.tiles * heads, S::kThreads, 0, st>>>(a);
            };
            if (!a.wide || a.k.token > 1 << 24 || a.v.token > 1 << 24) launch(std::integral_constant<int, tst::kAny>{});
            else {
                const int64_t whole = (int64_t)tokens * group / tst::Shape<TYPE, ROW, tst::kFast>::kRows * heads;   // tiles
                if constexpr (ROW <= 128) {
                    // Rows whose keys are shared, where there are fewer tiles than compute units (fp32, whose tiles are half as large: than twice as many) and keys to share.  us, shared
                    // and not, 32 heads of 128, 8 of keys: bf16 128 tokens 11.0 and 10.4, 256 12.3 and 13.4, 512 15.8 and 20.1 (heads of 64 11.1 and 16.5), 1024 31.0 and 33.2;
                    // fp32 32 tokens 12.4 and 11.5, 48 12.5 and 13.2, 256 25 and 33, 1024 85 and 104, 2048 295 and 219
                    const bool few = TYPE == TST_F32 ? whole < 2 * tst::compute_units() && tokens > 32 * (int64_t)sequences
                                                     : whole < tst::compute_units() && tokens > 128 * (int64_t)sequences;
                    if (few) {
                        launch(std::integral_constant<int, tst::kShared>{});
                        return hipGetLastError();
                    }
                }
                if constexpr (TYPE != TST_F32 && ROW <= 128) {
                    // Tiles of half the rows, two workgroups on a compute unit, where whole ones would leave compute units without any or with one (us, half and whole: 2048 tokens 61.5
                    // and 66.5, 3000 94 and 97, 4096 168 and 150), and for prompts that are short, so that a tile's start and end hide behind another's keys.  Prompts x their mean, of
                    // lengths all the way from the longest down: 128 x 43 37.5 and 48.6, 64 x 175 112 and 130, 64 x 350 264 and 283, 32 x 536 229 and 234, 64 x 614 583 and 603, 24 x 637
                    // 224 and 223, 16 x 657 157 and 155, 64 x 700 717 and 727, 24 x 725 275 and 268, 128 x 518 807 and 804; heads of 64: 64 x 350 152 and 154, 24 x 637 138 and 134.
                    // Between means of 500 and 750 the two are within 3 % of one another, so the border is there.  It cannot go by how lengths are spread, which the device alone
                    // knows: of prompts all alike half tiles stay ahead longer (32 x 640 220 and 227, 32 x 768 285 and 307, 32 x 1024 443 and 461; 128 x 640 772 and 757).
                    if (2 * whole < 3 * tst::compute_units() || tokens <= 640 * (int64_t)sequences) {
                        launch(std::integral_constant<int, tst::kFew>{});
                        return hipGetLastError();
                    }
                }
                launch(std::integral_constant<int, tst::kFast>{});
            }
            return hipGetLastError();
        });
    }));
}

}  // extern "C"
