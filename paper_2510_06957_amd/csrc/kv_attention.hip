// Attention of new tokens over a paged cache of 8-bit keys and values (tst_kv_attention).
//
// Z^T = K Q^T and Y^T = V^T P^T, so that a query's logits, weights and sums stay in the lanes with its number (mod 16) from one product to the next: no
// lane hands a weight to another.  A wavefront takes 64 tokens, four blocks of 16, at a time: quarter g of its lanes holds the logits of block g, and with
// them one scale of keys and one of values.  The 16 x 16 x 32 instruction does not mind in which order the rows of its operands stand, so row m of the
// t-th tile of keys is token 4 t + m % 4 of block m / 4, and a lane's 16 weights are those that the 16 codes of one channel in its block's layout meet.
//
// Codes become fp16 exactly (1024 + code + 128 by its bits, less 1152).  A query's row is scaled by a power of two so that its largest entry is in [2^14, 2^15) and
// cut into fp16 (11 bits, and 11 more in a second plane for fp32).  Weights are multiplied by their value's scale, and the products are held relative to the largest of
// them so far, at 2^7 of which fp16 begins (fp32: 2^15): with 11 bits down to 2^-21 of the largest and 2^-32 of it below (22 bits down to 2^-18, and 2^-40).  It is the
// product that counts: relative to the largest scale, a block that weighs nothing would cost others their bits (or, 2^33 above theirs, all of them).  Sums are fp32.
//
// The keys of a long sequence are cut into equal chunks, about as long as those of the others: the device finds the length from the lengths of all sequences, so that
// the workgroups have about as much to do each whatever the batch is, and the host knows how many there are at most.  k_kv_join joins the chunks of a tile of rows.
//
// Memory bounds long caches: 131072 tokens of 8 heads of 128 behind one of 32 query heads are 268 MB in 44 us (6.1 TB/s, part of them from the Infinity Cache) and 7.6 us that join, 64 sequences
// of up to 8192 tokens 366 MB in 81 us (4.5 TB/s) and 7.  A unit's keys and the pages of the one behind it are on their way while the last is worked on; values, which are needed last, are
// requested first.  Widening codes takes the vector units about as long as the bytes take to come, so two workgroups share a compute unit where registers allow.
#include "attention_internal.h"

namespace tst {
namespace {

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

constexpr int kWaves = 4, kUnit = 64;   // tokens of a wavefront at a time
constexpr float kNan = __builtin_nanf("");
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLeastProduct = 1e-33f;   // that products are relative to: 2^15 over it is finite

struct KvArgs {
    Cache cache;
    Sequences seqs;
    Rows q;
    int q_heads, group;         // query heads of a key head
    int parts;                  // chunks of a head that its sequences are cut into, but for their ends; 0: no sequence is cut
    float scale;
    bool wide;                  // rows of Q on 16-byte borders, of a multiple of 8 entries
    void *y;
    f32x4 *sums;                // [heads][items][tiles][64 lanes]: a chunk's own results
    float2 *states;             // [heads][items][16 x row tiles]: largest logit, sum of weights
    int items;                  // of a head, at most
};

__device__ __forceinline__ int units_of(const KvArgs &a, int i)
{
    const int most = a.seqs.columns << a.cache.page_shift;   // a length behind the table's end meets one block that is not there
    return (min(max(a.seqs.lens[i], 0), most + 1) + kUnit - 1) / kUnit;
}
template <int ROWS> __device__ __forceinline__ int tiles_of(const KvArgs &a, int i)
{
    return (span_of(a.seqs.offsets, a.seqs.tokens, i).n * a.group + ROWS - 1) / ROWS;   // (tokens * query heads <= 2^27)
}

// Sums of the values of lanes up to this one; in lane 63 that of all.
__device__ __forceinline__ int64_t wave_scan(int64_t v)
{
    auto step = [&](auto control, auto rows) {
        const unsigned lo = (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, decltype(control)::value, decltype(rows)::value, 0xf, false);
        const int hi = __builtin_amdgcn_update_dpp(0, (int)(v >> 32), decltype(control)::value, decltype(rows)::value, 0xf, false);
        v += (int64_t)((uint64_t)(unsigned)hi << 32 | lo);
    };
    typedef std::integral_constant<int, 0xf> All;
    step(std::integral_constant<int, 0x111>{}, All{});   // row_shr 1
    step(std::integral_constant<int, 0x112>{}, All{});
    step(std::integral_constant<int, 0x114>{}, All{});
    step(std::integral_constant<int, 0x118>{}, All{});
    step(std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xa>{});   // row_bcast 15
    step(std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xc>{});   // row_bcast 31
    return v;
}
__device__ __forceinline__ int64_t lane_of(int64_t v, int lane)
{
    return (int64_t)((uint64_t)(unsigned)__builtin_amdgcn_readlane((int)(v >> 32), lane) << 32 | (unsigned)__builtin_amdgcn_readlane((int)v, lane));
}
__device__ __forceinline__ int64_t wave_sum(int64_t v) { return lane_of(wave_scan(v), 63); }

// About how long chunks are, in units of 64 tokens: all of them in a.parts equal ones.  Whole rounds of the four wavefronts.  Every wavefront of the call comes to the
// same length, which is no shorter than that.
template <int ROWS> __device__ __forceinline__ int chunk_length(const KvArgs &a)
{
    int64_t all = 0;
    for (int i = threadIdx.x % 64; i < a.seqs.count; i += 64) all += (int64_t)tiles_of<ROWS>(a, i) * units_of(a, i);
    const float length = (float)wave_sum(all) * (1.00001f / (float)a.parts) + 1.f;   // (a division of 64 bits takes a microsecond)
    return ((int)fminf(length, 1 << 30) + kWaves - 1) / kWaves * kWaves;
}

// A sequence is cut into so many equal chunks that they come nearest to that length: at most a.parts and one for each tile in all.
__device__ __forceinline__ int chunks_of(const KvArgs &a, int i, int length) { return max((int)((unsigned)(units_of(a, i) + length / 2) / (unsigned)length), 1); }

// Item `at`: sequences in order, a sequence's tiles in order, a tile's chunks in order.  seq -1: there are fewer.
struct Item {
    int seq, tile, chunk, chunks;   // chunks of the tile
};
template <int ROWS> __device__ __forceinline__ Item find_item(const KvArgs &a, int length, int64_t at)
{
    const int lane = threadIdx.x % 64;
    int64_t before = 0;
    for (int base = 0; base < a.seqs.count; base += 64) {
        const int i = base + lane;
        const int chunks = i < a.seqs.count ? chunks_of(a, i, length) : 1;
        const int64_t mine = i < a.seqs.count ? (int64_t)tiles_of<ROWS>(a, i) * chunks : 0;
        const int64_t upto = wave_scan(mine);
        const unsigned long long behind = __ballot(before + upto > at);
        if (behind) {
            const int l = __ffsll(behind) - 1;
            const int n = __builtin_amdgcn_readlane(chunks, l);
            const int rest = (int)(at - (before + lane_of(upto, l) - lane_of(mine, l)));
            return Item{base + l, (int)((unsigned)rest / (unsigned)n), (int)((unsigned)rest % (unsigned)n), n};
        }
        before += lane_of(upto, 63);
    }
    return Item{-1, 0, 0, 0};
}
template <int ROWS> __device__ __forceinline__ int64_t items_before(const KvArgs &a, int seq, int length)
{
    int64_t n = 0;
    for (int i = threadIdx.x % 64; i < seq; i += 64) n += (int64_t)tiles_of<ROWS>(a, i) * chunks_of(a, i, length);
    return wave_sum(n);
}

// Tiles of sequence i have the numbers from offsets[i] * group / rows + i on.  tile -1: a number that none has.
struct Slot {
    int seq, tile;
};
template <int ROWS> __device__ __forceinline__ Slot find_slot(const KvArgs &a, int at)
{
    const int lane = threadIdx.x % 64;
    auto base = [&](int i) { return (a.seqs.offsets ? min(max(a.seqs.offsets[i], 0), a.seqs.tokens) : i) * a.group / ROWS + i; };
    int lo = 0, n = a.seqs.count;
    while (n > 1) {
        const int step = (n + 63) / 64, i = lo + lane * step;
        const bool before = lane * step < n && base(min(i, a.seqs.count - 1)) <= at;
        const int c = max(__popcll(__ballot(before)), 1) - 1;
        lo += c * step;
        n = min(step, n - c * step);
    }
    lo = uniform(lo);
    const int tile = uniform(at - base(lo));
    return Slot{lo, tile >= 0 && tile < tiles_of<ROWS>(a, lo) ? tile : -1};
}

// Four codes as fp16: 1024 + (code + 128) by its bits, less 1152.
__device__ __forceinline__ void widen(unsigned four, f16x2 &lo, f16x2 &hi)
{
    const unsigned u = four ^ 0x80808080u;
    const f16x2 off = {(_Float16)-1152.f, (_Float16)-1152.f};
    lo = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(u, 0x64646464u, 0x00050004u)) + off;
    hi = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(u, 0x64646464u, 0x00070006u)) + off;
}
__device__ __forceinline__ f16x8 widen8(unsigned a, unsigned b)
{
    f16x2 v[4];
    widen(a, v[0], v[1]);
    widen(b, v[2], v[3]);
    return __builtin_shufflevector(__builtin_shufflevector(v[0], v[1], 0, 1, 2, 3), __builtin_shufflevector(v[2], v[3], 0, 1, 2, 3), 0, 1, 2, 3, 4, 5, 6, 7);
}

template <int TYPE, int ROW, int RT> struct Shape {
    static constexpr int kPlanes = TYPE == TST_F32 ? 2 : 1;
    static constexpr int kSteps = ROW / 32;      // of 32 channels
    static constexpr int kWide = ROW / 64;       // loads of 16 bytes of a lane in a row of keys; 8 more bytes where ROW % 64 = 32
    static constexpr int kTiles = ROW / 16;      // of 16 channels
    // Products of weights and scales are kShift times those relative to the largest by which all was last scaled; what comes later may pass it kProductSlack times, and a logit the
    // largest by kSlack, before all is scaled anew.  fp16 holds 2^15.  fp32 has no room for that: the second plane's bits reach 2^-24.
    static constexpr float kShift = TYPE == TST_F32 ? 32768.f : 128.f, kSlack = TYPE == TST_F32 ? 0.f : 6.f, kProductSlack = TYPE == TST_F32 ? 1.f : 256.f;
};
// The channel that entry i of step j stands for in a lane of quarter g: 16 bytes of a row are two steps.
template <int ROW> __device__ __forceinline__ int channel(int j, int g) { return j < ROW / 64 * 2 ? j / 2 * 64 + g * 16 + j % 2 * 8 : j / 2 * 64 + g * 8; }

template <int TYPE, int ROW, int RT> struct Keys {
    u32x4 wide[4][Shape<TYPE, ROW, RT>::kWide];
    u32x2 rest[4];
};
// The entry of the page table that a lane's block goes by, on its way.
struct Page {
    int entry;
    bool in_table;
};

// The largest of the four quarters' values of a lane's number (mod 16); a NaN does not count.
__device__ __forceinline__ float quarters_max(float v)
{
    auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    const float m = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(m), __float_as_uint(m), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// Adds what another wavefront or chunk has, relative to largest logits of its own.
__device__ __forceinline__ float weight_of(float m, float all) { return m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - all); }

// A mean of values is no larger than they are, however its last bits are rounded.
template <int TYPE> __device__ __forceinline__ float bounded(float v)
{
    if constexpr (TYPE != TST_F32) return v;
    else return __builtin_elementwise_minimum(__builtin_elementwise_maximum(v, -3.402823466e38f), 3.402823466e38f);   // (a NaN stays one)
}

// o: sums of weights and values, in units of `unit` times the sum of weights.
template <int TYPE, int ROW, int RT> __device__ __forceinline__ void write_rows(const KvArgs &a, const Span &rows, int tile, int head, const f32x4 (&o)[RT][ROW / 16], const float (&sum)[RT], const float (&unit)[RT],
                                                                                const int (&limit)[RT])
{
    typedef typename Entry<TYPE>::bits Bits;
    const int lane = threadIdx.x % 64, g = lane / 16, size = a.cache.size;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const unsigned rho = tile * (16 * RT) + rt * 16 + lane % 16;
        if (rho >= (unsigned)(rows.n * a.group)) continue;
        const int t = rho / (unsigned)a.group, h = head * a.group + (int)(rho - t * a.group);
        Bits *out = static_cast<Bits *>(a.y) + ((int64_t)(rows.first + t) * a.q_heads + h) * size;
        const float inverse = limit[rt] == 0 ? 0.f : 1.f / sum[rt];
        const bool whole = (size & 3) == 0 && ((uintptr_t)a.y & (4 * sizeof(Bits) - 1)) == 0;
#pragma unroll
        for (int dt = 0; dt < ROW / 16; ++dt) {
            const int d = 16 * dt + 4 * g;
            Bits b[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) b[e] = Entry<TYPE>::put(bounded<TYPE>(o[rt][dt][e] * inverse * unit[rt]));
            if (whole) {
                if (d < size) __builtin_memcpy(__builtin_assume_aligned(out + d, 4 * sizeof(Bits)), b, sizeof(b));
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (d + e < size) out[d + e] = b[e];
            }
        }
    }
}

template <int TYPE, int ROW, int RT> __global__ void __launch_bounds__(64 * kWaves, ROW * RT <= 128 && TYPE != TST_F32 ? 2 : 1) k_kv_attention(KvArgs a)
{
    typedef Shape<TYPE, ROW, RT> S;
    typedef typename Entry<TYPE>::bits Bits;
    __shared__ f32x4 shared[kWaves / 2][RT * S::kTiles][64];
    __shared__ float2 states[kWaves][RT][16];
    __shared__ float references[kWaves][RT][16];
    const int wave = uniform(threadIdx.x / 64), lane = threadIdx.x % 64, g = lane / 16, m16 = lane % 16, head = blockIdx.y;
    Item it;
    int begin = 0, end = 0;
    if (a.parts) {
        const int length = uniform(chunk_length<16 * RT>(a));
        it = find_item<16 * RT>(a, length, blockIdx.x);
        if (it.seq < 0) return;
        const int units = units_of(a, it.seq), each = (unsigned)units / (unsigned)it.chunks, longer = units - each * it.chunks;   // the first ones by a unit
        begin = it.chunk * each + min(it.chunk, longer);
        end = begin + each + (it.chunk < longer);
    } else {
        const Slot slot = find_slot<16 * RT>(a, blockIdx.x);
        if (slot.tile < 0) return;
        it = Item{slot.seq, slot.tile, 0, 1};
        end = units_of(a, slot.seq);
    }
    const int seq = uniform(it.seq), tile = uniform(it.tile);
    begin = uniform(begin), end = uniform(end);
    const Span rows = span_of(a.seqs.offsets, a.seqs.tokens, seq);
    const int len = max(a.seqs.lens[seq], 0);

    // queries
    f16x8 q[RT][S::kPlanes][S::kSteps];
    // A logit is a sum of products times scale, log2 e, the keys' scale and 2^-up: mantissas and exponents apart, since the factors may be beyond 32 bits where logits are not.
    const float scale_mantissa = __builtin_amdgcn_frexp_mantf(a.scale) * (kLog2e / 2);
    const int scale_exponent = __builtin_amdgcn_frexp_expf(a.scale) + 1;
    float valid[RT]; // 1, or NaN for a row of Q that holds what is not finite
    int up[RT], limit[RT];   // keys that the row sees
    int least = INT_MAX;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const unsigned rho = tile * (16 * RT) + rt * 16 + m16;
        const bool there = rho < (unsigned)(rows.n * a.group);
        const int t = there ? rho / (unsigned)a.group : 0, h = head * a.group + (there ? (int)(rho - t * a.group) : 0);
        const Bits *row = static_cast<const Bits *>(a.q.data) + (int64_t)(rows.first + t) * a.q.token + h * a.q.head;
        limit[rt] = there ? max(len - rows.n + t + 1, 0) : 0;
        if (there) least = min(least, limit[rt]);
        float x[S::kSteps][8];
        unsigned most = 0;
#pragma unroll
        for (int j = 0; j < S::kSteps; ++j) {
            const int d = channel<ROW>(j, g);
            if (a.wide) {
                union {
                    u32x4 v[sizeof(Bits) / 2];
                    Bits e[8];
                } raw;
#pragma unroll
                for (int i = 0; i < (int)sizeof(Bits) / 2; ++i) raw.v[i] = d < a.cache.size ? reinterpret_cast<const u32x4 *>(row + d)[i] : u32x4{0, 0, 0, 0};
#pragma unroll
                for (int e = 0; e < 8; ++e) x[j][e] = there ? Entry<TYPE>::get(raw.e[e]) : 0.f;
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) x[j][e] = there && d + e < a.cache.size ? Entry<TYPE>::get(row[d + e]) : 0.f;
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) most = max(most, __float_as_uint(x[j][e]) & 0x7fffffffu);
        }
        most = max(most, (unsigned)__shfl_xor((int)most, 16));
        most = max(most, (unsigned)__shfl_xor((int)most, 32));
        const bool finite = most < 0x7f800000u;
        up[rt] = most == 0 || !finite ? 0 : 15 - __builtin_amdgcn_frexp_expf(__uint_as_float(most));
        valid[rt] = finite ? 1.f : kNan;
#pragma unroll
        for (int j = 0; j < S::kSteps; ++j)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float v = finite ? __builtin_ldexpf(x[j][e], up[rt]) : 0.f;
                const _Float16 hi = (_Float16)v;
                q[rt][0][j][e] = hi;
                if constexpr (S::kPlanes == 2) q[rt][1][j][e] = (_Float16)(v - (float)hi);
            }
    }
    for (int d = 1; d < 16; d <<= 1) least = min(least, __shfl_xor(least, d));
    least = uniform(least);   // all rows see the keys below this

    f32x4 o[RT][S::kTiles];
    // What a row's weights are relative to, and its products of weights and scales (those weights), by what the row itself sees alone; kShift over the latter.
    float most[RT], reference[RT], inverse[RT], sum[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        most[rt] = -INFINITY, sum[rt] = 0.f, reference[rt] = kLeastProduct, inverse[rt] = S::kShift / kLeastProduct;
#pragma unroll
        for (int dt = 0; dt < S::kTiles; ++dt) o[rt][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    // Loads do not depend on the lane or on what was loaded, so that each is waited for by itself: behind the last unit that one again, in place of pages that are none
    // page 0, whose scale becomes a NaN then (0 behind the sequence's end).
    const int32_t *table = a.seqs.table + seq * a.seqs.stride;
    const int page_blocks = a.cache.page_shift - 4, last = max(end - 1, 0);
    auto load_page = [&](int block) {
        const int column = block >> page_blocks;
        return Page{table[min(column, a.seqs.columns - 1)], column < a.seqs.columns};
    };
    auto is_page = [&](const Page &p) { return p.in_table && (unsigned)p.entry < (unsigned)a.cache.pages; };
    auto lies = [&](const Page &p, int block) { return block_at(a.cache, is_page(p) ? p.entry : 0, head, block); };
    auto scale_of = [&](float loaded, const Page &p, int block) { return block * kKvBlock >= len ? 0.f : is_page(p) ? loaded : kNan; };
    Keys<TYPE, ROW, RT> keys;
    auto load_keys = [&](int u, const Page &page) {
        const int block = 4 * u + m16 / 4;
        const int8_t *at = a.cache.k + (lies(page, block) * kKvBlock + m16 % 4) * ROW + g * 16;
#pragma unroll
        for (int t = 0; t < 4; ++t) {
#pragma unroll
            for (int w = 0; w < S::kWide; ++w) keys.wide[t][w] = *reinterpret_cast<const u32x4 *>(at + 4 * t * ROW + 64 * w);
            if constexpr (ROW % 64 != 0) keys.rest[t] = *reinterpret_cast<const u32x2 *>(at + 4 * t * ROW + 64 * S::kWide - g * 8);
        }
    };

    // The unit at hand and the next: its keys' page, its values' page, its scales; pages of the one behind.
    int u = begin + wave;
    if (u < end) {
        Page k_page = load_page(4 * u + m16 / 4), v_page = load_page(4 * u + g);
        int next = min(u + kWaves, last);
        Page k_next = load_page(4 * next + m16 / 4), v_next = load_page(4 * next + g);
        load_keys(u, k_page);
        int64_t v_place = lies(v_page, 4 * u + g);
        float k_loaded = a.cache.k_scale[v_place], v_loaded = a.cache.v_scale[v_place];
        for (; u < end; u += kWaves) {
            u32x4 values[S::kTiles];
            const int8_t *v_at = a.cache.v + (v_place * ROW + m16) * kKvBlock;
#pragma unroll
            for (int dt = 0; dt < S::kTiles; ++dt) values[dt] = *reinterpret_cast<const u32x4 *>(v_at + 16 * dt * kKvBlock);
            __builtin_amdgcn_sched_barrier(0);   // or the compiler moves the loads behind the work that hides them

            f32x4 z[RT][4];
#pragma unroll
            for (int t = 0; t < 4; ++t) {
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) z[rt][t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int j = 0; j < S::kSteps; ++j) {
                    const f16x8 k = j < 2 * S::kWide ? widen8(keys.wide[t][j / 2][j % 2 * 2], keys.wide[t][j / 2][j % 2 * 2 + 1]) : widen8(keys.rest[t][0], keys.rest[t][1]);
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                        for (int p = 0; p < S::kPlanes; ++p) z[rt][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k, q[rt][p][j], z[rt][t], 0, 0, 0);
                }
            }
            const float k_scale = scale_of(k_loaded, v_page, 4 * u + g), v_scale = scale_of(v_loaded, v_page, 4 * u + g);
            __builtin_amdgcn_sched_barrier(0);
            load_keys(next, k_next);
            v_place = lies(v_next, 4 * next + g);
            k_loaded = a.cache.k_scale[v_place], v_loaded = a.cache.v_scale[v_place];
            v_page = v_next;
            next = min(next + kWaves, last);
            k_next = load_page(4 * next + m16 / 4), v_next = load_page(4 * next + g);
            __builtin_amdgcn_sched_barrier(0);

            const bool cut = (u + 1) * kUnit > least;
            bool anew = false;
            const float mantissa = scale_mantissa * __builtin_amdgcn_frexp_mantf(k_scale);
            const int exponent = scale_exponent + __builtin_amdgcn_frexp_expf(k_scale);
            float top[RT], v_own[RT];     // v_own: 0 for a block that the row does not see
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                // at most 2^128 times a mantissa below 1: 0 times an infinity would be a NaN
                const float f = __builtin_ldexpf(mantissa * valid[rt], min(exponent - up[rt], 128));
                top[rt] = -INFINITY;
#pragma unroll
                for (int t = 0; t < 4; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e) z[rt][t][e] *= f;
                v_own[rt] = v_scale;
                if (cut) {
                    const int from = u * kUnit + g * kKvBlock;
                    if (from >= limit[rt]) v_own[rt] = 0.f;
#pragma unroll
                    for (int t = 0; t < 4; ++t)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (from + 4 * t + e >= limit[rt]) z[rt][t][e] = -INFINITY;
                }
#pragma unroll
                for (int t = 0; t < 4; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e) top[rt] = fmaxf(top[rt], z[rt][t][e]);
                // (where nothing was seen before, the first question says it)
                anew |= top[rt] > most[rt] + S::kSlack || __builtin_amdgcn_exp2f(top[rt] - most[rt]) * v_own[rt] > reference[rt] * S::kProductSlack;
            }
            if (__any(anew)) {
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
                    const float t = quarters_max(top[rt]), now = t > most[rt] + S::kSlack ? t : most[rt];
                    const float keep = now == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(most[rt] - now), was = fmaxf(keep * reference[rt], kLeastProduct);
                    const float v = quarters_max(__builtin_amdgcn_exp2f(top[rt] - now) * v_own[rt]), largest = v > was * S::kProductSlack ? v : was;
                    const float times = keep * reference[rt] / largest;     // 1 for a row that asked for nothing
                    most[rt] = now, reference[rt] = largest, inverse[rt] = S::kShift / largest;
                    sum[rt] *= keep;
#pragma unroll
                    for (int dt = 0; dt < S::kTiles; ++dt) o[rt][dt] *= times;
                }
            }
            f16x8 w[RT][S::kPlanes][2];
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                const float base = most[rt] == -INFINITY ? 0.f : most[rt];
                float s = 0.f;
#pragma unroll
                for (int t = 0; t < 4; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float p = __builtin_amdgcn_exp2f(z[rt][t][e] - base);
                        s += p;
                        float x = p * v_own[rt] * inverse[rt];     // (the scale over the reference may be beyond 32 bits)
                        if (cut) x = z[rt][t][e] == -INFINITY ? 0.f : x;
                        const _Float16 hi = (_Float16)x;
                        w[rt][0][t / 2][t % 2 * 4 + e] = hi;
                        if constexpr (S::kPlanes == 2) w[rt][1][t / 2][t % 2 * 4 + e] = (_Float16)(x - (float)hi);
                    }
                sum[rt] += s;
            }
#pragma unroll
            for (int dt = 0; dt < S::kTiles; ++dt)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const f16x8 v = widen8(values[dt][2 * j], values[dt][2 * j + 1]);
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                        for (int p = 0; p < S::kPlanes; ++p) o[rt][dt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, w[rt][p][j], o[rt][dt], 0, 0, 0);
                }
        }
    }

    // the wavefronts' sums: relative to the largest logit of all, and to the largest reference, so that they stay as far from the ends of 32 bits as they are; then two and two
    float all[RT], total[RT], unit[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        sum[rt] += __shfl_xor(sum[rt], 16);
        sum[rt] += __shfl_xor(sum[rt], 32);
        if (g == 0) states[wave][rt][m16] = float2{most[rt], sum[rt]}, references[wave][rt][m16] = reference[rt];
    }
    __syncthreads();
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        all[rt] = -INFINITY, total[rt] = 0.f;
        float common = kLeastProduct;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) all[rt] = fmaxf(all[rt], states[w][rt][m16].x);
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const float weight = weight_of(states[w][rt][m16].x, all[rt]);
            total[rt] += states[w][rt][m16].y * weight;
            common = fmaxf(common, references[w][rt][m16] * weight);
        }
        unit[rt] = common * (1.f / S::kShift);
        const float times = weight_of(most[rt], all[rt]) * reference[rt] / common;
#pragma unroll
        for (int dt = 0; dt < S::kTiles; ++dt) o[rt][dt] *= times;   // (a NaN of a row whose weights here are nothing beside others stays one)
    }
#pragma unroll
    for (int half = kWaves / 2; half; half >>= 1) {
        if (wave >= half && wave < 2 * half)
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                for (int dt = 0; dt < S::kTiles; ++dt) shared[wave - half][rt * S::kTiles + dt][lane] = o[rt][dt];
        __syncthreads();
        if (wave < half)
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                for (int dt = 0; dt < S::kTiles; ++dt) o[rt][dt] += shared[wave][rt * S::kTiles + dt][lane];
        __syncthreads();
    }
    if (wave != 0) return;
    if (it.chunks == 1) {
        write_rows<TYPE, ROW, RT>(a, rows, tile, head, o, total, unit, limit);
        return;
    }
    const int64_t place = (int64_t)head * a.items + blockIdx.x;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const float inverse = total[rt] == 0.f ? 0.f : 1.f / total[rt];     // (where nothing weighs anything sums are 0, or NaN)
#pragma unroll
        for (int dt = 0; dt < S::kTiles; ++dt) a.sums[(place * (RT * S::kTiles) + rt * S::kTiles + dt) * 64 + lane] = o[rt][dt] * inverse * unit[rt];
        if (g == 0) a.states[place * (RT * 16) + rt * 16 + m16] = float2{all[rt], total[rt]};
    }
}

// Joins the chunks of a tile, 16 channels of 16 rows at a time: where there are few tiles, each such part is a workgroup's, whose wavefronts share the chunks, else a
// wavefront's, one after another.  Chunks have results of their own, of which this is the mean: nothing in between is larger than they are.
template <int TYPE, int ROW, int RT> __global__ void __launch_bounds__(64 * kWaves) k_kv_join(KvArgs a)
{
    typedef typename Entry<TYPE>::bits Bits;
    constexpr int kTiles = ROW / 16;
    __shared__ f32x4 shared[kWaves][64];
    const int wave = uniform(threadIdx.x / 64), lane = threadIdx.x % 64, g = lane / 16, m16 = lane % 16, head = blockIdx.y;
    const Slot slot = find_slot<16 * RT>(a, blockIdx.x);
    if (slot.tile < 0) return;
    const int length = uniform(chunk_length<16 * RT>(a)), chunks = chunks_of(a, slot.seq, length);
    if (chunks == 1) return;
    const int64_t first = items_before<16 * RT>(a, slot.seq, length) + (int64_t)slot.tile * chunks;
    const int n = (int)min((int64_t)chunks, a.items - first);   // (fewer where offsets do not ascend)
    const int64_t place = (int64_t)head * a.items + first;
    const Span rows = span_of(a.seqs.offsets, a.seqs.tokens, slot.seq);
    const int sees_from = rows.n - max(a.seqs.lens[slot.seq], 0), size = a.cache.size;   // tokens of the call below it see nothing
    const bool share = gridDim.z > 1;
    for (int part = share ? blockIdx.z : wave; part < RT * kTiles; part += share ? RT * kTiles : kWaves) {
        const int rt = part / kTiles, dt = part % kTiles;
        const float2 *states = a.states + place * (RT * 16) + rt * 16 + m16;
        const f32x4 *sums = a.sums + (place * (RT * kTiles) + part) * 64 + lane;
        // the largest logit, and the sum of weights relative to it: a quarter's lanes have every fourth chunk
        float own = -INFINITY, total = 0.f;
#pragma unroll 4
        for (int c = g; c < n; c += 4) {
            const float2 s = states[(int64_t)c * (RT * 16)];
            const float now = fmaxf(own, s.x);
            total = total * weight_of(own, now) + s.y * weight_of(s.x, now);
            own = now;
        }
        const float all = quarters_max(own);
        total *= weight_of(own, all);
        total += __shfl_xor(total, 16);
        total += __shfl_xor(total, 32);
        const float inverse = 1.f / total;
        f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
        for (int c = share ? wave : 0; c < n; c += share ? kWaves : 1) {
            const float2 s = states[(int64_t)c * (RT * 16)];
            const f32x4 v = sums[(int64_t)c * (RT * kTiles) * 64];
            o += weight_of(s.x, all) * s.y * inverse * v;
        }
        if (share) {
            shared[wave][lane] = o;
            __syncthreads();
            if (wave != 0) return;
            for (int w = 1; w < kWaves; ++w) o += shared[w][lane];
        }
        const unsigned rho = slot.tile * (16 * RT) + rt * 16 + m16;
        if (rho >= (unsigned)(rows.n * a.group)) continue;
        const int t = rho / (unsigned)a.group, h = head * a.group + (int)(rho - t * a.group);
        Bits *out = static_cast<Bits *>(a.y) + ((int64_t)(rows.first + t) * a.q_heads + h) * size;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (16 * dt + 4 * g + e < size) out[16 * dt + 4 * g + e] = Entry<TYPE>::put(t >= sees_from ? bounded<TYPE>(o[e]) : 0.f);
    }
}

// How a call is cut.  To know the chunks every workgroup reads all lengths, and their sums make a second launch: 5 us and more, which short sequences do not give back.
// No sequence of at most kShort units is cut, and none of up to kMiddle where the tiles of all heads are enough to share the card in turns (us, cut and whole, 32 query and 8
// key heads of 128, sequences x tokens of the table: 1 x 500 12.5 and 9.5, 64 x 2000 36.9 and 30.0, 128 x 2000 62.5 and 52.7, 64 x 4000 55.7 and 55.4, 8 x 4000 19.8 and 28.2,
// 64 x 8000 88 and 101, 16 x 16000 48 and 102).  Else the sequences of a head are cut into about as many chunks as the card holds workgroups of it where these are more than
// twice the tiles, and into twice as many where not, since lengths are uneven and a second turn fills what the first leaves (once, twice and three times: 64 sequences of up to
// 8192 96.0, 90.2 and 91.2; 8 of 8000 in 32 rows each 88, 82 and 87; 64 of 8000 alike 188, 199 and 205).
constexpr int kShort = 32, kMiddle = 80;
struct Cut {
    int row_tiles, parts;
    int64_t tiles, items;   // of a head, at most
    size_t states, total;
};
Cut cut_of(const tst_kv_cache_t *c, const tst_sequences_t *s, int q_heads)
{
    Cut k{};
    const int group = q_heads / c->heads, row = kv_row(c->head_size);
    const int64_t rows = (int64_t)s->tokens * group;   // of a key head
    k.row_tiles = s->sequences && rows > (int64_t)s->sequences * 16 && row <= 128 ? 2 : 1;
    k.tiles = rows / (16 * k.row_tiles) + s->sequences;
    const int slots = blocks_of((row * k.row_tiles <= 128 ? 2 : 1) * compute_units(), c->heads);   // by the kernels' registers
    const int64_t longest = ((int64_t)s->columns * c->page_tokens + kUnit) / kUnit;   // units that a sequence can have
    const bool whole = longest <= kShort || (longest <= kMiddle && 3 * longest <= k.tiles * c->heads);
    if (s->sequences <= 1024 && k.tiles <= 16 * (int64_t)slots && !whole) k.parts = 2 * k.tiles > slots ? 2 * slots : slots;
    k.items = k.tiles + k.parts;
    const size_t states = (size_t)k.items * c->heads * k.row_tiles * 16;
    k.states = k.parts ? round256(states * row * sizeof(float)) : 0;
    k.total = k.parts ? k.states + round256(states * sizeof(float2)) : 0;
    return k;
}

}  // namespace
}  // namespace tst

extern "C" {

int tst_kv_attention_workspace_bytes(const tst_kv_cache_t *cache, const tst_sequences_t *sequences, int q_heads, size_t *bytes)
{
    if (int rc = tst::check_cache(cache)) return rc;
    if (int rc = tst::check_sequences(cache, sequences)) return rc;
    if (!bytes || q_heads < 1 || q_heads > TST_MAX_HEADS || q_heads % cache->heads || (int64_t)sequences->tokens * q_heads > TST_MAX_ROWS) return TSTGEMM_EINVAL;
    *bytes = sequences->tokens ? tst::cut_of(cache, sequences, q_heads).total : 0;
    return TSTGEMM_OK;
}

int tst_kv_attention(const tst_heads_t *Q, int type, int q_heads, const tst_kv_cache_t *cache, const tst_sequences_t *sequences, float scale, void *Y,
                     void *workspace, size_t workspace_bytes, void *stream)
{
    size_t need = 0;
    if (int rc = tst_kv_attention_workspace_bytes(cache, sequences, q_heads, &need)) return rc;
    if (!tst::type_ok(type) || !tst::scale_ok(scale)) return TSTGEMM_EINVAL;
    if (sequences->sequences == 0 || sequences->tokens == 0) return TSTGEMM_OK;
    if (!tst::rows_ok(Q, type) || !Y || !tst::aligned(Y, tst::type_bytes(type))) return TSTGEMM_EINVAL;
    if (need && (!workspace || workspace_bytes < need)) return TSTGEMM_EWORKSPACE;
    if (need && !tst::aligned(workspace, 256)) return TSTGEMM_EINVAL;
    const tst::Cut cut = tst::cut_of(cache, sequences, q_heads);
    tst::KvArgs a{tst::cache_of(cache), tst::sequences_of(sequences), tst::rows_of(Q), q_heads, q_heads / cache->heads, cut.parts, scale, false, Y,
                  static_cast<tst::f32x4 *>(workspace), reinterpret_cast<float2 *>(static_cast<char *>(workspace) + cut.states), (int)cut.items};
    const int64_t per = 16 / (int64_t)tst::type_bytes(type);
    a.wide = tst::aligned(Q->data, 16) && Q->token_stride % per == 0 && Q->head_stride % per == 0 && cache->head_size % 8 == 0;
    return tst::status(tst::for_type(type, [&](auto t) {
        return tst::for_row(cache->head_size, [&](auto r) {
            constexpr int TYPE = decltype(t)::value, ROW = decltype(r)::value, MOST = ROW <= 128 ? 2 : 1;
            hipStream_t st = static_cast<hipStream_t>(stream);
            const dim3 grid((unsigned)cut.items, cache->heads);
            if (cut.row_tiles == 1) tst::k_kv_attention<TYPE, ROW, 1><<<grid, 64 * tst::kWaves, 0, st>>>(a);
            else tst::k_kv_attention<TYPE, ROW, MOST><<<grid, 64 * tst::kWaves, 0, st>>>(a);
            if (cut.parts) {
                if (hipError_t e = hipGetLastError()) return e;
                const dim3 joins((unsigned)cut.tiles, cache->heads, cut.tiles * cache->heads < tst::compute_units() ? ROW / 16 * cut.row_tiles : 1);
                if (cut.row_tiles == 1) tst::k_kv_join<TYPE, ROW, 1><<<joins, 64 * tst::kWaves, 0, st>>>(a);
                else tst::k_kv_join<TYPE, ROW, MOST><<<joins, 64 * tst::kWaves, 0, st>>>(a);
            }
            return hipGetLastError();
        });
    }));
}

}  // extern "C"
