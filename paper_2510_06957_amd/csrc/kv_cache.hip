// A paged cache of keys and values in 8 bits: appending to it with the rotation by positions (tst_kv_append) and reading it back (tst_kv_read).
//
// A block of 16 tokens of a head is a wavefront's, keys and values apart: it finds the largest entry of the block's new tokens, and with it the
// block's scale, before anything is rounded, and nobody else writes there.  Of values, lane (u, j) has channels 8 u .. 8 u + 7 of tokens 4 j .. 4 j + 3, so that the
// four codes of a channel make a dword of the layout [channel][token]; of keys and queries whose halves are rotated into one another it has 8 channels of either half.
//
// Memory bounds long calls: 6912 tokens of 32 query and 8 key heads of 128, bf16, are 155 MB in 29.9 us (5.2 TB/s) appended and 42 MB in 11 us (3.9 TB/s) read back, which have just been
// written.  Short ones are latency: a token 3.8 us (lens, table, rows, scale one after another), 64 tokens 4.8.  Each wavefront therefore has all its rows on their way at once.
#include "attention_internal.h"

namespace tst {
namespace {

constexpr int kWaves = 4;
constexpr float kNan = __builtin_nanf("");

struct AppendArgs {
    Cache cache;
    Sequences seqs;
    Rows k, v, q;
    int q_heads, kv_groups;   // workgroups of a block's heads that have keys and values; those behind have queries
    const float *cos, *sin;
    int positions, pairs;
    bool interleaved;
    void *q_out, *k_out;
};

// Channels d .. d + 7 of a row of `size` entries, 0 behind its end.
template <int TYPE, bool WIDE> __device__ __forceinline__ void load8(const typename Entry<TYPE>::bits *row, int d, int size, float (&x)[8])
{
    typedef typename Entry<TYPE>::bits Bits;
    if constexpr (WIDE) {
        union {
            u32x4 v[sizeof(Bits) / 2];
            Bits e[8];
        } u;
#pragma unroll
        for (int i = 0; i < (int)sizeof(Bits) / 2; ++i) u.v[i] = reinterpret_cast<const u32x4 *>(row + d)[i];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = Entry<TYPE>::get(u.e[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = d + i < size ? Entry<TYPE>::get(row[d + i]) : 0.f;
    }
}
template <int TYPE, bool WIDE> __device__ __forceinline__ void store8(typename Entry<TYPE>::bits *row, int d, int size, const float (&x)[8])
{
    typedef typename Entry<TYPE>::bits Bits;
    if constexpr (WIDE) {
        union {
            u32x4 v[sizeof(Bits) / 2];
            Bits e[8];
        } u;
#pragma unroll
        for (int i = 0; i < 8; ++i) u.e[i] = Entry<TYPE>::put(x[i]);
#pragma unroll
        for (int i = 0; i < (int)sizeof(Bits) / 2; ++i) reinterpret_cast<u32x4 *>(row + d)[i] = u.v[i];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (d + i < size) row[d + i] = Entry<TYPE>::put(x[i]);
    }
}

// How rows are read: an entry at a time; 8 at a time, on borders; so, and rotated in halves that fill the head.
enum Reading { kNarrow, kWide, kHalves };

// Which 8 channels (kHalves: twice 8) of which tokens of a block a lane has.
template <int HOW, int SIZES> struct Lanes {   // SIZES 1: heads of up to 128 entries, 2: 256
    static constexpr int kUnits = HOW == kHalves ? 2 : 1, kAcross = (HOW == kHalves ? 8 : 16) * SIZES, kStep = 64 / kAcross, kPasses = kKvBlock / kStep;
};

// Channels d .. d + 7 of a row, rotated by position p: each product and each sum is rounded to fp32 (no fma), so that codes are defined bit for bit.
template <int TYPE, int HOW> __device__ __forceinline__ void rotated8(const AppendArgs &a, const typename Entry<TYPE>::bits *row, int d, int p, float (&x)[8])
{
#pragma clang fp contract(off)
    load8<TYPE, HOW != kNarrow>(row, d, a.cache.size, x);
    const int P = a.pairs;
    if (d >= 2 * P) return;
    const bool there = p >= 0 && p < a.positions;
    const float *cs = a.cos + (int64_t)(there ? p : 0) * P, *sn = a.sin + (int64_t)(there ? p : 0) * P;
    if constexpr (HOW != kNarrow) {   // pairs are a multiple of 8 (of 4 if they are neighbours)
        if (a.interleaved) {
            const f32x4 c = *reinterpret_cast<const f32x4 *>(cs + d / 2), s = *reinterpret_cast<const f32x4 *>(sn + d / 2);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float x0 = x[2 * i], x1 = x[2 * i + 1];
                const float ci = there ? c[i] : kNan, si = there ? s[i] : kNan;
                const float a0 = x0 * ci, b0 = x1 * si, a1 = x1 * ci, b1 = x0 * si;
                x[2 * i] = a0 - b0;
                x[2 * i + 1] = a1 + b1;
            }
        } else {
            const int at = d < P ? d : d - P;
            float other[8];
            load8<TYPE, true>(row, d < P ? d + P : d - P, a.cache.size, other);
            f32x4 c[2], s[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) c[i] = reinterpret_cast<const f32x4 *>(cs + at)[i], s[i] = reinterpret_cast<const f32x4 *>(sn + at)[i];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float ci = there ? c[i / 4][i % 4] : kNan, si = there ? s[i / 4][i % 4] : kNan;
                const float m = x[i] * ci, n = other[i] * si;
                x[i] = d < P ? m - n : m + n;
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int e = d + i;
            if (e >= 2 * P) break;
            const bool low = a.interleaved ? e % 2 == 0 : e < P;
            const int at = a.interleaved ? e / 2 : (low ? e : e - P), mate = a.interleaved ? e ^ 1 : (low ? e + P : e - P);
            const float c = there ? cs[at] : kNan, s = there ? sn[at] : kNan;
            const float m = x[i] * c, n = Entry<TYPE>::get(row[mate]) * s;
            x[i] = low ? m - n : m + n;
        }
    }
}

// The same for halves: cos and sin of 8 pairs of a position, and both halves' channels by them.
struct Angles {
    f32x4 c[2], s[2];
};
__device__ __forceinline__ Angles angles_of(const AppendArgs &a, int pair, int p)
{
    const bool there = p >= 0 && p < a.positions;
    const int64_t at = (int64_t)(there ? p : 0) * a.pairs + pair;
    Angles g;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        g.c[i] = reinterpret_cast<const f32x4 *>(a.cos + at)[i], g.s[i] = reinterpret_cast<const f32x4 *>(a.sin + at)[i];
#pragma unroll
        for (int e = 0; e < 4; ++e) g.c[i][e] = there ? g.c[i][e] : kNan, g.s[i][e] = there ? g.s[i][e] : kNan;
    }
    return g;
}
__device__ __forceinline__ void rotate(const Angles &g, float (&x)[8], float (&y)[8])
{
#pragma clang fp contract(off)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float c = g.c[i / 4][i % 4], s = g.s[i / 4][i % 4];
        const float a = x[i] * c, b = y[i] * s, d = y[i] * c, e = x[i] * s;
        x[i] = a - b;
        y[i] = d + e;
    }
}

__device__ __forceinline__ int code_of(float y, float inverse)
{
    const float q = __builtin_rintf(y * inverse);
    return (int)fminf(fmaxf(q, -127.f), 127.f);
}
__device__ __forceinline__ unsigned rescaled(unsigned four, float share)
{
    unsigned out = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) out |= ((unsigned)(int)__builtin_rintf((float)(int8_t)(four >> 8 * i) * share) & 255u) << 8 * i;
    return out;
}

// A block's scale with what comes to it.
struct Scale {
    float scale, inverse, share;   // share: what the codes that are there are multiplied with
    bool finite, grown;
};
__device__ __forceinline__ Scale scale_of(unsigned most, float before, bool some)
{
    const float largest = __uint_as_float(wave_max(most));
    Scale s;
    s.finite = largest <= 3.402823466e38f && before == before;
    s.scale = s.finite ? fmaxf(before, largest / 127.f) : kNan;
    s.inverse = s.finite ? fminf(1.f / s.scale, 3.402823466e38f) : 0.f;   // scale 0: 0 * FLT_MAX = 0
    s.grown = s.finite && s.scale > before && some;
    s.share = s.grown ? before / s.scale : 1.f;
    return s;
}
__device__ __forceinline__ unsigned four_codes(const float *x, const Scale &s)
{
    unsigned q = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) q |= (s.finite ? (unsigned)code_of(x[e], s.inverse) & 255u : 0u) << 8 * e;
    return q;
}
__device__ __forceinline__ void widest(unsigned &most, const float (&x)[8])
{
#pragma unroll
    for (int e = 0; e < 8; ++e) most = max(most, __float_as_uint(x[e]) & 0x7fffffffu);
}

// What a wavefront appends: tokens from .. to of a block, rows row0 .. of the call.
struct Piece {
    int head, seq, block, from, to, row0;
};

template <int TYPE, int HOW, int SIZES> __device__ __forceinline__ void append_keys(const AppendArgs &a, const Piece &p)
{
    typedef typename Entry<TYPE>::bits Bits;
    typedef Lanes<HOW, SIZES> L;
    const int lane = threadIdx.x % 64, size = a.cache.size, row = kv_row(size), count = (size + 7) / 8 / L::kUnits, k = min(lane % L::kAcross, count - 1);
    const int page = page_of(a.cache, a.seqs, p.seq, p.block);
    const int64_t at = block_at(a.cache, max(page, 0), p.head, p.block);
    const Bits *data = static_cast<const Bits *>(a.k.data) + p.head * a.k.head;
    float x[L::kPasses][L::kUnits][8];
    unsigned most = 0;
#pragma unroll
    for (int i = 0; i < L::kPasses; ++i) {      // rows of the call in place of others
        const int token = min(max(lane / L::kAcross + i * L::kStep, p.from), p.to);
        const Bits *r = data + (int64_t)(p.row0 + token - p.from) * a.k.token;
        if constexpr (HOW == kHalves) {
            load8<TYPE, true>(r, 8 * k, size, x[i][0]);
            load8<TYPE, true>(r, a.pairs + 8 * k, size, x[i][1]);
            rotate(angles_of(a, 8 * k, p.block * kKvBlock + token), x[i][0], x[i][1]);
        } else rotated8<TYPE, HOW>(a, r, 8 * k, p.block * kKvBlock + token, x[i][0]);
#pragma unroll
        for (int u = 0; u < L::kUnits; ++u) widest(most, x[i][u]);
    }
    float *scales = a.cache.k_scale + at;
    const float before = p.from > 0 ? *scales : 0.f;
    const Scale s = scale_of(most, before, p.from > 0);
    if (lane == 0 && page >= 0) *scales = s.scale;
    if (lane % L::kAcross >= count) return;
#pragma unroll
    for (int i = 0; i < L::kPasses; ++i) {
        const int token = lane / L::kAcross + i * L::kStep;
        const bool mine = token >= p.from && token <= p.to;
        if (token > p.to || (!mine && !s.grown)) continue;
#pragma unroll
        for (int u = 0; u < L::kUnits; ++u) {
            const int d = 8 * k + u * a.pairs;
            if (mine && a.k_out) store8<TYPE, HOW != kNarrow>(static_cast<Bits *>(a.k_out) + ((int64_t)(p.row0 + token - p.from) * a.cache.heads + p.head) * size, d, size, x[i][u]);
            if (page < 0) continue;
            u32x2 *codes = reinterpret_cast<u32x2 *>(a.cache.k + (at * kKvBlock + token) * row + d);
            *codes = mine ? u32x2{four_codes(x[i][u], s), four_codes(x[i][u] + 4, s)} : u32x2{rescaled((*codes)[0], s.share), rescaled((*codes)[1], s.share)};
        }
    }
}

template <int TYPE, int HOW, int SIZES> __device__ __forceinline__ void append_values(const AppendArgs &a, const Piece &p, unsigned *lds)
{
    typedef typename Entry<TYPE>::bits Bits;
    const int lane = threadIdx.x % 64, j = lane % 4, size = a.cache.size, row = kv_row(size), units = (size + 7) / 8;
    const int page = page_of(a.cache, a.seqs, p.seq, p.block);
    if (page < 0) return;
    const int64_t at = block_at(a.cache, page, p.head, p.block);
    u32x4 *codes = reinterpret_cast<u32x4 *>(a.cache.v + at * kKvBlock * row);
    const Bits *data = static_cast<const Bits *>(a.v.data) + p.head * a.v.head;
    float x[SIZES][4][8];
    unsigned most = 0;
#pragma unroll
    for (int i = 0; i < SIZES; ++i)
#pragma unroll
        for (int t = 0; t < 4; ++t) {           // rows of the call in place of others
            const int token = min(max(4 * j + t, p.from), p.to);
            load8<TYPE, HOW != kNarrow>(data + (int64_t)(p.row0 + token - p.from) * a.v.token, 8 * min(lane / 4 + 16 * i, units - 1), size, x[i][t]);
            widest(most, x[i][t]);
        }
    float *scales = a.cache.v_scale + at;
    const float before = p.from > 0 ? *scales : 0.f;
    u32x4 old[2 * SIZES];
    if (p.from > 0) {
#pragma unroll
        for (int i = 0; i < 2 * SIZES; ++i) old[i] = codes[min(lane + 64 * i, size - 1)];
    }
    const Scale s = scale_of(most, before, p.from > 0);
    if (lane == 0) *scales = s.scale;
    // dwords of four tokens, rows of a channel through the LDS, joined with the tokens that were there; zeros behind the last
#pragma unroll
    for (int i = 0; i < SIZES; ++i) {
        const int u = lane / 4 + 16 * i;
        if (u >= units) continue;
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            unsigned q[4];
#pragma unroll
            for (int t = 0; t < 4; ++t) q[t] = 4 * j + t <= p.to ? four_codes(x[i][t] + 4 * w, s) : 0u;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                unsigned four = 0;
#pragma unroll
                for (int t = 0; t < 4; ++t) four |= (q[t] >> 8 * e & 255u) << 8 * t;
                lds[(8 * u + 4 * w + e) * 4 + j] = four;
            }
        }
    }
    order_wave();
#pragma unroll
    for (int i = 0; i < 2 * SIZES; ++i) {
        const int d = lane + 64 * i;
        if (d >= size) continue;
        u32x4 four = reinterpret_cast<const u32x4 *>(lds)[d];
        if (p.from > 0) {
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const unsigned kept = s.grown ? rescaled(old[i][w], s.share) : old[i][w];
                unsigned mask = 0;   // bytes of tokens before `from`
#pragma unroll
                for (int t = 0; t < 4; ++t) mask |= 4 * w + t < p.from ? 255u << 8 * t : 0u;
                four[w] = (kept & mask) | (four[w] & ~mask);
            }
        }
        codes[d] = four;
    }
}

// Four query heads from h0 on.
template <int TYPE, int HOW, int SIZES> __device__ __forceinline__ void rotate_queries(const AppendArgs &a, const Piece &p, int h0)
{
    typedef typename Entry<TYPE>::bits Bits;
    typedef Lanes<HOW, SIZES> L;
    const int lane = threadIdx.x % 64, size = a.cache.size, count = (size + 7) / 8 / L::kUnits, k = lane % L::kAcross, heads = min(a.q_heads - h0, 4);
    if (heads <= 0 || k >= count) return;
    for (int t = lane / L::kAcross; t <= p.to - p.from; t += L::kStep) {
        const int r = p.row0 + t, position = p.block * kKvBlock + p.from + t;
        const Bits *in = static_cast<const Bits *>(a.q.data) + (int64_t)r * a.q.token;
        Bits *out = static_cast<Bits *>(a.q_out) + (int64_t)r * a.q_heads * size;
        float x[4][L::kUnits][8];
        if constexpr (HOW == kHalves) {
            const Angles g = angles_of(a, 8 * k, position);
#pragma unroll
            for (int h = 0; h < 4; ++h) {
                const Bits *row = in + min(h0 + h, a.q_heads - 1) * a.q.head;
                load8<TYPE, true>(row, 8 * k, size, x[h][0]);
                load8<TYPE, true>(row, a.pairs + 8 * k, size, x[h][1]);
            }
#pragma unroll
            for (int h = 0; h < 4; ++h) rotate(g, x[h][0], x[h][1]);
        } else {
#pragma unroll
            for (int h = 0; h < 4; ++h) rotated8<TYPE, HOW>(a, in + min(h0 + h, a.q_heads - 1) * a.q.head, 8 * k, position, x[h][0]);
        }
#pragma unroll
        for (int h = 0; h < 4; ++h)
#pragma unroll
            for (int u = 0; u < L::kUnits; ++u)
                if (h < heads) store8<TYPE, HOW != kNarrow>(out + (int64_t)(h0 + h) * size, 8 * k + u * a.pairs, size, x[h][u]);
    }
}

template <int TYPE, int HOW, int SIZES> __global__ void __launch_bounds__(64 * kWaves) k_kv_append(AppendArgs a)
{
    __shared__ __attribute__((aligned(16))) unsigned lds[kWaves][128 * SIZES * kKvBlock / 4];
    const int wave = uniform(threadIdx.x / 64);
    const int at = blockIdx.x;
    const int seq = a.seqs.offsets ? uniform(find_sequence(a.seqs.offsets, a.seqs.tokens, a.seqs.count, kKvBlock, 2, at)) : at;
    const Span rows = span_of(a.seqs.offsets, a.seqs.tokens, seq);
    const int piece = a.seqs.offsets ? at - (rows.first / kKvBlock + 2 * seq) : 0;
    const int len = max(a.seqs.lens[seq], 0), first = len - rows.n;   // position of the first row; negative where there are more rows
    const int block = (first >> 4) + piece;
    if (rows.n == 0 || piece < 0 || block > (len - 1) >> 4) return;
    const int from = max(first - block * kKvBlock, 0), to = min(len - 1 - block * kKvBlock, kKvBlock - 1);
    Piece p{0, seq, block, from, to, rows.first + (block * kKvBlock + from - first)};
    if ((int)blockIdx.y >= a.kv_groups) {
        rotate_queries<TYPE, HOW, SIZES>(a, p, ((blockIdx.y - a.kv_groups) * kWaves + wave) * 4);
        return;
    }
    const int item = blockIdx.y * kWaves + wave;
    p.head = item >> 1;
    if (p.head >= a.cache.heads) return;
    if (item & 1) append_values<TYPE, HOW, SIZES>(a, p, lds[wave]);
    else append_keys<TYPE, HOW, SIZES>(a, p);
}

// What a code stands for, rounded to fp32 (the compiler would otherwise round the product to fp16 at once).
__device__ __forceinline__ float value_of(unsigned four, int i, float scale)
{
    float v = (float)(int8_t)(four >> 8 * i) * scale;
    asm("" : "+v"(v));
    return v;
}

struct ReadArgs {
    Cache cache;
    Sequences seqs;
    void *k_out, *v_out;
};

template <int TYPE, bool WIDE> __global__ void __launch_bounds__(64 * kWaves) k_kv_read(ReadArgs a)
{
    typedef typename Entry<TYPE>::bits Bits;
    const int wave = uniform(threadIdx.x / 64), lane = threadIdx.x % 64;
    const int at = blockIdx.x;
    const int seq = a.seqs.offsets ? uniform(find_sequence(a.seqs.offsets, a.seqs.tokens, a.seqs.count, kKvBlock, 2, at)) : at;
    const Span rows = span_of(a.seqs.offsets, a.seqs.tokens, seq);
    const int piece = a.seqs.offsets ? at - (rows.first / kKvBlock + 2 * seq) : 0;
    const int len = max(a.seqs.lens[seq], 0), first = len - rows.n;
    const int block = (first >> 4) + piece;
    const int item = blockIdx.y * kWaves + wave;
    if (rows.n == 0 || piece < 0 || block > (len - 1) >> 4 || item >= 2 * a.cache.heads) return;
    const int from = max(first - block * kKvBlock, 0), to = min(len - 1 - block * kKvBlock, kKvBlock - 1);
    const int row0 = rows.first + (block * kKvBlock + from - first);
    const bool values = item & 1;
    const int head = item >> 1, size = a.cache.size, units = (size + 7) / 8, row = kv_row(size);
    const int page = page_of(a.cache, a.seqs, seq, block);
    const int64_t place = page < 0 ? 0 : block_at(a.cache, page, head, block);
    const float scale = page < 0 ? kNan : (values ? a.cache.v_scale : a.cache.k_scale)[place];
    const int8_t *codes = (values ? a.cache.v : a.cache.k) + place * kKvBlock * row;
    Bits *out = static_cast<Bits *>(values ? a.v_out : a.k_out) + ((int64_t)row0 * a.cache.heads + head) * size;
    const int64_t next = (int64_t)a.cache.heads * size;   // entries from token to token
    if (!values) {
        const int across = units <= 8 ? 8 : units <= 16 ? 16 : 32, u = lane & (across - 1), step = 64 / across;
        if (u >= units) return;
        for (int t0 = from + lane / across; t0 <= to; t0 += 4 * step) {      // four rows at a time
            u32x2 eight[4];
#pragma unroll
            for (int b = 0; b < 4; ++b) eight[b] = *reinterpret_cast<const u32x2 *>(codes + min(t0 + b * step, to) * row + 8 * u);
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                if (t0 + b * step > to) continue;
                float x[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = value_of(eight[b][e / 4], e % 4, scale);
                store8<TYPE, WIDE>(out + (t0 + b * step - from) * next, 8 * u, size, x);
            }
        }
        return;
    }
    // two neighbouring channels a lane, and both of a token at once where that is on a border
    for (int d = 2 * lane; d < size; d += 128) {
        const u32x4 *at = reinterpret_cast<const u32x4 *>(codes) + d;
        const u32x4 two[2] = {at[0], at[1]};     // (rows of codes are longer than an odd size)
#pragma unroll
        for (int t = 0; t < kKvBlock; ++t) {
            if (t < from || t > to) continue;
            Bits pair[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) pair[i] = Entry<TYPE>::put(value_of(two[i][t / 4], t % 4, scale));
            Bits *to2 = out + (t - from) * next + d;
            if constexpr (WIDE) __builtin_memcpy(__builtin_assume_aligned(to2, sizeof(pair)), pair, sizeof(pair));
            else {
                to2[0] = pair[0];
                if (d + 1 < size) to2[1] = pair[1];
            }
        }
    }
}

bool wide(const Rows &x, int type)
{
    const int64_t per = 16 / (int64_t)type_bytes(type);
    return aligned(x.data, 16) && x.token % per == 0 && x.head % per == 0;
}

}  // namespace

int check_cache(const tst_kv_cache_t *c)
{
    size_t codes = 0, scales = 0;
    if (!c || c->struct_size != sizeof(tst_kv_cache_t) || tst_kv_cache_bytes(c->pages, c->page_tokens, c->heads, c->head_size, &codes, &scales) != TSTGEMM_OK)
        return TSTGEMM_EINVAL;
    return c->k_codes && c->v_codes && c->k_scale && c->v_scale && aligned(c->k_codes, 16) && aligned(c->v_codes, 16) && aligned(c->k_scale, 4) && aligned(c->v_scale, 4)
               ? TSTGEMM_OK : TSTGEMM_EINVAL;
}

int check_sequences(const tst_kv_cache_t *c, const tst_sequences_t *s)
{
    if (!s || s->struct_size != sizeof(tst_sequences_t) || s->sequences < 0 || s->sequences > TST_MAX_SEQUENCES || s->tokens < 0 || s->tokens > TST_MAX_TOKENS)
        return TSTGEMM_EINVAL;
    if (!s->offsets && s->tokens != s->sequences) return TSTGEMM_EINVAL;
    if (s->columns < 1 || s->table_stride < s->columns || s->table_stride > INT64_MAX / 4 / (TST_MAX_SEQUENCES + 1) || (int64_t)s->columns * c->page_tokens > kMaxPositions)
        return TSTGEMM_EINVAL;
    if (s->sequences == 0 || s->tokens == 0) return TSTGEMM_OK;
    return s->lens && s->table && aligned(s->offsets, 4) && aligned(s->lens, 4) && aligned(s->table, 4) ? TSTGEMM_OK : TSTGEMM_EINVAL;
}

// Strides up to 2^38 keep every offset of a row and head below 2^63.
bool rows_ok(const tst_heads_t *x, int type)
{
    constexpr int64_t most = (int64_t)1 << 38;
    return x && x->data && aligned(x->data, type_bytes(type)) && x->token_stride >= 0 && x->head_stride >= 0 && x->token_stride <= most && x->head_stride <= most;
}

}  // namespace tst

extern "C" {

int tst_kv_row(int head_size) { return head_size < 1 || head_size > TST_MAX_HEAD_SIZE ? 0 : tst::kv_row(head_size); }

int tst_kv_cache_bytes(int pages, int page_tokens, int heads, int head_size, size_t *codes, size_t *scales)
{
    const int row = tst_kv_row(head_size);
    if (!codes || !scales || pages < 1 || page_tokens < 16 || page_tokens > 256 || (page_tokens & (page_tokens - 1)) || heads < 1 || heads > TST_MAX_HEADS || !row)
        return TSTGEMM_EINVAL;
    *scales = (size_t)pages * heads * (page_tokens / tst::kKvBlock);
    *codes = *scales * tst::kKvBlock * row;
    return TSTGEMM_OK;
}

int tst_kv_append(const tst_kv_cache_t *cache, const tst_sequences_t *sequences, int type, const tst_heads_t *K, const tst_heads_t *V,
                  const tst_heads_t *Q, int q_heads, const tst_rotation_t *rotation, void *q_out, void *k_out, void *stream)
{
    if (int rc = tst::check_cache(cache)) return rc;
    if (int rc = tst::check_sequences(cache, sequences)) return rc;
    if (!tst::type_ok(type) || (Q && (q_heads < 1 || q_heads > TST_MAX_HEADS)) || (!Q && q_out)) return TSTGEMM_EINVAL;
    const tst_rotation_t *r = rotation;
    if (r && (r->struct_size != sizeof(tst_rotation_t) || !r->cos || !r->sin || !tst::aligned(r->cos, 4) || !tst::aligned(r->sin, 4) || r->positions < 1 || r->pairs < 1 ||
              r->pairs > cache->head_size / 2))
        return TSTGEMM_EINVAL;
    if (sequences->sequences == 0 || sequences->tokens == 0) return TSTGEMM_OK;
    const size_t entry = tst::type_bytes(type);
    if (!tst::rows_ok(K, type) || !tst::rows_ok(V, type) || (Q && (!q_out || !tst::rows_ok(Q, type))) || !tst::aligned(q_out, entry) || !tst::aligned(k_out, entry)) return TSTGEMM_EINVAL;
    tst::AppendArgs a{tst::cache_of(cache), tst::sequences_of(sequences), tst::rows_of(K), tst::rows_of(V), tst::rows_of(Q), Q ? q_heads : 0,
                      tst::blocks_of(2 * cache->heads, tst::kWaves), r ? r->cos : nullptr, r ? r->sin : nullptr, r ? r->positions : 0, r ? r->pairs : 0,
                      r && r->interleaved, q_out, k_out};
    // vectors of 16 bytes: rows, their pairs and the angles lie on borders
    const bool wide = tst::wide(a.k, type) && tst::wide(a.v, type) && (!Q || (tst::wide(a.q, type) && tst::aligned(q_out, 16))) && tst::aligned(k_out, 16) && cache->head_size % 8 == 0 &&
                      a.pairs % (a.interleaved ? 4 : 8) == 0 && tst::aligned(a.cos, 16) && tst::aligned(a.sin, 16);
    const dim3 grid(sequences->offsets ? tst::pieces(sequences->tokens, sequences->sequences, tst::kKvBlock, 2) : sequences->sequences,
                    a.kv_groups + tst::blocks_of(a.q_heads, 4 * tst::kWaves));
    return tst::status(tst::for_type(type, [&](auto t) {
        constexpr int TYPE = decltype(t)::value;
        hipStream_t st = static_cast<hipStream_t>(stream);
        auto launch = [&](auto how) {
            if (cache->head_size <= 128) tst::k_kv_append<TYPE, decltype(how)::value, 1><<<grid, 64 * tst::kWaves, 0, st>>>(a);
            else tst::k_kv_append<TYPE, decltype(how)::value, 2><<<grid, 64 * tst::kWaves, 0, st>>>(a);
        };
        if (wide && a.pairs > 0 && !a.interleaved && 2 * a.pairs == cache->head_size) launch(std::integral_constant<int, tst::kHalves>{});
        else if (wide) launch(std::integral_constant<int, tst::kWide>{});
        else launch(std::integral_constant<int, tst::kNarrow>{});
        return hipGetLastError();
    }));
}

int tst_kv_read(const tst_kv_cache_t *cache, const tst_sequences_t *sequences, int type, void *k_out, void *v_out, void *stream)
{
    if (int rc = tst::check_cache(cache)) return rc;
    if (int rc = tst::check_sequences(cache, sequences)) return rc;
    if (!tst::type_ok(type)) return TSTGEMM_EINVAL;
    if (sequences->sequences == 0 || sequences->tokens == 0) return TSTGEMM_OK;
    const size_t entry = tst::type_bytes(type);
    if (!k_out || !v_out || !tst::aligned(k_out, entry) || !tst::aligned(v_out, entry)) return TSTGEMM_EINVAL;
    const tst::ReadArgs a{tst::cache_of(cache), tst::sequences_of(sequences), k_out, v_out};
    const bool wide = tst::aligned(k_out, 16) && tst::aligned(v_out, 16) && cache->head_size % 8 == 0;
    const dim3 grid(sequences->offsets ? tst::pieces(sequences->tokens, sequences->sequences, tst::kKvBlock, 2) : sequences->sequences,
                    tst::blocks_of(2 * cache->heads, tst::kWaves));
    return tst::status(tst::for_type(type, [&](auto t) {
        constexpr int TYPE = decltype(t)::value;
        hipStream_t st = static_cast<hipStream_t>(stream);
        if (wide) tst::k_kv_read<TYPE, true><<<grid, 64 * tst::kWaves, 0, st>>>(a);
        else tst::k_kv_read<TYPE, false><<<grid, 64 * tst::kWaves, 0, st>>>(a);
        return hipGetLastError();
    }));
}

}  // extern "C"
