// Shared by the operators of tst_attention.h.
#pragma once
#include <climits>

#include "ops_internal.h"
#include "tst_attention.h"

namespace tst {

constexpr int kKvBlock = TST_KV_BLOCK;
constexpr int kMaxPositions = 1 << 30;   // of a table; a length may be any int, and positions go by it as it is

inline __host__ __device__ int kv_row(int size) { return size <= 64 ? 64 : size <= 96 ? 96 : size <= 128 ? 128 : size <= 192 ? 192 : 256; }

// call(std::integral_constant<int, row>) for a run-time head size
template <typename F> inline hipError_t for_row(int size, F call)
{
    switch (kv_row(size)) {
    case 64: return call(std::integral_constant<int, 64>{});
    case 96: return call(std::integral_constant<int, 96>{});
    case 128: return call(std::integral_constant<int, 128>{});
    case 192: return call(std::integral_constant<int, 192>{});
    default: return call(std::integral_constant<int, 256>{});
    }
}

// The cache and the sequences as kernels take them.
struct Cache {
    int8_t *k, *v;
    float *k_scale, *v_scale;
    int pages, page_shift, heads, size;   // page_shift: log2 of page_tokens
    __device__ int blocks() const { return 1 << (page_shift - 4); }   // of a page
};
struct Sequences {
    int count, tokens, columns;
    const int32_t *offsets, *lens, *table;
    int64_t stride;
};
struct Rows {
    const void *data;
    int64_t token, head;
};

int check_cache(const tst_kv_cache_t *c);                              // TSTGEMM_OK or EINVAL (kv_cache.hip)
int check_sequences(const tst_kv_cache_t *c, const tst_sequences_t *s);
bool rows_ok(const tst_heads_t *x, int type);
inline bool scale_ok(float scale) { return scale <= 0x1p127f && scale >= -0x1p127f; }   // times log2 e it is finite
inline Cache cache_of(const tst_kv_cache_t *c)
{
    return Cache{c->k_codes, c->v_codes, c->k_scale, c->v_scale, c->pages, __builtin_ctz((unsigned)c->page_tokens), c->heads, c->head_size};
}
inline Sequences sequences_of(const tst_sequences_t *s)
{
    return Sequences{s->sequences, s->tokens, s->columns, s->offsets, s->lens, s->table, s->table_stride};
}
inline Rows rows_of(const tst_heads_t *x) { return x ? Rows{x->data, x->token_stride, x->head_stride} : Rows{nullptr, 0, 0}; }

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// Rows first .. first + n - 1 of packed operands: whatever the arrays hold, rows that are there.
struct Span {
    int first, n;
};
__device__ __forceinline__ Span span_of(const int32_t *offsets, int tokens, int i)
{
    if (offsets == nullptr) return Span{i, 1};
    const int a = min(max(offsets[i], 0), tokens), b = min(max(offsets[i + 1], 0), tokens);
    return Span{a, max(b - a, 0)};
}

// Pieces of `per` rows are dealt to workgroups without the host knowing the sequences' lengths: sequence i has the numbers from
// offsets[i] / per + extra i on, as many as it can have pieces (extra 1: pieces from its own first row on; 2: from borders of positions).  The
// sequence that number `at` belongs to; a wavefront looks at 64 places at a time.
__device__ __forceinline__ int find_sequence(const int32_t *offsets, int tokens, int count, int per, int extra, int at)
{
    const int lane = threadIdx.x % 64;
    int lo = 0, n = count;
    while (n > 1) {
        const int step = (n + 63) / 64, i = lo + lane * step;
        const bool before = lane * step < n && min(max(offsets[min(i, count)], 0), tokens) / per + extra * i <= at;
        const int c = max(__popcll(__ballot(before)), 1) - 1;
        lo += c * step;
        n = min(step, n - c * step);
    }
    return lo;
}
inline int pieces(int tokens, int sequences, int per, int extra) { return tokens / per + extra * sequences; }

// Where a block of 16 positions lies: page * heads * blocks of a page ..., or -1 for a page that is none of the cache's.
__device__ __forceinline__ int page_of(const Cache &c, const Sequences &s, int seq, int block)
{
    const int column = block >> (c.page_shift - 4);
    if (block < 0 || column >= s.columns) return -1;
    const int page = s.table[seq * s.stride + column];
    return page >= 0 && page < c.pages ? page : -1;
}
__device__ __forceinline__ int64_t block_at(const Cache &c, int page, int head, int block)   // in blocks
{
    return ((int64_t)page * c.heads + head) * c.blocks() + (block & (c.blocks() - 1));
}

}  // namespace tst
