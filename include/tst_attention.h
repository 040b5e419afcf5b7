/*
 * What a token sees of the tokens before it, for one MI355X (gfx950): a paged cache of keys and values in 8 bits, and attention over it
 * and over whole prompts.
 *
 *   tst_kv_append      new keys and values into the cache, with the rotation by their positions on the way
 *   tst_kv_read        the values that the codes of tokens stand for
 *   tst_kv_attention   attention of new tokens over the cache
 *   tst_attention      causal attention over whole prompts, packed one behind another
 *
 * C ABI of libtstgemm.so with the rules of tst_ops.h: plain pointers and sizes, HOST or DEVICE said of each, TSTGEMM_OK or a negative
 * TSTGEMM_E* code, nothing thrown, printed or allocated, no host synchronisation: every call only enqueues kernels on `stream` and can
 * be captured into a graph.  DEVICE operands must not overlap outputs or the workspace.  Sums, softmax statistics and scales are fp32.
 * Repeated calls on the same operands give bit-identical results.
 */
#ifndef TST_ATTENTION_H
#define TST_ATTENTION_H

#include "tst_ops.h"

#ifdef __cplusplus
extern "C" {
#endif

#define TST_KV_BLOCK 16          /* tokens that share a scale */
#define TST_MAX_HEAD_SIZE 256
#define TST_MAX_HEADS 1024
#define TST_MAX_SEQUENCES (1 << 20)
#define TST_MAX_TOKENS (1 << 22) /* rows of packed operands */
#define TST_MAX_ROWS (1 << 27)   /* rows x query heads */
#define TST_MAX_SEQUENCE_HEADS (1 << 22) /* sequences x heads of keys, of tst_attention (a grid counts no more) */

/*
 * A cache of one layer: `pages` pages of page_tokens tokens.  A code q in a block of 16 tokens of a head stands for q * scale.
 *   k_codes [pages][heads][page_tokens][row]              k_scale [pages][heads][page_tokens / 16]
 *   v_codes [pages][heads][page_tokens / 16][row][16]     v_scale the same      (a block's tokens of one channel lie together)
 * with row = tst_kv_row(head_size); channels behind head_size are there and have to be 0 (clear a new cache).
 */
typedef struct tst_kv_cache {
    size_t struct_size;          /* sizeof(tst_kv_cache_t) */
    int pages;                   /* >= 1 */
    int page_tokens;             /* 16, 32, 64, 128 or 256 */
    int heads;                   /* 1 .. 1024 */
    int head_size;               /* 1 .. 256 */
    int8_t *k_codes, *v_codes;   /* DEVICE, 16-byte aligned */
    float *k_scale, *v_scale;    /* DEVICE */
} tst_kv_cache_t;

/* Entries of a row of codes: head_size padded to 64, 96, 128, 192 or 256; 0 for a size that there is not. */
int tst_kv_row(int head_size);
/* Bytes of k_codes (and of v_codes), entries of k_scale (and of v_scale).  Errors: EINVAL. */
int tst_kv_cache_bytes(int pages, int page_tokens, int heads, int head_size, size_t *codes, size_t *scales);

/*
 * The sequences of a call.  Rows offsets[i] .. offsets[i + 1] - 1 of packed operands are the LAST tokens of sequence i, which has lens[i]
 * tokens, those of the call among them; its token at position p lies in page table[i * table_stride + p / page_tokens].  The three arrays are
 * read on the device when the call runs, so that a captured call goes by what they hold then.
 * Rows in front of offsets[0] and behind offsets[sequences] are left as they are.  Rows whose position is negative (more rows than
 * lens[i]) or whose page is not one of the cache's are not appended, and what is read in their place is NaN; nothing is read or written outside
 * the operands whatever the arrays hold.  lens[i] <= 0: an empty sequence; a length may be any other number, and positions behind the table's end have no page.
 */
typedef struct tst_sequences {
    size_t struct_size;          /* sizeof(tst_sequences_t) */
    int sequences;               /* 0 .. 2^20 */
    int tokens;                  /* rows of packed operands, 0 .. 2^22 */
    const int32_t *offsets;      /* DEVICE, sequences + 1, ascending; or NULL: a row for each sequence (tokens == sequences) */
    const int32_t *lens;         /* DEVICE, sequences */
    const int32_t *table;        /* DEVICE */
    int columns;                 /* of the table, >= 1; columns * page_tokens <= 2^30 */
    int64_t table_stride;        /* entries from row to row, >= columns */
} tst_sequences_t;

/* Packed rows of heads: entry [t][h][d] at data + t * token_stride + h * head_stride + d. */
typedef struct tst_heads {
    const void *data;            /* DEVICE, aligned to its type */
    int64_t token_stride, head_stride;   /* entries, >= 0 */
} tst_heads_t;

/*
 * The rotation by positions: for pair i of `pairs`, with c = cos[p][i], s = sin[p][i] of position p,
 *   y[a] = fl(fl(x[a] c) - fl(x[b] s)),   y[b] = fl(fl(x[b] c) + fl(x[a] s))       each in fp32
 * with (a, b) = (i, i + pairs), or (2 i, 2 i + 1) if `interleaved`; channels from 2 pairs on are left as they are.
 */
typedef struct tst_rotation {
    size_t struct_size;          /* sizeof(tst_rotation_t) */
    const float *cos, *sin;      /* DEVICE, positions x pairs, dense; a position that there is not has NaN */
    int positions, pairs;        /* pairs >= 1, 2 pairs <= head_size */
    int interleaved;
} tst_rotation_t;

/*
 * Append: keys K (rotated, if `rotation` is not NULL) and values V of the call's rows go into the cache.  For each block of 16 tokens and head that
 * rows of the call fall into, with a = the largest magnitude of the block's new entries:
 *   s = max(fl(a / 127), old scale if tokens of the block were there before the call),   r = min(fl(1 / s), FLT_MAX)
 *   q = clamp(rint(fl(x r)), -127, 127) for new entries;  rint(fl(q fl(old scale / s))) for codes that were there, where s is larger than the old scale
 * (ties to even).  A block of zeros has scale 0; one that has taken in an infinity or a NaN has scale NaN until it is begun anew.  Appending the
 * same rows again changes nothing.  Codes of a block behind its last token are not defined.
 * A call must not append to a block twice, by two sequences or by one whose table has a page twice; where the tables say so all the same, what is there then is not defined.
 * Q (heads of q_heads) and K come back rotated, rounded to `type`, in q_out [tokens][q_heads][head_size] and k_out [tokens][heads][head_size] where those
 * are not NULL.  q_out needs Q.  Channels that are rotated are NaN in rows whose position is negative or behind what the rotation has.
 * Errors: EINVAL, EHIP.
 */
int tst_kv_append(const tst_kv_cache_t *cache, const tst_sequences_t *sequences, int type, const tst_heads_t *K, const tst_heads_t *V,
                  const tst_heads_t *Q, int q_heads, const tst_rotation_t *rotation, void *q_out, void *k_out, void *stream);

/*
 * What the codes of the call's rows stand for, fl(q * scale), rounded to `type`: k_out, v_out [tokens][heads][head_size], DEVICE.
 * Errors: EINVAL, EHIP.
 */
int tst_kv_read(const tst_kv_cache_t *cache, const tst_sequences_t *sequences, int type, void *k_out, void *v_out, void *stream);

/*
 * Attention over the cache: the row of Q at position p of its sequence, head h, sees the keys of head h / (q_heads / heads) at positions 0 .. p:
 *   Y = sum_j w_j v_j / sum_j w_j,   w_j = e^(scale q.k_j - max)
 * with the values that codes stand for; |scale| <= 2^127.  The new tokens have been appended before.  A row that sees nothing is zeros.
 * q_heads: a multiple of the cache's heads, at most 1024 of them, tokens * q_heads <= 2^27; Y: DEVICE, [tokens][q_heads][head_size] of `type`.  Queries keep 22 bits or those of their type
 * relative to the largest of their row.  Products of a weight and its value's scale keep 11 bits in 16-bit types and 22 in fp32, down to 2^-21 (2^-18) of the largest of them that the row
 * sees; those below are off by up to 2^-32 (2^-40) of it.  Logits are fp32: one beyond that is an infinity; weights are too: below 2^-126 of
 * the row's largest they are 0.
 * A row of Q that holds an infinity or a NaN is NaN, and so is a row that sees a block whose scale is none.
 * workspace: DEVICE, 256-byte aligned, at least tst_kv_attention_workspace_bytes() of the same cache, sequences and q_heads on the same device (0 may be enough).  It goes by tokens, sequences,
 * heads, q_heads, head_size and the table's width in tokens, columns * page_tokens, not by what the arrays hold: ask again when one of these changes, a wider table among them.
 * Calls that may overlap need different workspaces.  Errors: EINVAL, EWORKSPACE, EHIP.
 */
int tst_kv_attention_workspace_bytes(const tst_kv_cache_t *cache, const tst_sequences_t *sequences, int q_heads, size_t *bytes);
int tst_kv_attention(const tst_heads_t *Q, int type, int q_heads, const tst_kv_cache_t *cache, const tst_sequences_t *sequences, float scale, void *Y,
                     void *workspace, size_t workspace_bytes, void *stream);

/*
 * Causal attention over whole prompts: rows offsets[i] .. offsets[i + 1] - 1 are sequence i; its row p, head h, sees keys of rows 0 .. p of the sequence,
 * head h / (q_heads / heads), as above.  offsets: DEVICE, sequences + 1, ascending.  Y: DEVICE, [tokens][q_heads][head_size] of `type`.  Rows outside the sequences
 * are left as they are.  Weights are rounded to 8 bits for bf16, 11 for fp16 (down to 2^-21 of the row's largest, and 2^-32 of it below) and 24 for fp32 in the second product, sums are fp32.
 * Logits are fp32 too, one beyond that is an infinity, and weights: below 2^-126 of the row's largest they are 0.  A mean of finite values is finite, however large they are; rows whose sums pass 2^128 on the way, or are not finite, take their
 * tile twice as long, and lose bits of values below 2^-94.
 * What a row does not see does not touch it, infinities and NaN among it.  A row of Q that holds one is NaN or infinite, and so is a row that sees one in a key (but for keys
 * whose logit is -infinity, which weigh nothing in 16 bits; in fp32, held in three planes, any infinity makes a NaN) and a channel of a row that sees one in that channel of a value.
 * tokens * q_heads <= 2^27, sequences * heads <= 2^22, |scale| <= 2^127.  Errors: EINVAL, EHIP.
 */
int tst_attention(const tst_heads_t *Q, const tst_heads_t *K, const tst_heads_t *V, int type, int q_heads, int heads, int head_size, const int32_t *offsets,
                  int sequences, int tokens, float scale, void *Y, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* TST_ATTENTION_H */
