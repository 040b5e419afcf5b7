/*
 * Operators around the sparse ternary product of tstgemm.h, for one AMD MI355X (gfx950): what else a model with quantised
 * weights runs for each token it answers with.
 *
 *   tst_quantize, tst_w8_gemm, tst_w8_linear   layers in 8 bits with a scale for each token and each output channel
 *   tst_moe                                    a whole mixture-of-experts feed-forward layer for a few tokens
 *   tst_logprobs                               log probabilities of given tokens, with entropy and the top alternatives
 *
 * C ABI of libtstgemm.so, with the rules of tstgemm.h: plain pointers and sizes, every pointer argument says whether it is HOST or
 * DEVICE memory, TSTGEMM_OK or a negative TSTGEMM_E* code, no function throws, aborts or prints, no mutable global state.  Every
 * call only enqueues kernels on `stream` (a hipStream_t, NULL = the null stream): no allocation, no host synchronisation, so it can
 * be captured into a graph.  DEVICE operands must not overlap outputs or the workspace.  Sizes of zero where a count of tokens or
 * rows is meant (M, T, R) are allowed and launch nothing.  Repeated calls on the same operands give bit-identical results.
 *
 * Types of activations, results and logits; all sums, softmax statistics and scales are fp32 (or int32, exact).
 */
#ifndef TST_OPS_H
#define TST_OPS_H

#include "tstgemm.h"

#ifdef __cplusplus
extern "C" {
#endif

#define TST_F32 0
#define TST_BF16 1
#define TST_F16 2

/*
 * Quantise tokens: for each row m of X, with a = max_k |X[m][k]|,
 *   scale[m] = fl32(a / 127),   Q[m][k] = rint(fl32(X[m][k] * min(fl32(127 / a), FLT_MAX)))   (ties to even; -127 .. 127).
 * A row of zeros has scale 0 and codes 0.  A row that holds an infinity or a NaN has scale NaN and codes 0, so that what is made from
 * it is NaN in that row and nowhere else.
 * X: DEVICE, M rows of K entries of `type` (TST_*), x_stride entries apart (>= K).  Q: DEVICE, M rows of K bytes, q_stride
 * bytes apart (>= K); only the K bytes of a row are written.  tst_w8_gemm() wants rows on 16-byte borders.  scale: DEVICE, M.
 * M >= 0, 1 <= K <= 2^30.  Errors: EINVAL, EHIP.
 */
int tst_quantize(const void *X, int type, int64_t x_stride, int8_t *Q, int64_t q_stride, float *scale, int M, int K, void *stream);

/*
 * Device form of 8-bit weights: 16 columns x 64 rows at a time in one piece of 1 KiB, [column block][row block][16 rows][column][row],
 * which is how both matrix instructions take them, K and N padded with zeros to multiples of 64 and 16.
 * tst_w8_bytes: bytes of one K x N matrix (a multiple of 1024).  K <= 131071, so that a sum of K products of codes, -128 included,
 * fits 32 bits.
 * tst_w8_pack: W: DEVICE, `count` matrices of K x N int8, row-major, one behind another; packed: DEVICE, count * tst_w8_bytes(),
 * 16-byte aligned, fully overwritten, below 64 GiB a matrix.  Errors: EINVAL, ETOOBIG, EHIP.
 */
int tst_w8_bytes(int K, int N, size_t *bytes);
int tst_w8_pack(const int8_t *W, int count, int K, int N, void *packed, void *stream);

/*
 * Y[m][n] = fl(sum_k Q[m][k] W[k][n]) * scale[m] * w_scale[n] + b[n]: the sum in int32, exact, rounded to fp32 once, then two products
 * and the bias in fp32, rounded to y_type once.
 * Q: DEVICE, M rows of K codes, q_stride bytes apart; Q 16-byte aligned and q_stride a multiple of 16, at most 4 MiB (or M = 1).
 * What lies between K and the next 16-byte border of a row is read and does not matter; nothing behind that border is read.
 * scale: DEVICE, M.  packed: DEVICE, tst_w8_pack() of W.  w_scale: DEVICE, N.  b: DEVICE, N, or NULL.  Y: DEVICE, M x N of y_type,
 * row-major, aligned to its type.  0 <= M <= 1048560, N < 2^27 - 15.  Errors: EINVAL, EHIP.
 */
int tst_w8_gemm(const int8_t *Q, int64_t q_stride, const float *scale, const void *packed, const float *w_scale, const float *b,
                void *Y, int y_type, int M, int K, int N, void *stream);

/*
 * tst_w8_gemm() of tst_quantize(X), bit for bit; X and Y of the same type.  workspace: DEVICE, 256-byte aligned, at least
 * tst_w8_linear_workspace_bytes() (codes and scales).  Calls that may overlap need different workspaces.
 * Errors: EINVAL, EWORKSPACE, EHIP.
 */
int tst_w8_linear_workspace_bytes(int M, int K, size_t *bytes);
int tst_w8_linear(const void *X, int type, int64_t x_stride, const void *packed, const float *w_scale, const float *b, void *Y,
                  int M, int K, int N, void *workspace, size_t workspace_bytes, void *stream);

/*
 * A mixture-of-experts feed-forward layer for a few tokens, router included.  For each token t (row of X):
 *   l[e] = sum_d X[t][d] router[e][d];  the top_k experts with the largest l, largest first (ties: lowest e; a NaN counts as largest)
 *   p    = softmax over the chosen l (normalize != 0), or the chosen entries of the softmax over all l (normalize == 0)
 *   g    = gate_scale[e][f] sum_d X[t][d] gate[e][d][f],  u the same with up,  h[f] = g / (1 + e^-g) * u
 *   Y[t][c] = sum over the chosen e of down_scale[e][c] sum_f (p h[f]) down[e][f][c]
 * Weights are 8-bit with a scale for each output channel (ternary matrices are a case of them); X, router and Y have one type.  The
 * activations keep the bits of their type in the products, h the 24 of fp32, and sums are fp32.  A token that holds an infinity or a NaN has NaN results and does not touch the others.
 */
typedef struct tst_moe {
    size_t struct_size;        /* sizeof(tst_moe_t) */
    int type;                  /* TST_* of X, router and Y */
    int experts, width, inner; /* E <= 512, D, F (both <= 131071) */
    const void *router;        /* DEVICE, E x D of `type`, row-major */
    const void *gate, *up;     /* DEVICE, tst_w8_pack() of E matrices D x F */
    const void *down;          /* DEVICE, tst_w8_pack() of E matrices F x D */
    const float *gate_scale, *up_scale, *down_scale;   /* DEVICE, E x F, E x F, E x D */
} tst_moe_t;

#define TST_MOE_MAX_EXPERTS 512
#define TST_MOE_MAX_TOP 16

/*
 * X: DEVICE, T rows of D entries, x_stride entries apart.  Y: DEVICE, T x D.  ids, p: DEVICE, T x top_k each (int32, fp32), largest
 * logit first.  T >= 0 (each expert's weights are read once for up to 64 tokens), 1 <= top_k <= min(E, 16).
 * workspace: DEVICE, 256-byte aligned, at least tst_moe_workspace_bytes().  Errors: EINVAL, EWORKSPACE, EHIP.
 */
int tst_moe_workspace_bytes(const tst_moe_t *moe, int T, int top_k, size_t *bytes);
int tst_moe(const void *X, int64_t x_stride, const tst_moe_t *moe, int top_k, int normalize, void *Y, int32_t *ids, float *p, int T,
            void *workspace, size_t workspace_bytes, void *stream);

/*
 * Log probabilities.  For each row z of logits, with m = max z and S = sum_v e^(z[v] - m):
 *   of_token[r][c] = z[tokens[r][c]] - m - log S          for each of C given tokens
 *   entropy[r]     = log S - sum_v e^(z[v]-m) (z[v]-m) / S   (a term whose e^(z[v]-m) is 0 counts 0)
 *   top_ids[r]     = the `top` largest logits' tokens, largest first (ties: the lowest token; a NaN counts as largest)
 *   of_top[r]      = their log probabilities
 * Entries of -infinity, and of the type's lowest value, are masked ones: probability 0, log probability -infinity (or as low as the
 * subtraction gives).  A row with nothing but -infinity, with +infinity or with a NaN has no distribution: its entropy and log
 * probabilities are NaN; a token outside 0 .. V-1 has NaN.
 * logits: DEVICE, R rows of V entries of `type`, stride entries apart (>= V).  tokens: DEVICE, R x C, int32 (token_bytes 4) or int64
 * (8); C = 0 for none.  of_token: R x C fp32; entropy: R fp32 or NULL; top_ids: R x top int32; of_top: R x top fp32.
 * R >= 0, 1 <= V <= 2^30, 0 <= top <= min(V, 64), 0 <= C <= 64.
 * workspace: DEVICE, 256-byte aligned, at least tst_logprobs_workspace_bytes() (0 for many rows).
 * Errors: EINVAL, EWORKSPACE, EHIP.
 */
#define TST_LOGPROBS_MAX_TOP 64
#define TST_LOGPROBS_MAX_TOKENS 64
int tst_logprobs_workspace_bytes(int R, int V, int top, size_t *bytes);
int tst_logprobs(const void *logits, int type, int64_t stride, const void *tokens, int token_bytes, int C, int top, float *of_token,
                 float *entropy, int32_t *top_ids, float *of_top, int R, int V, void *workspace, size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* TST_OPS_H */
