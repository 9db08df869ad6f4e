/*
 * cocod_lm.h -- operators for workers that train a language model (part of libcocod.so).
 *
 * Algorithm 1 of arxiv 1906.12043, Step II asks for every worker's mini-batch gradient; these calls form it for models
 * made of wide layers and a vocabulary, for all workers of the GPU at once:
 *
 *     cocod_grouped_*   products of rows with their own group's weights, forward and backward
 *     cocod_act_*       activations kept from the forward pass in 8 bits, and their use in the backward pass
 *     cocod_vocab_*     softmax cross-entropy over a large vocabulary, and its gradient
 *     cocod_expert_*    tokens sorted by expert, the rows of the products, and back, with the gradients
 *     cocod_token_*     log probabilities of given tokens, entropy, top alternatives (a router's choice among them), and the gradient
 *
 * Groups.  The rows of all groups (workers, whose mini-batches M_i may differ in size, Section 3.2; or experts) lie one
 * behind the other in one matrix: row m belongs to group g when offsets[g] <= m < offsets[g + 1].  offsets: device,
 * G + 1 int32, rising from 0 to M; groups may be empty.  The offsets are only read on the device.  Offsets that do not
 * rise from 0 to M never lead to an access outside the matrices; the next cocod_lm_check reports them (INVALID;
 * a product without any rows looks at none).
 *
 * Matrices are row-major; a leading dimension (row stride) and a group stride are in elements, so that the weights may be
 * views of the engine's K x P bf16 copy (cocod_get_bf16_shadow) and the weight gradients views of the K x P fp32
 * gradients that cocod_local_step takes.  Every base address has to be a multiple of 16 bytes, and so has every stride;
 * n and k have to be multiples of 8 (INVALID otherwise).  A result may not lie on an operand (but see act_relu_grad).
 *
 * Precision: bf16 operands, products and sums in fp32, one rounding at the end where the result is bf16.
 *
 * Same conventions as cocod.h: int return codes (COCOD_*), device pointers on the device current at create, one host
 * thread per handle, asynchronous on the given stream.  The calls on one handle use scratch of the handle: order them
 * (one stream, or events).  Calls can be captured into a CUDA graph.
 * workspace: device memory lent for the call (until the stream has passed it), 256-byte aligned.
 *
 * An earlier form of the weight gradients (tensor maps modified on the device, scratch recycled between handles) once ended in an illegal
 * address whose cause was not found.  Neither is left: copies go through maps of whole matrices only, made on the host.
 */
#ifndef COCOD_LM_H
#define COCOD_LM_H

#include <stdint.h>

#include "cocod.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct cocod_lm cocod_lm_handle;

enum { COCOD_BF16 = 0, COCOD_F32 = 1 };      /* type of a result */

#define COCOD_LM_MAX_GROUPS 1024

/* Allocates the kernels' scratch (flags, parts of sums), about 20 MB.  Errors: INVALID, OOM, CUDA. */
int cocod_lm_create(cocod_lm_handle **out);
int cocod_lm_destroy(cocod_lm_handle *h);

/* Synchronise `stream` and report what the kernels of this handle met since the last check: COCOD_ERR_TIMEOUT (a kernel
 * gave up a wait), COCOD_ERR_INVALID (offsets that do not rise from 0 to M, a label beyond the vocabulary, an expert beyond their
 * count, or a place beyond the rows), COCOD_OK. */
int cocod_lm_check(cocod_lm_handle *h, cocod_stream_t stream);

/* Number of kernels launched by this handle so far. */
int64_t cocod_lm_launch_count(const cocod_lm_handle *h);

/* ---------------------------------------------------------------------------------------------
 * Products by group.  w: G x [n][k] bf16 (ldw >= k, w_stride between groups).
 *
 * forward        y[m][j]    = sum_i x[m][i] w[g][j][i]        x: M x k,  y: M x n
 * input_grad     dx[m][i]   = sum_j dy[m][j] w[g][j][i]       dy: M x n, dx: M x k
 * weight_grad    dw[g][j][i] = sum_{m in g} dy[m][j] x[m][i]  dw: G x [n][k], written completely (an empty group: 0)
 *
 * out_type: COCOD_BF16 or COCOD_F32.  Long reductions may be cut into parts whose sums are joined in a fixed order; results do not
 * change from call to call. */
int cocod_grouped_forward(cocod_lm_handle *h, int G, const int32_t *offsets, int64_t M, int64_t n, int64_t k,
                          const void *x, int64_t ldx, const void *w, int64_t ldw, int64_t w_stride,
                          void *y, int64_t ldy, int out_type, cocod_stream_t stream);
int cocod_grouped_input_grad(cocod_lm_handle *h, int G, const int32_t *offsets, int64_t M, int64_t n, int64_t k,
                             const void *dy, int64_t lddy, const void *w, int64_t ldw, int64_t w_stride,
                             void *dx, int64_t lddx, int out_type, cocod_stream_t stream);
int cocod_grouped_weight_grad(cocod_lm_handle *h, int G, const int32_t *offsets, int64_t M, int64_t n, int64_t k,
                              const void *dy, int64_t lddy, const void *x, int64_t ldx,
                              void *dw, int64_t lddw, int64_t dw_stride, int out_type, cocod_stream_t stream);

/* ---------------------------------------------------------------------------------------------
 * Activations in 8 bits.  A block is 128 consecutive columns of a row (the last one of a row may be shorter).  With amax
 * the largest finite magnitude of the block and e the least integer >= -126 with amax <= 127 * 2^e,
 *     q = sign(x) * max(1, rint(|x| / 2^e)) for x != 0, else 0              (half to even)
 * stands for q * 2^e: within half a unit of x (within one for |x| < 2^e / 2: the sign of a value always survives, so that
 * the gate of a ReLU can be taken from it; and within one where e is 122: bf16 ends below 64 * 2^122, so |q| stops at 63), and exact in bf16.  q = -128 marks a value that was not finite; a block that holds
 * one has scale byte 255 and reads as NaN.
 *   q      : M x k int8, row stride ldq (a multiple of 16, >= k); what lies behind a row's k values is never written, and read at
 *            most up to the next multiple of 8 bytes (whatever it holds)
 *   scales : ceil(k / 128) x M bytes, e + 127 (or 255)
 *
 * act_pack       x: M x k bf16 (any k and ldx, any 2-byte alignment; 16-byte aligned rows are faster)
 * act_unpack     y: M x k bf16
 * act_relu_grad  dz = (q > 0) ? dh : 0  (NaN where q marks a value that was not finite), dh, dz: M x k bf16; dz may be dh
 * weight_grad_packed  as cocod_grouped_weight_grad, with x as the checkpoint stands for it.  With a workspace of M * k * 2 bytes the
 *   checkpoint is turned into bf16 there first, otherwise inside the product; the results are the same.
 *   cocod_grouped_packed_workspace: the bytes with which the call is faster (0 where it is faster without). */
int cocod_act_pack(cocod_lm_handle *h, int64_t M, int64_t k, const void *x, int64_t ldx, int8_t *q, int64_t ldq,
                   uint8_t *scales, cocod_stream_t stream);
int cocod_act_unpack(cocod_lm_handle *h, int64_t M, int64_t k, const int8_t *q, int64_t ldq, const uint8_t *scales,
                     void *y, int64_t ldy, cocod_stream_t stream);
int cocod_act_relu_grad(cocod_lm_handle *h, int64_t M, int64_t k, const void *dh, int64_t lddh, const int8_t *q, int64_t ldq,
                        void *dz, int64_t lddz, cocod_stream_t stream);
int cocod_grouped_weight_grad_packed(cocod_lm_handle *h, int G, const int32_t *offsets, int64_t M, int64_t n, int64_t k,
                                     const void *dy, int64_t lddy, const int8_t *q, int64_t ldq, const uint8_t *scales,
                                     void *dw, int64_t lddw, int64_t dw_stride, int out_type,
                                     void *workspace, int64_t workspace_bytes, cocod_stream_t stream);
int64_t cocod_grouped_packed_workspace(int G, int64_t M, int64_t n, int64_t k);

/* ---------------------------------------------------------------------------------------------
 * Softmax cross-entropy over a vocabulary of V entries, each group with an output matrix w[g] (V x D) of its own:
 *     l[r][v] = sum_i x[r][i] w[g][v][i],   row_loss[r] = log sum_v exp(l[r][v]) - l[r][label_r],
 *     loss[g] = sum over the group's rows of a_r row_loss[r],
 *     dx[r] = a_r sum_v (softmax - onehot)[r][v] w[g][v],   dw[g][v] = sum_r a_r (softmax - onehot)[r][v] x[r].
 * a_r = row_weights[r], or, where row_weights is NULL, 1 / (rows of the group that take part): the mean.
 * Rows whose label is negative (or whose weight is 0) take no part whatever they hold: row_loss and dx are 0 there.  A
 * group of which no row takes part has loss 0 and dw 0.  A label >= V is reported by cocod_lm_check; its row takes no part.
 *   x: M x D bf16;  w: bf16;  labels: M int32;  row_weights: M fp32 or NULL;  loss: G fp32;  row_loss: M fp32
 *   dx: M x D bf16;  dw: G x [V][D], bf16 or fp32, written completely.  V: any; D: a multiple of 8.
 * The logits are never written.  cocod_vocab_loss keeps two numbers for each row and 64 or 128 entries; cocod_vocab_loss_grad keeps
 * exp(l - l[label]) in bf16 for as many rows at a time as the workspace holds (at least 256, or all), and adds up dw over
 * these passes in fp32.  cocod_vocab_workspace: the bytes for one pass over all rows, or, if that is more than `limit`,
 * for the most rows that stay within it (more than `limit` if not even the fewest do); less: COCOD_ERR_TOO_LARGE.
 * Precision: the exponentials and a_r x / sum are rounded to bf16 as operands of the gradients' products (a term of dx carries a
 * relative error of up to 2^-8, the label's none; a term of dw up to 3 * 2^-8, also where dw is fp32); the losses are formed in fp32. */
int64_t cocod_vocab_workspace(int G, int64_t M, int64_t V, int64_t D, int with_grad, int dw_type, int64_t limit);
int cocod_vocab_loss(cocod_lm_handle *h, int G, const int32_t *offsets, int64_t M, int64_t V, int64_t D, const void *x, int64_t ldx,
                     const void *w, int64_t ldw, int64_t w_stride, const int32_t *labels, const float *row_weights, float *loss,
                     float *row_loss, void *workspace, int64_t workspace_bytes, cocod_stream_t stream);
int cocod_vocab_loss_grad(cocod_lm_handle *h, int G, const int32_t *offsets, int64_t M, int64_t V, int64_t D, const void *x, int64_t ldx,
                          const void *w, int64_t ldw, int64_t w_stride, const int32_t *labels, const float *row_weights, float *loss,
                          float *row_loss, void *dx, int64_t lddx, void *dw, int64_t lddw, int64_t dw_stride, int dw_type,
                          void *workspace, int64_t workspace_bytes, cocod_stream_t stream);

/* ---------------------------------------------------------------------------------------------
 * Tokens sorted by expert and back.  Token t has k slots s = t k + j, slot s goes to expert experts[t][j]; N = T k.
 *
 * expert_sort      the slots in the order of their experts (stable: of one expert, in their own order).  order[r]: the slot of row r;
 *                  place[s]: the row of slot s; counts[e]: the slots of expert e; offsets: E + 1 values, as the products by group take them.
 *   A negative number is a slot that takes no part; one >= E too, and the next cocod_lm_check reports it.  Such slots' rows lie behind the last
 *   expert's and count as its own in the offsets, which so rise from 0 to N always (counts[E - 1] leaves them out); place[s] is the
 *   bitwise complement of the row there.
 * expert_rows      rows[place[s]] = x[s / k]; zeros in the rows of slots that take no part
 * expert_join      y[t] = sum_j weights[t][j] rows[place[t][j]] over the slots that take part, in fp32 in the order of j; weights NULL: the sum
 *                  alone, which is the gradient of expert_rows
 * expert_join_grad drows[place[s]] = weights[s] dy[s / k] (zeros in rows of slots that take no part), dweights[s] = <dy[s / k], rows[place[s]]>
 *                  (0 there); a result may not lie on an operand
 *   experts: T x k int32, row stride ld; order, place, weights, dweights: N values; k <= 32, E <= COCOD_LM_MAX_GROUPS, N < 2^31 - 1024
 *   x, y, dy: T x D; rows, drows: N x D; type: COCOD_BF16 or COCOD_F32, any D, row stride and alignment (rows that start at multiples of 16 bytes
 *   and hold a multiple of them are faster).  Rows that no place names are not written.  A place beyond the rows is
 *   reported by cocod_lm_check and left out.
 * workspace: cocod_expert_workspace bytes (4-byte aligned; may be 0); less: COCOD_ERR_TOO_LARGE. */
#define COCOD_LM_MAX_CHOICES 32
int64_t cocod_expert_workspace(int64_t T, int k, int E);
int cocod_expert_sort(cocod_lm_handle *h, int64_t T, int k, int E, const int32_t *experts, int64_t ld, int32_t *offsets, int32_t *counts, int32_t *order,
                      int32_t *place, void *workspace, int64_t workspace_bytes, cocod_stream_t stream);
int cocod_expert_rows(cocod_lm_handle *h, int64_t T, int k, int64_t D, const void *x, int64_t ldx, const int32_t *place, void *rows, int64_t ld, int type,
                      cocod_stream_t stream);
int cocod_expert_join(cocod_lm_handle *h, int64_t T, int k, int64_t D, const void *rows, int64_t ld, int type, const int32_t *place, const float *weights, void *y,
                      int64_t ldy, int out_type, cocod_stream_t stream);
int cocod_expert_join_grad(cocod_lm_handle *h, int64_t T, int k, int64_t D, const void *dy, int64_t lddy, const void *rows, int64_t ld, const int32_t *place,
                           const float *weights, void *drows, int64_t ld_drows, float *dweights, int type, cocod_stream_t stream);

/* ---------------------------------------------------------------------------------------------
 * Log probabilities of given tokens.  logits: M x V (type COCOD_BF16 or COCOD_F32, any row stride and alignment); y = scale * logits, 1e-30 <= scale <= 1e30;
 *     log_sum[r] = log sum_v exp y[r][v],   log p = y - log_sum,   logp[r] = log p[r][tokens[r]],
 *     entropy[r] = - sum_v p log p,   top_tokens[r][j]: the token with the j-th largest logit (of equal ones the lower first), top_logp: its log p.
 * tokens: M int32, or NULL: no tokens, logp is not written.  A row whose token is negative takes no part whatever it holds: its results are 0, its
 * top_tokens -1; so does one whose token is >= V, which the next cocod_lm_check reports.  top: 0 .. 32, at most V.
 * A logit of -inf has probability 0.  A row of nothing else: log_sum and every log p are -inf, entropy and gradient 0.  A row with a NaN or
 * +inf: NaN for logp, entropy, log_sum and top_logp; top_tokens orders NaN before all others.
 *
 * token_logprobs_grad   dlogits = scale * (given - p * (sum of given + d_entropy * (log p + entropy))), with `given` the sum of d_logp at the row's token
 *   and d_top at its top_tokens (a repeated or negative one is allowed: added up, left out).  log_sum and entropy are those of the forward call; log p
 *   is y - log_sum in fp32, off by up to 2^-23 (|y| + |log_sum|) also where p is near 1.
 *   d_logp, d_entropy, d_top: NULL where there are none (entropy is read only with d_entropy; top_tokens and d_top are M x top).  dlogits:
 *   M x V of the logits' type; may be the logits themselves (same address and stride). */
#define COCOD_LM_MAX_TOP 32
int cocod_token_logprobs(cocod_lm_handle *h, int64_t M, int64_t V, const void *logits, int64_t ld, int type, const int32_t *tokens, float scale, int top,
                         float *logp, float *entropy, float *log_sum, float *top_logp, int32_t *top_tokens, cocod_stream_t stream);
int cocod_token_logprobs_grad(cocod_lm_handle *h, int64_t M, int64_t V, const void *logits, int64_t ld, int type, const int32_t *tokens, float scale, int top,
                              const int32_t *top_tokens, const float *log_sum, const float *entropy, const float *d_logp, const float *d_entropy,
                              const float *d_top, void *dlogits, int64_t ld_dlogits, cocod_stream_t stream);

/* Self-test of the bounded waits of the product kernels: one launch (pairs of thread blocks when `pair` is not 0) whose
 * copies are never issued.  Every wait ends after at most 1.5 * wait_ms (1 .. 2000), COCOD_ERR_TIMEOUT is returned and the
 * context stays usable. */
int cocod_grouped_wait_selftest(int wait_ms, int pair, cocod_stream_t stream);

#ifdef __cplusplus
}
#endif
#endif /* COCOD_LM_H */
