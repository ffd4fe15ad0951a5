/*
 * ebsp_training.h -- C ABI of the training operators next to the ZipLine
 * barrier search (ebsp_zipline.h), for MI355X (gfx950).
 *
 * The search decides how many iterations every worker runs before the next
 * barrier (Fig. 1 of the ElasticBSP paper, arXiv 2001.01347).  The operators
 * here are what lies on either side of that decision: what a worker computes in
 * an iteration, and what the server does with the workers' pushes at a barrier
 * (Section III).  The paper trains other networks and leaves the merge to its
 * parameter server; the formulas are stated with each operator.
 *
 * As in ebsp_zipline.h: data pointers are DEVICE pointers owned by the caller,
 * calls only enqueue kernels on `stream` (no memory set or copy), allocate
 * nothing, and return EBSP_OK or a negative EBSP_ERR_* code with nothing
 * enqueued (EBSP_ERR_LAUNCH may follow earlier launches of the same call);
 * ebsp_last_error() says what was wrong.  A stream may be captured into a HIP
 * graph around a call; the first call on a device also asks the runtime for the
 * device's name, so make one call before capturing.
 *
 * Matrices are row-major with unit stride along a row; ld* is the distance
 * between rows in elements and at least the row's length.  Any alignment of an
 * element's own size is right; rows that start at multiples of 16 bytes are
 * faster.  Outputs must not overlap inputs except where stated.
 */
#ifndef EBSP_TRAINING_H
#define EBSP_TRAINING_H

#include "ebsp_zipline.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types. */
#define EBSP_BF16  0
#define EBSP_F16   1
#define EBSP_F32   2

/* Return code besides those of ebsp_zipline.h. */
#define EBSP_ERR_ARGUMENT     -6   /* an element type, activation, stride or number is not one that the call takes */

/* Activations of the gated feed-forward block. */
#define EBSP_ACT_SILU       0      /* g * sigmoid(g)                                        */
#define EBSP_ACT_GELU       1      /* g * Phi(g), Phi the normal distribution function      */
#define EBSP_ACT_GELU_TANH  2      /* g/2 * (1 + tanh(sqrt(2/pi) * (g + 0.044715 * g^3)))   */
#define EBSP_ACT_RELU       3
#define EBSP_ACT_SIGMOID    4

/*
 * Gated feed-forward block, forward:
 *
 *     g = x Wg^T     u = x Wu^T     h = act(g) * u
 *
 *   x       in  [M][K], rows ldx apart
 *   wg, wu  in  [F][K], rows ldwg and ldwu apart
 *   h       out [M][F], rows ldh apart
 *   g, u    out [M][F] float, rows ldg apart: what ebsp_gated_ff_backward
 *               needs.  Both NULL where there will be no backward pass; h
 *               alone is written then.
 * The others of one element type `dtype`; sums are held in 32 bits and rounded once.
 * M == 0 or F == 0 is a valid no-op, K == 0 gives zero products.  M, K and F are
 * below 2^31, M x F below 2^56.
 *
 * ebsp_gated_ff_forward_split does the same with a workspace, 256-byte aligned:
 * where ebsp_gated_ff_forward_workspace_bytes(M, K, F, dtype) is not 0 and the
 * workspace is that large, long sums of few results run in several parts side by
 * side, which is faster there.  NULL or less room: as ebsp_gated_ff_forward.
 */
int ebsp_gated_ff_forward(const void* x, int64_t ldx, const void* wg, int64_t ldwg, const void* wu, int64_t ldwu,
                          int64_t M, int64_t K, int64_t F, int32_t dtype, int32_t act,
                          void* h, int64_t ldh, float* g, float* u, int64_t ldg, void* stream);
size_t ebsp_gated_ff_forward_workspace_bytes(int64_t M, int64_t K, int64_t F, int32_t dtype);
int ebsp_gated_ff_forward_split(const void* x, int64_t ldx, const void* wg, int64_t ldwg, const void* wu, int64_t ldwu,
                                int64_t M, int64_t K, int64_t F, int32_t dtype, int32_t act,
                                void* h, int64_t ldh, float* g, float* u, int64_t ldg,
                                void* workspace, size_t workspace_bytes, void* stream);

/*
 * Its backward pass: from dh = dL/dh,
 *
 *     du = dh * act(g)          dg = dh * u * act'(g)
 *     dx = dg Wg + du Wu        dWg = dg^T x        dWu = du^T x
 *
 *   dh       in  [M][F], rows lddh apart;  g, u: as the forward pass left them
 *   dx       out [M][K], rows lddx apart, or NULL: not wanted
 *   dwg, dwu out [F][K], rows lddw apart, or both NULL: not wanted
 *   workspace    at least ebsp_gated_ff_workspace_bytes(M, F, dtype) bytes,
 *                256-byte aligned (it holds dg and du, rounded to dtype; in fp16
 *                times a common power of two where their largest is above 65504
 *                or below 2^-6).  With
 *                ebsp_gated_ff_split_workspace_bytes(M, K, F, dtype) bytes, where
 *                that is more, long sums of small results run in several parts
 *                side by side, which is faster (dx where tokens are few, the
 *                weights' gradients where tokens are many and matrices small).
 * M == 0 gives zero weight gradients, F == 0 a zero dx.
 */
size_t ebsp_gated_ff_workspace_bytes(int64_t M, int64_t F, int32_t dtype);
size_t ebsp_gated_ff_split_workspace_bytes(int64_t M, int64_t K, int64_t F, int32_t dtype);
int ebsp_gated_ff_backward(const void* dh, int64_t lddh, const void* x, int64_t ldx, const void* wg, int64_t ldwg,
                           const void* wu, int64_t ldwu, const float* g, const float* u, int64_t ldg,
                           int64_t M, int64_t K, int64_t F, int32_t dtype, int32_t act,
                           void* dx, int64_t lddx, void* dwg, void* dwu, int64_t lddw,
                           void* workspace, size_t workspace_bytes, void* stream);

/* Status bit of a row of the distillation loss (status[n], beside EBSP_STATUS_OK). */
#define EBSP_STATUS_RANGE      4   /* an index or a label is V or more: that entry or term is left out */

#define EBSP_DISTILL_TOP_MAX 1024  /* most entries of a row */

/*
 * Distillation from a teacher's top logits.  A row holds the student's logits s
 * over a vocabulary of V and the teacher's largest logits t_k with their places
 * i_k, k < top.  With a temperature T, q = softmax(t / T) over the row's
 * entries, p = softmax(s / T) and p1 = softmax(s):
 *
 *     loss = kl_weight * T^2 * sum_k q_k (log q_k - log p[i_k])
 *            - ce_weight * log p1[label]
 *     dloss/ds[j] = kl_weight * T * (p[j] - sum_{k: i_k = j} q_k)
 *            + ce_weight * (p1[j] - [j = label])
 *
 *   logits    in  [N][V] of type dtype, rows ld apart
 *   top_index in  [N][top], rows ldt apart; index_bytes says which: 4 or 8 (signed).
 *                 Negative: padding, no entry.  Entries of one place add up.
 *   top_logit in  [N][top] of type top_dtype, rows ldt apart; -inf weighs nothing
 *   labels    in  [N] int64, or NULL: no second term; negative: none in this row
 *   loss      out [N] float
 *   stats     out [N][3] float: what ebsp_distill_backward needs of the
 *                 forward pass; or NULL
 *   dloss     in  [N] float: dL/dloss of every row
 *   dlogits   out [N][V] of type dtype, rows ldd apart: dL/ds.  May be the
 *                 logits themselves (same rows): they are overwritten then
 *   status    out [N] int32, or NULL
 *   workspace     at least ebsp_distill_workspace_bytes(N, V, dtype) bytes,
 *                 256-byte aligned (may be NULL when that is 0)
 * A row without entries has no first term and its gradient no p.  Logits of -inf
 * (masked places) have p = 0, and where the teacher gives such a place weight the
 * loss is +inf.  A temperature is positive, log2(e) / T a finite float.
 * ebsp_distill_forward gives the loss, ebsp_distill_backward the
 * gradient from its stats, ebsp_distill_loss_grad both in one pass where a step's
 * dloss is known beforehand (1 / N for a mean).  top_index and top_logit may be
 * NULL when top is 0.  N == 0 is a valid no-op; V is at least 1; more than some
 * four million rows are refused (EBSP_ERR_SHAPE): split them.
 */
size_t ebsp_distill_workspace_bytes(int64_t N, int64_t V, int32_t dtype);
int ebsp_distill_forward(const void* logits, int64_t ld, int64_t N, int64_t V, int32_t dtype,
                         const void* top_index, int32_t index_bytes, const void* top_logit, int32_t top_dtype, int64_t ldt, int32_t top,
                         const int64_t* labels, float temperature, float kl_weight, float ce_weight,
                         float* loss, float* stats, int32_t* status, void* workspace, size_t workspace_bytes, void* stream);
int ebsp_distill_backward(const void* logits, int64_t ld, int64_t N, int64_t V, int32_t dtype,
                          const void* top_index, int32_t index_bytes, const void* top_logit, int32_t top_dtype, int64_t ldt, int32_t top,
                          const int64_t* labels, float temperature, float kl_weight, float ce_weight,
                          const float* stats, const float* dloss, void* dlogits, int64_t ldd, void* stream);
int ebsp_distill_loss_grad(const void* logits, int64_t ld, int64_t N, int64_t V, int32_t dtype,
                           const void* top_index, int32_t index_bytes, const void* top_logit, int32_t top_dtype, int64_t ldt, int32_t top,
                           const int64_t* labels, float temperature, float kl_weight, float ce_weight,
                           const float* dloss, float* loss, void* dlogits, int64_t ldd, int32_t* status,
                           void* workspace, size_t workspace_bytes, void* stream);

#define EBSP_MERGE_WORKERS_MAX 4096   /* most workers of a merge */

/*
 * What the server does at a barrier (Section III): the workers' pushes, each the
 * change of its weights since the last barrier, merged by the iterations that the
 * search gave the workers (iters[b] of ebsp_zipline_batch and the others, still on
 * the device), and applied to the server's weights:
 *
 *     c_p = iters[p] / sum iters     avg = sum_p c_p * push_p
 *     v'  = momentum * v + avg       w'  = w + lr * (nesterov ? avg + momentum * v' : v')
 *
 * and without a velocity w' = w + lr * avg.  (The paper leaves the server's
 * update open; weights by iterations are this library's reading, momentum the
 * usual choice for merged local steps.)
 *
 *   pushes       in  [P][n] of type dtype, a worker's row `stride` after the one before
 *   iters        in  [P] int32.  A worker with 0 or less has no part in the merge
 *                    and its row is not read; with no worker left nothing changes
 *   weights      in  [n] float;   weights_out  out [n] float, may be weights itself
 *   velocity     in  [n] float;   velocity_out out [n] float, may be velocity
 *                    itself; both NULL: no momentum
 *   pull         out [n] of type pull_dtype: w' rounded, what the workers fetch; or NULL
 * Sums are held in 32 bits and run in an order that P and n fix: results do not
 * vary.  P is 1 to EBSP_MERGE_WORKERS_MAX, n below 2^34, or at most 2^34 - 1024
 * where the pushes are fp32.  n == 0 is a valid no-op.
 */
int ebsp_merge_pushes(const void* pushes, int64_t stride, int32_t P, int64_t n, int32_t dtype, const int32_t* iters,
                      const float* weights, const float* velocity, float lr, float momentum, int32_t nesterov,
                      float* weights_out, float* velocity_out, void* pull, int32_t pull_dtype, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* EBSP_TRAINING_H */
