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

/*
 * The residual stream around a block, and the norm in front of the next: a row x of
 * the stream, a block's output b for it, weights w and w', a gate g, a scale a and
 * kept elements z (see dropout, below):
 *
 *     h = b * (mean b^2 + eps)^-1/2      d = h * w'   (no post_weight: d = b)
 *     y = x + a * g * z * d              n = y * (mean y^2 + eps)^-1/2 * w
 *
 * Without a branch y = x is not written, and n alone comes back.
 *
 *   x           in  [M][K] of type stream_dtype, rows ldx apart: dtype itself, or EBSP_F32
 *   branch      in  [M][K] of type dtype, rows ldb apart, or NULL: none
 *   weight      in  [K] of type dtype
 *   post_weight in  [K] of type dtype, or NULL: no norm behind the block
 *   gate        in  of type dtype: [K] where ldgate is 0, otherwise [M][K], rows
 *                   ldgate apart; or NULL: 1
 *   p, seed, offset, rng   dropout of the block's output, as below; p 0: none
 *   y           out [M][K] of type stream_dtype, rows ldy apart; may be x itself (same rows)
 *   n           out [M][K] of type dtype, rows ldn apart
 *   stats       out [M][2] float: the two inverse roots, for the backward pass; or NULL
 * Sums are held in 32 bits; n comes from y before y is rounded.  M == 0 or K == 0
 * is a valid no-op, M is below 2^31, K below 2^30; more rows than a launch has
 * threads for (some four million of K above 4096, 500 million of K up to 64) are
 * refused (EBSP_ERR_SHAPE).
 */
int ebsp_residual_norm_forward(const void* x, int64_t ldx, const void* branch, int64_t ldb, int64_t M, int64_t K, int32_t stream_dtype, int32_t dtype,
                               const void* weight, const void* post_weight, const void* gate, int64_t ldgate, float scale, float eps, float p,
                               uint64_t seed, uint64_t offset, const int64_t* rng, void* y, int64_t ldy, void* n, int64_t ldn, float* stats, void* stream);

/*
 * Its backward pass, from dy and dn (either may be NULL: zero) and the forward pass' y
 * (x itself where there was no branch), stats and operands; the same p, seed, offset
 * and rng give the same kept elements.
 *
 *   dx          out [M][K] of type stream_dtype, rows lddx apart; may be dy itself (same rows)
 *   dbranch     out [M][K] of type dtype, rows lddb apart
 *   dweight, dpost_weight   out [K] of type dtype
 *   dgate       out of type dtype: [K] where ldgate is 0, otherwise [M][K], rows lddgate apart
 *                   Each of the five may be NULL: not wanted.
 *   workspace   at least ebsp_residual_norm_workspace_bytes(M, K) bytes, 256-byte
 *               aligned; may be NULL where no gradient of [K] is wanted
 * Columns are summed in 32 bits in an order that the sizes fix: results do not vary.
 * M == 0 gives zero gradients of [K].
 */
size_t ebsp_residual_norm_workspace_bytes(int64_t M, int64_t K);
int ebsp_residual_norm_backward(const void* dy, int64_t lddy, const void* dn, int64_t lddn, const void* y, int64_t ldy, const void* branch, int64_t ldb,
                                int64_t M, int64_t K, int32_t stream_dtype, int32_t dtype, const void* weight, const void* post_weight, const void* gate,
                                int64_t ldgate, float scale, float p, uint64_t seed, uint64_t offset, const int64_t* rng, const float* stats, void* dx,
                                int64_t lddx, void* dbranch, int64_t lddb, void* dweight, void* dpost_weight, void* dgate, int64_t lddgate,
                                void* workspace, size_t workspace_bytes, void* stream);
/*
 * The same from the forward pass' x, not overwritten since, in the place of y, for a stream
 * of 16 bits that a branch was joined to: the stream is formed again in 32 bits. Such a y
 * was rounded behind its norm, and dweight shows it at the size of its own rounding. (A
 * y of EBSP_F32, and one that is x, are as the norm took them: refused here.)
 */
int ebsp_residual_norm_backward_from_x(const void* dy, int64_t lddy, const void* dn, int64_t lddn, const void* x, int64_t ldx, const void* branch, int64_t ldb,
                                       int64_t M, int64_t K, int32_t stream_dtype, int32_t dtype, const void* weight, const void* post_weight, const void* gate,
                                       int64_t ldgate, float scale, float p, uint64_t seed, uint64_t offset, const int64_t* rng, const float* stats, void* dx,
                                       int64_t lddx, void* dbranch, int64_t lddb, void* dweight, void* dpost_weight, void* dgate, int64_t lddgate,
                                       void* workspace, size_t workspace_bytes, void* stream);

/*
 * Dropout: out = x / (1 - p) where an element is kept, otherwise 0 (whatever x is
 * there).  Which are kept is computed, not stored, so the same call on a gradient is
 * the backward pass.  p is taken to a multiple of 2^-16, and element k of row r is dropped where
 * its 16 bits are below p * 2^16: those of number k % 8, counted from the low end of
 * the first word, in the four words that Philox4x32 of seven rounds (Salmon et al.,
 * 2011) makes of the counter (k / 8, r, offset's low and high word) and the key
 * (seed's low and high word).
 *
 *   x      in  [M][K] of type dtype, rows ldx apart
 *   rng    in  [2] int64 on the device: seed and offset; or NULL: the two arguments
 *              (a replayed graph draws anew where the program moves the offset on)
 *   out    out [M][K] of type dtype, rows ldout apart; may be x itself (same rows)
 * M == 0 or K == 0 is a valid no-op, M is below 2^31, K below 2^30; more elements than
 * some 137 * 10^9 are refused (EBSP_ERR_SHAPE).
 */
int ebsp_dropout(const void* x, int64_t ldx, int64_t M, int64_t K, int32_t dtype, float p, uint64_t seed, uint64_t offset, const int64_t* rng,
                 void* out, int64_t ldout, void* stream);

/*
 * Log-probabilities of tokens: for a row's logits s, its token t and a temperature T,
 *
 *     logp = log softmax(s / T)[t]     dlogp/ds[j] = ([j = t] - softmax(s / T)[j]) / T
 *
 *   logits  in  [N][V] of type dtype, rows ld apart
 *   tokens  in  [N] int64; negative: none in this row, whose logits are not read then.
 *               logp and the gradient of such a row are 0
 *   logp    out [N] float
 *   stats   out [N][3] float: what ebsp_token_logp_backward needs; or NULL
 *   status  out [N] int32, or NULL: EBSP_STATUS_RANGE where a token is V or more; that
 *               row counts as one without a token
 *   dlogp   in  [N] float: dL/dlogp of every row
 *   dlogits out [N][V] of type dtype, rows ldd apart: dL/ds.  May be the logits
 *               themselves (same rows): they are overwritten then
 *   workspace   at least ebsp_token_logp_workspace_bytes(N, V, dtype) bytes,
 *               256-byte aligned (may be NULL when that is 0)
 * Logits of -inf (masked places) weigh nothing; a token at such a place has logp -inf.
 * A temperature is positive, log2(e) / T a finite float.  N == 0 is a valid no-op; V
 * is at least 1; more than some four million rows are refused (EBSP_ERR_SHAPE).
 */
size_t ebsp_token_logp_workspace_bytes(int64_t N, int64_t V, int32_t dtype);
int ebsp_token_logp(const void* logits, int64_t ld, int64_t N, int64_t V, int32_t dtype, const int64_t* tokens, float temperature,
                    float* logp, float* stats, int32_t* status, void* workspace, size_t workspace_bytes, void* stream);
int ebsp_token_logp_backward(const void* logits, int64_t ld, int64_t N, int64_t V, int32_t dtype, const int64_t* tokens, float temperature,
                             const float* stats, const float* dlogp, void* dlogits, int64_t ldd, void* stream);

/*
 * Clipped policy loss with a KL term, token by token: with logp as above, old its
 * value under the policy that drew the token, A the token's advantage and ref its
 * value under a reference,
 *
 *     x = exp(logp - old)
 *     loss = -min(x * A, min(max(x, 1 - clip_low), 1 + clip_high) * A)
 *            + kl_weight * (exp(ref - logp) - (ref - logp) - 1)
 *
 * and its gradient over the logits: dL/dlogp is -x * A (0 where the clipped term is
 * the smaller) - kl_weight * (exp(ref - logp) - 1).
 *
 *   old_logp, advantage  in  [N] float
 *   ref_logp  in  [N] float, or NULL: no KL term
 *   clip_low, clip_high  not negative; infinite: no border on that side
 *   loss      out [N] float;  logp  out [N] float, or NULL
 *   dloss     in  [N] float: dL/dloss of every row
 * The others as above; a row without a token has loss 0, and its old_logp, advantage and
 * ref_logp are not read.  ebsp_policy_forward gives the loss (its workspace:
 * ebsp_token_logp_workspace_bytes), ebsp_policy_backward the gradient from its stats,
 * ebsp_policy_loss_grad both in one pass where a step's dloss is known beforehand
 * (workspace: ebsp_policy_workspace_bytes).  A masked token (logp -inf) has x = 0; with a
 * KL term its loss is +inf and its row's gradient is not finite.
 */
size_t ebsp_policy_workspace_bytes(int64_t N, int64_t V, int32_t dtype);
int ebsp_policy_forward(const void* logits, int64_t ld, int64_t N, int64_t V, int32_t dtype, const int64_t* tokens, float temperature,
                        const float* old_logp, const float* advantage, const float* ref_logp, float clip_low, float clip_high, float kl_weight,
                        float* loss, float* logp, float* stats, int32_t* status, void* workspace, size_t workspace_bytes, void* stream);
int ebsp_policy_backward(const void* logits, int64_t ld, int64_t N, int64_t V, int32_t dtype, const int64_t* tokens, float temperature,
                         const float* old_logp, const float* advantage, const float* ref_logp, float clip_low, float clip_high, float kl_weight,
                         const float* stats, const float* dloss, void* dlogits, int64_t ldd, void* stream);
int ebsp_policy_loss_grad(const void* logits, int64_t ld, int64_t N, int64_t V, int32_t dtype, const int64_t* tokens, float temperature,
                          const float* old_logp, const float* advantage, const float* ref_logp, float clip_low, float clip_high, float kl_weight,
                          const float* dloss, float* loss, float* logp, void* dlogits, int64_t ldd, int32_t* status,
                          void* workspace, size_t workspace_bytes, void* stream);

/* Kinds of preference loss, of the margin h of a pair. */
#define EBSP_PREFERENCE_SIGMOID 0  /* -(1 - smoothing) log sigmoid(beta h) - smoothing log sigmoid(-beta h) */
                                   /* (a term of weight 0 is 0, whatever the margin)                           */
#define EBSP_PREFERENCE_HINGE   1  /* max(0, 1 - beta h)                                                    */
#define EBSP_PREFERENCE_SQUARE  2  /* (h - 1 / (2 beta))^2                                                  */

/*
 * Preference loss of pairs of answers.  The rows of all answers stand one behind the
 * other, answer 2i the preferred of pair i, answer 2i + 1 the other; with the rows'
 * logp as above (at temperature 1) and reference sums ref,
 *
 *     sum_a = the sum of logp over answer a's tokens (with `mean` divided by their number)
 *     h_i = (sum_2i - ref_2i) - (sum_2i+1 - ref_2i+1)
 *
 * and the loss of pair i is a function of h_i, of the kind named.
 *
 *   tokens  in  [N] int64; negative: this row has none (a prompt), and is not read
 *   starts  in  [2 pairs + 1] int64, on the device: answer a is rows starts[a] to
 *               starts[a + 1] - 1 (none where they are equal).  Rows before the first
 *               answer and behind the last are not read; their gradient is 0
 *   ref     in  [2 pairs] float, or NULL: zeros
 *   loss    out [pairs] float;  sums  out [2 pairs] float, or NULL
 *   saved   out [N + pairs][3] float: what ebsp_preference_backward needs; or NULL
 *   status  out [pairs] int32, or NULL: EBSP_STATUS_RANGE where a token of the pair is V
 *               or more (it counts as none), and for every pair where any start is before
 *               0, beyond N or below the one before: no pair's loss and sums mean anything
 *               then, and the gradient is 0
 *   dloss   in  [pairs] float: dL/dloss of every pair
 *   workspace   ebsp_preference_workspace_bytes, 256-byte aligned; for ebsp_preference_forward
 *               with `saved`, ebsp_token_logp_workspace_bytes are enough
 * beta is positive; smoothing, 0 to 1, is of the sigmoid loss alone.  Sums over an
 * answer and what follows of them are held in 64 bits, in an order that the sizes fix.
 * ebsp_preference_loss_grad gives loss and gradient where dloss is known beforehand.
 */
size_t ebsp_preference_workspace_bytes(int64_t N, int64_t pairs, int64_t V, int32_t dtype);
int ebsp_preference_forward(const void* logits, int64_t ld, int64_t N, int64_t V, int32_t dtype, const int64_t* tokens, const int64_t* starts,
                            int64_t pairs, const float* ref, float beta, int32_t kind, float smoothing, int32_t mean, float* loss, float* sums,
                            float* saved, int32_t* status, void* workspace, size_t workspace_bytes, void* stream);
int ebsp_preference_backward(const void* logits, int64_t ld, int64_t N, int64_t V, int32_t dtype, const int64_t* tokens, const int64_t* starts,
                             int64_t pairs, const float* saved, const float* dloss, void* dlogits, int64_t ldd, void* stream);
int ebsp_preference_loss_grad(const void* logits, int64_t ld, int64_t N, int64_t V, int32_t dtype, const int64_t* tokens, const int64_t* starts,
                              int64_t pairs, const float* ref, float beta, int32_t kind, float smoothing, int32_t mean, const float* dloss, float* loss,
                              float* sums, void* dlogits, int64_t ldd, int32_t* status, void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* EBSP_TRAINING_H */
