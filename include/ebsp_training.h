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
 *   g, u    out [M][F], rows ldg apart: what ebsp_gated_ff_backward needs.
 *               Both NULL where there will be no backward pass; h alone is
 *               written then.
 * All of one element type `dtype`; sums are held in 32 bits and rounded once.
 * M == 0 or F == 0 is a valid no-op, K == 0 gives zero products.
 */
int ebsp_gated_ff_forward(const void* x, int64_t ldx, const void* wg, int64_t ldwg, const void* wu, int64_t ldwu,
                          int64_t M, int64_t K, int64_t F, int32_t dtype, int32_t act,
                          void* h, int64_t ldh, void* g, void* u, int64_t ldg, void* stream);

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
 *                256-byte aligned (it holds dg and du, rounded to dtype).
 * M == 0 gives zero weight gradients, F == 0 a zero dx.
 */
size_t ebsp_gated_ff_workspace_bytes(int64_t M, int64_t F, int32_t dtype);
int ebsp_gated_ff_backward(const void* dh, int64_t lddh, const void* x, int64_t ldx, const void* wg, int64_t ldwg,
                           const void* wu, int64_t ldwu, const void* g, const void* u, int64_t ldg,
                           int64_t M, int64_t K, int64_t F, int32_t dtype, int32_t act,
                           void* dx, int64_t lddx, void* dwg, void* dwu, int64_t lddw,
                           void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* EBSP_TRAINING_H */
