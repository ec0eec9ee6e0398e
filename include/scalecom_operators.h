/*
 * scalecom_operators.h -- C ABI of the learner-side operators (B200, sm_100a).
 *
 * scalecom_step() compresses the gradients that n learners hand over and applies
 * the averaged result.  This header has what stands on either side of it when
 * the learners are transformer blocks: the computations whose backward passes
 * write a learner's gradient vector, and the matrix-aware update of the weights.
 *
 *   layer norm            forward, and backward with gamma's and beta's gradients
 *   gated feed-forward    y = (act(x Wg^T) * (x Wu^T)) Wd^T, forward and backward
 *   orthogonalised update Newton-Schulz iteration on a momentum's matrices
 *
 * Conventions (those of scalecom.h; error codes and scalecom_strerror are shared)
 *   - All matrices are row-major.  "ld" is the distance of two rows in ELEMENTS and
 *     at least the row's length.  Any alignment of the element type is accepted;
 *     16-byte aligned bases and row distances take the fast path.
 *   - Weights of a layer norm, statistics and their gradients are fp32 (slices of
 *     the flat vectors of scalecom_step).  Activations are fp32, fp16 or bf16.
 *   - Sums, statistics and accumulators are held in fp32 or more whatever the
 *     type; outputs are rounded once.  Results do not depend on launch timing:
 *     the same call on the same inputs gives the same bits.
 *   - Calls are asynchronous on the handle's stream, except that a call whose
 *     scratch is larger than any before it on the handle waits for the stream
 *     and allocates (scalecom_ops_reserve does that ahead of time; what a call takes is
 *     what scalecom_ops_workspace says after it on a new handle).
 *   - Calls may be captured into a CUDA graph.  One that would have to allocate is then
 *     refused with BAD_STATE.  A graph replays with the scratch of its capture, which the
 *     handle keeps, outgrown or not, until it is destroyed: replays have to come before
 *     that, and stand in line with the handle's other calls.
 *   - Outputs must not overlap inputs or one another unless stated (equality of
 *     base pointers is rejected with ALIAS; partial overlap is undefined).
 *   - Nothing is launched when an argument is rejected.  Sizes of zero that are
 *     said to be accepted make the call a no-op or fill the outputs as stated.
 */
#ifndef SCALECOM_OPERATORS_H
#define SCALECOM_OPERATORS_H

#include <stdint.h>

#include "scalecom.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct scalecom_ops scalecom_ops;

/* Element types. */
#define SCALECOM_F32  0
#define SCALECOM_F16  1
#define SCALECOM_BF16 2

/* Activations of the gated feed-forward block. */
#define SCALECOM_ACT_SILU      0  /* g / (1 + exp(-g))                                           */
#define SCALECOM_ACT_GELU      1  /* g Phi(g), Phi the normal distribution function              */
#define SCALECOM_ACT_GELU_TANH 2  /* g/2 (1 + tanh(sqrt(2/pi) (g + 0.044715 g^3)))               */
#define SCALECOM_ACT_RELU      3  /* max(g, 0); its derivative at 0 is 0                         */

/* Largest rows, width, tokens, hidden, rows and cols of one call (each). */
#define SCALECOM_OPS_MAX_DIM (1 << 26)

/*
 * Operator handle on the current device: a stream binding (default: the legacy
 * default stream) and scratch memory.  Holds no state between calls.  Every DEVICE
 * pointer of its calls is one that this device can read, or write, itself.
 * Errors: NULL_PTR, ALLOC, CUDA (also: not a compute capability 10.0 device).
 */
int scalecom_ops_create(scalecom_ops** out);
void scalecom_ops_destroy(scalecom_ops* ops);                          /* NULL is accepted; waits for the stream */
int scalecom_ops_set_stream(scalecom_ops* ops, void* cuda_stream);     /* waits for the old stream first        */
int scalecom_ops_reserve(scalecom_ops* ops, int64_t bytes);            /* scratch of at least so many bytes     */
int scalecom_ops_workspace(const scalecom_ops* ops, int64_t* bytes);   /* scratch held now                      */

/*
 * Wait for the stream and report the device-side status: OK, TIMEOUT (a bounded
 * wait in a kernel expired; outputs since the last OK are undefined and the handle
 * refuses further calls with BAD_STATE until scalecom_ops_reset) or CUDA.
 */
int scalecom_ops_status(scalecom_ops* ops);
int scalecom_ops_reset(scalecom_ops* ops);

/*
 * Layer norm of `rows` rows of `width` elements:
 *   mean = sum x / width,  rstd = 1 / sqrt(sum (x - mean)^2 / width + eps)
 *   y = (x - mean) * rstd * gamma + beta
 *   dtype       of x and y.
 *   gamma, beta DEVICE fp32[width]; NULL: ones, zeros.
 *   y           may be x itself with the same row distance.
 *   mean, rstd  DEVICE fp32[rows], written; NULL (each) if not wanted.
 * rows = 0 is accepted (nothing is done); width >= 1.  eps >= 0, finite.
 * A row of equal values gives y = beta (with eps > 0, and its sum within fp32's range); NaN and infinities stay in their row.
 */
int scalecom_layer_norm(scalecom_ops* ops, int32_t dtype, int64_t rows, int64_t width,
                        const void* x, int64_t ldx, const float* gamma, const float* beta, float eps,
                        void* y, int64_t ldy, float* mean, float* rstd);

/*
 * Its backward pass, with xh = (x - mean) * rstd and w = dy * gamma:
 *   dx = rstd * (w - mean_row(w) - xh * mean_row(w * xh))
 *   dgamma = sum over rows of dy * xh,  dbeta = sum over rows of dy
 *   gamma       NULL: ones.      dx  may be dy itself (same row distance); NULL if not wanted.
 *   dgamma, dbeta  DEVICE fp32[width], written (not added to); NULL (each) if not wanted.
 * rows = 0: dgamma and dbeta are filled with zeros.
 * Scratch: 32 * width bytes for each multiprocessor (rows longer than 8192 elements: 2 KB * multiprocessors * 8 + 8 * width in all).
 */
int scalecom_layer_norm_backward(scalecom_ops* ops, int32_t dtype, int64_t rows, int64_t width,
                                 const void* dy, int64_t lddy, const void* x, int64_t ldx, const float* gamma,
                                 const float* mean, const float* rstd, void* dx, int64_t lddx,
                                 float* dgamma, float* dbeta);

/*
 * Gated feed-forward block on `tokens` rows of `width` elements:
 *   g = x Wg^T,  u = x Wu^T,  h = act(g) * u,  y = h Wd^T
 *   w_gate, w_up  DEVICE [hidden][width], contiguous.   w_down  DEVICE [width][hidden], contiguous.
 *   dtype         of x, the weights, y and saved.
 *   saved         DEVICE [2][tokens][hidden], written: g, then u, for the backward pass; NULL if not wanted.
 * 16-bit types: products of the type's own values with fp32 accumulation; h (and saved) are rounded to the
 * type once, after the activation.  fp32: every operand is split into two fp16 planes after scaling by a power
 * of two (22 mantissa bits; values under 2^-39 of a tensor's largest magnitude are lost) and three products of planes
 * are accumulated in fp32, which keeps fp32's accuracy; a non-finite operand may make NaN of whatever it is multiplied
 * into.  (Few tokens are multiplied in fp32 as they are.)  g Phi(g) is formed with 1 + erf: far out on the negative side
 * the error is some 2^-25 of g, not of the value.
 * tokens = 0 is accepted (nothing is done); width, hidden >= 1.
 */
int scalecom_gated_ffn(scalecom_ops* ops, int32_t dtype, int32_t act, int64_t tokens, int64_t width, int64_t hidden,
                       const void* x, int64_t ldx, const void* w_gate, const void* w_up, const void* w_down,
                       void* y, int64_t ldy, void* saved);

/*
 * Its backward pass:
 *   dh = dy Wd,  du = dh * act(g),  dg = dh * u * act'(g),  h = act(g) * u
 *   dx = dg Wg + du Wu,  dWg = dg^T x,  dWu = du^T x,  dWd = dy^T h
 *   saved       as the forward pass wrote it.
 *   wgrad_type  type of dw_gate, dw_up, dw_down: dtype, or SCALECOM_F32 (the type of the vectors that
 *               scalecom_step compresses; 16-bit activations with fp32 gradients are the common mixture).
 *   dx, dw_gate, dw_up, dw_down  written; NULL (each) if not wanted.  Contiguous like the weights.
 * dg, du and h are rounded to dtype before they are multiplied (fp32: split into planes as above).
 * tokens = 0: the weight gradients are filled with zeros.
 */
int scalecom_gated_ffn_backward(scalecom_ops* ops, int32_t dtype, int32_t wgrad_type, int32_t act,
                                int64_t tokens, int64_t width, int64_t hidden,
                                const void* dy, int64_t lddy, const void* x, int64_t ldx,
                                const void* w_gate, const void* w_up, const void* w_down, const void* saved,
                                void* dx, int64_t lddx, void* dw_gate, void* dw_up, void* dw_down);

/*
 * Orthogonalise `batch` matrices of rows x cols elements: with X = G / (|G|_F + eps) and, for each of `steps`
 * steps with coefficients (a, b, c),
 *   A = X X^T,  X <- a X + (b A + c A A) X      (X^T X and products from the right when rows > cols)
 * and out = scale * X.  The singular vectors of G are kept, its singular values are driven towards 1.
 *   in_type, in     of the updates; matrix i starts at in + i * in_stride elements, its rows ld_in apart.
 *   out_type, out   the same for the result; `out` may be `in` itself with the same layout and type.
 *   coefficients    HOST float[3 * ncoef]; ncoef is 1 (the same in every step) or steps.  |.| <= 63 each.
 * Precision follows the output: 16-bit outputs iterate on fp16 values of the power-of-two scaled X and A with fp32
 * accumulation (bf16 iterates would lose the small singular values); fp32 outputs iterate on pairs of fp16 planes,
 * three products each, at fp32's accuracy.  Entries of the normalised X are held to 2^-35 at best: a G whose norm is far
 * below eps gives an X that much smaller than 1, and keeps fewer bits.  The scales follow the coefficients: whichever are
 * accepted, results are finite as long as no entry of an X, of its A and of aI + bA + cAA passes 2^75.
 * steps = 0 gives scale * G / (|G|_F + eps).  A zero matrix gives zeros (eps > 0); a NaN or an infinity makes NaN of
 * its own matrix only.  batch = 0 is accepted; rows, cols >= 1; steps <= 64; eps >= 0 and finite; scale finite.
 */
int scalecom_orthogonalise(scalecom_ops* ops, int64_t batch, int64_t rows, int64_t cols,
                           int32_t in_type, const void* in, int64_t ld_in, int64_t in_stride,
                           int32_t out_type, void* out, int64_t ld_out, int64_t out_stride,
                           int32_t steps, const float* coefficients, int32_t ncoef, float eps, float scale);

#ifdef __cplusplus
}
#endif
#endif /* SCALECOM_OPERATORS_H */
