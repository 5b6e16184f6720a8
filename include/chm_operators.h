/*
 * libchm - operators of a pipeline stage's training step.
 *
 * A scenario (chm.h) is made of the forward and backward times and the memory of every layer on every node.  These are some of the
 * operators that such a step consists of, for one stage on one MI355X (gfx950): the gated feed-forward block forward and backward,
 * the embedding's lookup and gradient, and the global gradient norm with the clipping that ends a step (no attention, norms, output
 * head or optimizer).  All of them run in hand-written HIP kernels; there is no other path.
 *
 * Conventions, beside those of chm.h
 *   - Tensors are DEVICE memory of the caller, aligned to their element size, rows of `ld` elements (>= the row's length).
 *     Outputs must not lie over inputs, scratch or each other, except where a call says so (CHM_ERR_ARG); columns of the same rows of
 *     memory may be different tensors.
 *   - Calls are asynchronous on hip_stream, allocate nothing, and may be captured into a graph.  Scratch is device memory of
 *     the caller, 16-byte aligned, at least as long as the matching *_sizes / *_scratch call says; it is free again when the call's
 *     work on the stream has finished.
 *   - Sums are taken in float32 (sums of squares in float64) in a fixed order: the same inputs give the same bits.
 *   - Not a number and infinities pass through as the formulas have them.
 */
#ifndef CHM_OPERATORS_H
#define CHM_OPERATORS_H
#include "chm.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { CHM_F32 = 0, CHM_BF16 = 1, CHM_F16 = 2 };                             /* types of elements */
enum { CHM_ACT_SILU = 0, CHM_ACT_GELU = 1, CHM_ACT_GELU_TANH = 2 };          /* g sigmoid(g); g Phi(g); its tanh form */

/* ---- Gated feed-forward block -------------------------------------------------------------------------
 * y = h w_down^T,  h = act(g) * u,  g = x w_gate^T,  u = x w_up^T
 * x [tokens, width]; w_gate, w_up [features, width]; w_down [width, features]; y [tokens, width].  No biases.
 * The two projections, the activation and the product are one kernel; h is rounded to the tensors' type between the kernels
 * (in half precision it overflows beyond 65504 as every value of that type does). */
typedef struct {
  int32_t dtype;                              /* CHM_BF16 or CHM_F16: type of all tensors */
  int32_t activation;                         /* CHM_ACT_* */
  int64_t tokens, width, features;            /* tokens >= 0, the others >= 1; tokens below 2^31 - 2^13, width up to 2^22, features
                                                 up to 2^21; both up to 2^24 in forward calls of up to 8 tokens */
  const void *x, *w_gate, *w_up, *w_down;
  int64_t ld_x, ld_gate, ld_up, ld_down;
  void *saved;                                /* g and u as the backward pass wants them (opaque, 16-byte aligned): written by the
                                                 forward call, read by the backward call; NULL in a forward call: not kept */
} chm_ffn;

/* The block forward.  With few tokens (up to 8; 24 or 48 with small weights, 32 with large ones that do not start on 16 bytes) it is
 * bound by reading the weights and runs on kernels for that.  y may lie over x.
 * Errors: CHM_ERR_ARG, CHM_ERR_LIMIT (scratch too short), CHM_ERR_HIP. */
int chm_ffn_forward(const chm_ffn *f, void *y, int64_t ld_y, void *scratch, uint64_t scratch_bytes, void *hip_stream);

/* Gradients of a scalar of which dy is the gradient with respect to y:
 *   dh = dy w_down;  du = dh * act(g);  dg = dh * u * act'(g)
 *   dx = dg w_gate + du w_up;  dw_gate = dg^T x;  dw_up = du^T x;  dw_down = dy^T h
 * dh, h, dg and du are worked out in float32, from g and u of 16 significant bits, and h, dg and du are rounded to the tensors' type once,
 * where they enter a product: against the formulas in 64 bits results are off by 1.4 times what one rounding to that type makes. */
typedef struct {
  const void *dy;                             /* [tokens, width], the tensors' type */
  void *dx;                                   /* [tokens, width], the tensors' type */
  void *dw_gate, *dw_up, *dw_down;            /* shaped like the weights, of type grad_dtype */
  int64_t ld_dy, ld_dx, ld_dw_gate, ld_dw_up, ld_dw_down;
  int32_t grad_dtype;                         /* the tensors' type or CHM_F32 */
  int32_t accumulate;                         /* 1: dw_* += (the micro-batches of a step), 0: dw_* = */
} chm_ffn_gradients;

/* Bytes of `saved` and of the scratch of both calls, for these sizes, rows and alignments of the tensors (an operand whose rows do
 * not start on 16 bytes is packed into scratch).  g: nullable, then *backward_scratch is 0.  Host only.  Errors: CHM_ERR_ARG. */
int chm_ffn_sizes(const chm_ffn *f, const chm_ffn_gradients *g, uint64_t *saved, uint64_t *forward_scratch, uint64_t *backward_scratch);

/* Errors: CHM_ERR_ARG (dw_gate and dw_up must have rows of equal length), CHM_ERR_LIMIT (scratch too short), CHM_ERR_HIP. */
int chm_ffn_backward(const chm_ffn *f, const chm_ffn_gradients *g, void *scratch, uint64_t scratch_bytes, void *hip_stream);

/* ---- Embedding -----------------------------------------------------------------------------------------
 * tokens: n whole numbers of index_bits (32 or 64) bits.  A number outside [0, rows) stands for no token (padding, or a token of
 * another shard of the table): its row of the output is zero and it adds to no gradient. */
/* out[t] = scale * table[tokens[t]]; all of type dtype (CHM_F32, CHM_BF16, CHM_F16).  Errors: CHM_ERR_ARG, CHM_ERR_HIP. */
int chm_embedding_lookup(int32_t dtype, int32_t index_bits, const void *tokens, int64_t n, const void *table, int64_t ld_table,
                         int64_t rows, int64_t width, float scale, void *out, int64_t ld_out, void *hip_stream);

/* grad[v] = scale * sum of dy[t] over the t with tokens[t] = v, in the order of t (accumulate: grad[v] +=, rows that no token
 * names are not touched).  grad is of the type of dy or CHM_F32.  n below 2^31, rows below 2^31.
 * Errors: CHM_ERR_ARG, CHM_ERR_LIMIT (scratch too short), CHM_ERR_HIP. */
int chm_embedding_gradient_scratch(int64_t n, int64_t rows, int64_t width, uint64_t *bytes);
int chm_embedding_gradient(int32_t dtype, int32_t grad_dtype, int32_t index_bits, const void *tokens, int64_t n, const void *dy,
                           int64_t ld_dy, int64_t rows, int64_t width, float scale, void *grad, int64_t ld_grad, int32_t accumulate,
                           void *scratch, uint64_t scratch_bytes, void *hip_stream);

/* ---- Global gradient norm and clipping -----------------------------------------------------------------
 * norm = sqrt(sum over all tensors of g^2);  out = g * min(1, max_norm / (norm + 1e-6)).
 * A handle holds the list of tensors (a training program's gradients stay where they are from step to step); it belongs to the
 * device that was current when it was loaded, and its calls must be issued on one stream or after the caller has waited. */
typedef struct {
  const void *grad;                           /* dense */
  void *out;                                  /* of the same type and length; NULL: in place */
  int64_t n;                                  /* elements, >= 0 */
  int32_t dtype;                              /* CHM_F32, CHM_BF16 or CHM_F16 */
} chm_gradient;
typedef struct chm_gradients chm_gradients;
/* Synchronous.  Errors: CHM_ERR_ARG, CHM_ERR_HIP; *out is NULL then. */
int chm_load_gradients(const chm_gradient *list, int32_t count, chm_gradients **out);
/* *d_sumsq (device) = sum of squares over the handle's tensors: what the stages of a pipeline add up. */
int chm_gradient_sumsq(chm_gradients *g, double *d_sumsq, void *hip_stream);
/* *d_norm (device) = the norm; the tensors are clipped.  d_sumsq (device, nullable): the sum of squares over all stages;
 * NULL: that of the handle's own tensors.  In place, tensors that need no clipping are not written.  max_norm >= 0.
 * A tensor that is listed twice, or a result over another tensor, is CHM_ERR_ARG here (the sum of squares counts it twice). */
int chm_clip_gradients(chm_gradients *g, float max_norm, const double *d_sumsq, float *d_norm, void *hip_stream);
/* Waits for the device's work on the handle. */
void chm_free_gradients(chm_gradients *g);

#ifdef __cplusplus
}
#endif
#endif
