/*
 * libchm - operators of a pipeline stage's training step.
 *
 * A scenario (chm.h) is made of the forward and backward times and the memory of every layer on every node.  These are some of the
 * operators that such a step consists of, for one stage on one MI355X (gfx950): the gated feed-forward block forward and backward,
 * the embedding's lookup and gradient, rotary positions, attention forward and backward, and the global gradient norm with the clipping
 * that ends a step (no projections, norms, output head or optimizer).  All of them run in hand-written HIP kernels; there is no other path.
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

/* ---- Rotary positions ----------------------------------------------------------------------------------
 * Pair i of every head (i < pairs) is turned by the angle positions[axis[i]][t] * frequencies[i] (radians) of its token t:
 *   a' = a cos - b sin,  b' = a sin + b cos;  backwards: by the negative angle, which is the gradient of the forward call.
 * The pair is the elements i and i + pairs (CHM_PAIRS_HALVES) or 2 i and 2 i + 1 (CHM_PAIRS_NEIGHBOURS); elements from 2 pairs on are
 * copied.  One axis for text, more for images (height, width) and video (time, height, width).  Angles are worked out in float64 and
 * reduced to a turn, the sine and cosine in float32: positions may lie far out. */
enum { CHM_PAIRS_HALVES = 0, CHM_PAIRS_NEIGHBOURS = 1 };
typedef struct {
  int32_t dtype;                              /* of x and out: CHM_F32, CHM_BF16 or CHM_F16 */
  int32_t index_bits;                         /* of the positions: 32 or 64 (signed) */
  int32_t pairing;                            /* CHM_PAIRS_* */
  int32_t axes;                               /* >= 1 */
  int64_t tokens, heads;                      /* >= 0, below 2^31 */
  int32_t head_dim, pairs;                    /* 1 <= pairs <= 128, 2 pairs <= head_dim <= 2^20 */
  const void *x;                              /* [tokens, heads, head_dim], strides in elements; x may be out (the same strides) */
  void *out;
  int64_t x_token, x_head, out_token, out_head;
  const void *positions;                      /* [axes, tokens], any strides */
  int64_t positions_axis, positions_token;
  const double *frequencies;                  /* HOST, [pairs], finite; read by the call */
  const int32_t *axis;                        /* HOST, [pairs], each in [0, axes); NULL: all 0 */
} chm_rotary;
/* Errors: CHM_ERR_ARG, CHM_ERR_HIP. */
int chm_rotary_turn(const chm_rotary *r, int32_t backwards, void *hip_stream);

/* ---- Attention -----------------------------------------------------------------------------------------
 * q [batch, tokens, heads, dim], k and v [batch, keys, kv_heads, dim]; query head h reads key head h / (heads / kv_heads).
 *   x = scale q.k;  z = x, or cap tanh(x / cap) where cap > 0;  s = z - slopes[h] |i + keys - tokens - j|
 *   y_i = sum over the visible j of exp(s_ij) v_j / sum over the visible j of exp(s_ij)
 * Query i stands at position i + keys - tokens (new tokens behind those whose keys are there).  Visible are the keys j
 *   - of its own document (documents: a number a token; outside [0, 2^31 - 1) it stands for none, such a token sees nothing and is seen by nobody),
 *   - causal: up to its own position, and wherever prefix[j] is set (a prompt that all of its document sees).
 * A query that sees nothing has a result of zeros and no gradient.  Queries, keys, values and dy of tokens of no document may hold anything; a
 * value that is not finite at a key which some queries see may reach the results of others of the same sequence, and so may a query or dy that is not
 * finite, of a token that has a document, the gradients of keys that it does not see.
 * Gradients, of a scalar of which dy is the gradient with respect to y:
 *   ds = p (dy.v - dy.y);  dq = scale sum_j ds z' k;  dk = scale sum_i ds z' q;  dv = sum_i p dy    (sums over the group's heads)
 * p and ds are worked out in float32 and rounded to the tensors' type once, where they enter a product (in small calls the gradients' products also
 * take what that took): against the formulas in 64 bits gradients are off by up to 1.5 times (1.1 times) what one rounding to that type makes.  In float16 that
 * holds for small and large dy, too: p and ds are rounded 2^12 times as large, a row's ds by a smaller power of two where they would pass what float16 holds. */
typedef struct {
  int32_t dtype;                              /* CHM_BF16 or CHM_F16: type of all tensors */
  int32_t causal;
  int64_t batch, tokens, keys, heads, kv_heads;   /* heads a multiple of kv_heads; tokens and keys up to 2^30, tokens * heads / kv_heads below 2^31 - 2^13 */
  int64_t dim;                                /* 1 to 128 */
  const void *q, *k, *v;
  int64_t q_stride[3], k_stride[3], v_stride[3];  /* elements from one sequence, token, head to the next; >= 0 */
  float scale, cap;                           /* scale > 0, cap finite and >= 0, 0: none; scale and scale / cap up to 1e30 */
  const float *slopes;                        /* [heads], nullable */
  int32_t index_bits;                         /* of the documents: 32 or 64 (signed) */
  const void *q_documents, *k_documents;      /* [batch, tokens], [batch, keys], rows of ld; both or neither (where there are queries and keys) */
  int64_t ld_q_documents, ld_k_documents;
  const uint8_t *prefix;                      /* [batch, keys], rows of ld_prefix, 0 or not; nullable; causal only */
  int64_t ld_prefix;
  void *saved;                                /* what the backward pass wants (opaque, 16-byte aligned), what the tokens' documents are among it: written by the
                                                 forward call, read by the backward call, all else of whose description is the same; NULL in a forward
                                                 call: not kept */
} chm_attention;

typedef struct {
  const void *dy, *y;                         /* [batch, tokens, heads, dim]; y: the forward call's result */
  void *dq, *dk, *dv;                         /* shaped like q, k, v */
  int64_t dy_stride[3], y_stride[3], dq_stride[3], dk_stride[3], dv_stride[3];
} chm_attention_gradients;

/* Bytes of `saved` and of the scratch of both calls (an input whose rows do not start on 16 bytes is packed into scratch).  g: nullable,
 * then *backward_scratch is 0.  Host only.  Errors: CHM_ERR_ARG. */
int chm_attention_sizes(const chm_attention *a, const chm_attention_gradients *g, uint64_t *saved, uint64_t *forward_scratch, uint64_t *backward_scratch);

/* With up to 32 tokens times heads of a group it is bound by reading the keys and values, and runs on a kernel for that; few rows over many keys are
 * split over the keys and joined.  A launch has fewer than 2^24 workgroups: calls of more tiles (32 rows of a small call, 64 or 128 of others; 64 or 128 keys of dk and dv)
 * times sequences and key heads are refused, by chm_attention_sizes as well, and so are inputs of 2^35 elements and more that have to be packed.  Errors: CHM_ERR_ARG, CHM_ERR_LIMIT (scratch too short), CHM_ERR_HIP. */
int chm_attention_forward(const chm_attention *a, void *y, const int64_t y_stride[3], void *scratch, uint64_t scratch_bytes, void *hip_stream);
int chm_attention_backward(const chm_attention *a, const chm_attention_gradients *g, void *scratch, uint64_t scratch_bytes, void *hip_stream);

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
