/*
 * sc_block.h - the operators of an encoder block beside its attention (sc.h):
 * matrix products in 8-bit integers, and the norms before and after a block
 * fused with the block's gate and the residual's scale, with their gradients.
 *
 *   sc_quantize_rows_i8    8-bit rows with one scale per token;
 *   sc_quantize_weight_i8  8-bit weights with one scale per output channel, laid
 *                          out once for the products;
 *   sc_linear_i8           out = act(x . W + bias) on them, sums in int32;
 *   sc_block_norm          r = res_scale x + gate * post(t), y = pre(r), y also
 *                          as 8-bit rows for the next product;
 *   sc_block_norm_backward its gradients;
 *   sc_encoder_stack_i8    sc_encoder_stack (sc.h) with these products, biases,
 *                          norm weights, residual scale and gates: the form in
 *                          which a trained encoder is served.
 *
 * The conventions of sc.h hold: device tensors owned by the caller, scratch
 * memory from `workspace`, everything enqueued on `stream` without
 * synchronisation or allocation (all calls may be captured into a graph),
 * arguments checked on the host before anything is enqueued, and no state kept
 * between calls.  Tensors are dense and row-major.  Rows come as a padded
 * batch: sequence b of B holds valid_len[b] of n rows, 0 <= valid_len[b] <= n
 * (device int32 [B]; values outside are clamped), or n without valid_len
 * (NULL).  Output rows of padding are zero, and padding rows of inputs are not
 * read into any result.  Every result is deterministic, and a row's result
 * depends neither on the other rows nor on the batch.  Tensors are aligned to
 * their elements, 8-bit rows and workspaces to 16 bytes.
 */
#ifndef SC_BLOCK_H_
#define SC_BLOCK_H_

#include "sc.h"

#ifdef __cplusplus
extern "C" {
#endif

#define SC_I8 2 /* 8-bit integers, one float32 scale per row (beside SC_F32, SC_BF16) */

/* ------------------------------------------------------- 8-bit products -- */

/* Bytes of a row of K 8-bit values: K rounded up to 128.  The bytes beyond K
 * are zero wherever the library writes such rows, and have to be zero (in the
 * rows or in the weights) where it reads them.  0 for K < 1. */
int64_t sc_i8_pitch(int64_t K);

/*
 * 8-bit rows: for a row x of K values with a = max_k |x_k|,
 *   scale = a / 127 (float32),  q_k = the integer nearest to 127 x_k / a,
 *   halves to the even one (of the exact quotient, whatever the type of x);
 * a row of zeros gives scale 0 and zeros; a row with an infinity or a NaN
 * gives scale NaN and zeros, so that every product of it is NaN.
 *   x      [B, n, K] in dtype (SC_F32 or SC_BF16).
 *   xq     int8 [B, n, sc_i8_pitch(K)];  scale  float32 [B, n].
 *   Padding rows: zeros, scale 0.
 * Errors: SC_EINVAL (null or overlapping buffers, sizes below 1, dtype, xq not
 * 16-byte aligned), SC_EUNSUPPORTED (B n >= 2^31, K >= 2^29).
 */
sc_status sc_quantize_rows_i8(int32_t B, int32_t n, int32_t K, const int32_t *valid_len, int32_t dtype,
                              const void *x, int8_t *xq, float *scale, void *stream);

/*
 * 8-bit weights of sc_linear_i8 from W [K, N] (row-major, dtype SC_F32 or
 * SC_BF16): the rule of sc_quantize_rows_i8 for every column of W.
 *   wq  int8 [N, sc_i8_pitch(K)] (output channel-major), scale float32 [N].
 * Weights quantised elsewhere serve as well in this layout.
 * Errors as for sc_quantize_rows_i8; N pitch >= 2^32 is SC_EUNSUPPORTED.
 */
sc_status sc_quantize_weight_i8(int32_t K, int32_t N, int32_t dtype, const void *w, int8_t *wq, float *scale,
                                void *stream);

#define SC_ACT_NONE 0
#define SC_ACT_GELU 1 /* v * Phi(v), float32 before the store: within 2.4e-7, and 3e-5 of the value down to v = -9 */

typedef struct sc_linear_desc {
  int32_t B, n, K, N;        /* rows as above, K inputs, N outputs per row */
  const int32_t *valid_len;  /* device int32 [B], or NULL                  */
  int32_t x_dtype;           /* SC_F32, SC_BF16 or SC_I8                   */
  int32_t out_dtype;         /* SC_F32 or SC_BF16                          */
  int32_t act;               /* SC_ACT_*                                   */
} sc_linear_desc;

size_t sc_linear_i8_workspace_size(const sc_linear_desc *desc);

/*
 * out[b,j,:] = act(x_scale[b,j] * w_scale[:] * (xq[b,j,:] . wq[:,:]^T) + bias[:])
 * for j < valid_len[b], 0 for the padding rows.  The sum of products is exact
 * (int32; K <= 131072, integers from -127 to 127), everything after it float32,
 * rounded once to out_dtype.
 *   x        SC_I8: the 8-bit rows [B, n, sc_i8_pitch(K)] (16-byte aligned), with
 *            x_scale float32 [B, n].  SC_F32, SC_BF16: [B, n, K], quantised in
 *            the call as by sc_quantize_rows_i8; x_scale must be NULL.
 *   wq, w_scale  as sc_quantize_weight_i8 lays them out (wq 16-byte aligned).
 *   bias     float32 [N] or NULL.
 *   out      [B, n, N] in out_dtype.
 * The product has no gradient to speak of (rounding is constant almost
 * everywhere); it serves trained models.
 * Errors: SC_EINVAL (null pointers, sizes, types, alignment, out overlapping
 * an input or the workspace), SC_EUNSUPPORTED (K > 131072, B n >= 2^31, B n
 * pitch >= 2^32, N pitch >= 2^32; with valid_len, B > 8192), SC_EWORKSPACE.
 */
sc_status sc_linear_i8(const sc_linear_desc *desc, const void *x, const float *x_scale, const int8_t *wq,
                       const float *w_scale, const float *bias, void *out, void *workspace, size_t ws_bytes,
                       void *stream);

/* ---------------------------------------------------------- block norms -- */

#define SC_NORM_LAYER 0 /* (v - mean) / sqrt(var + eps), biased variance */
#define SC_NORM_RMS 1   /* v / sqrt(mean(v^2) + eps)                      */

#define SC_GATE_NONE 0
#define SC_GATE_CHANNEL 1  /* gate float32 [D]           */
#define SC_GATE_SEQUENCE 2 /* gate [B, D] in dtype       */
#define SC_GATE_TOKEN 3    /* gate [B, n, D] in dtype    */

typedef struct sc_norm_desc {
  int32_t B, n, D;          /* rows as above, D channels, D <= 4096        */
  const int32_t *valid_len; /* device int32 [B], or NULL                   */
  int32_t kind;             /* SC_NORM_*: of both norms                    */
  int32_t post, pre;        /* 0 or 1: norm after the block, norm before the next */
  int32_t gate_mode;        /* SC_GATE_*                                   */
  float eps;                /* > 0                                         */
  float res_scale;          /* of the residual x                           */
  int32_t dtype;            /* SC_F32 or SC_BF16: x, t, r, y, gradients    */
} sc_norm_desc;

/*
 * What stands between two blocks of an encoder, per row:
 *   u = post ? norm(t) * post_w + post_b : t          norm after the block
 *   r = res_scale * x + gate * u                      gated, scaled residual
 *   y = norm(r) * pre_w + pre_b       (pre = 1)       norm before the next block
 * Post-norm encoders use y alone (pre = 1, post = 0); pre-norm encoders keep r
 * as the residual and feed y to the next block; post = 1 adds the second norm
 * of a sandwich.  All of it is float32 from the rows as read; y is made of the
 * unrounded r.
 *   x, t     [B, n, D] in dtype: residual and block output.  t may be NULL
 *            (r = res_scale * x) without post and gate.
 *   gate     by gate_mode, NULL for SC_GATE_NONE.
 *   post_w, post_b, pre_w, pre_b   float32 [D]; NULL = 1 and 0.
 *   r        [B, n, D] in dtype or NULL; may be x itself (in place).
 *   y        [B, n, D] in dtype or NULL (pre only).
 *   yq, yscale  the rows of y (as stored, in dtype) as sc_quantize_rows_i8
 *            gives them, int8 [B, n, sc_i8_pitch(D)] and float32 [B, n]; both
 *            or neither (pre only).  At least one of r, y and yq.
 * Errors: SC_EINVAL, SC_EUNSUPPORTED (D > 4096, B n >= 2^31).
 */
sc_status sc_block_norm(const sc_norm_desc *desc, const void *x, const void *t, const void *gate,
                        const float *post_w, const float *post_b, const float *pre_w, const float *pre_b, void *r,
                        void *y, int8_t *yq, float *yscale, void *stream);

size_t sc_block_norm_backward_workspace_size(const sc_norm_desc *desc);

/*
 * Gradients of sc_block_norm from dr = dL/dr and dy = dL/dy ([B, n, D] in
 * dtype; either may be NULL, dy is for pre = 1).  The forward's inputs are read
 * again, nothing of it has to be kept.
 *   dx, dt   [B, n, D] in dtype.
 *   dgate    in the gate's own shape and type.
 *   dpost_w, dpost_b, dpre_w, dpre_b   float32 [D].
 * Each output may be NULL (not computed), at least one is not; those of absent
 * parts (gate, norms) must be.  Sums over rows are float32 in a fixed order,
 * without atomics.  Outputs must not overlap each other or the inputs, except
 * that dx may be dr itself and dt may be dy itself.
 * Errors: SC_EINVAL, SC_EUNSUPPORTED, SC_EWORKSPACE.
 */
sc_status sc_block_norm_backward(const sc_norm_desc *desc, const void *x, const void *t, const void *gate,
                                 const float *post_w, const float *post_b, const float *pre_w, const float *pre_b,
                                 const void *dr, const void *dy, void *dx, void *dt, void *dgate, float *dpost_w,
                                 float *dpost_b, float *dpre_w, float *dpre_b, void *workspace, size_t ws_bytes,
                                 void *stream);

/* ---------------------------------------------------------------- stack -- */

/* One 8-bit product of a layer, laid out by sc_quantize_weight_i8. */
typedef struct sc_i8_weight {
  const int8_t *wq;
  const float *scale;
  const float *bias; /* or NULL */
} sc_i8_weight;

/* One layer of sc_encoder_stack_i8 (all pointers to the device). */
typedef struct sc_layer_i8 {
  sc_i8_weight qkv; /* D -> 3 D, columns q | k | v                      */
  sc_i8_weight o;   /* D -> D                                           */
  sc_i8_weight w1;  /* D -> ffn_dim                                     */
  sc_i8_weight w2;  /* ffn_dim -> D                                     */
  const float *gate1, *ln1_w, *ln1_b; /* float32 [D] or NULL: after the attention     */
  const float *gate2, *ln2_w, *ln2_b; /* float32 [D] or NULL: after the feed-forward  */
} sc_layer_i8;

size_t sc_encoder_stack_i8_workspace_size(const sc_attn_desc *desc, int32_t n_layers, int32_t ffn_dim);

/*
 * sc_encoder_stack on 8-bit products, with the parts that a trained encoder
 * has: with lin(w, v) the product of sc_linear_i8 on the rows of v, quantised
 * per token,
 *   qkv = bf16(lin(qkv, x));  O and the pruning as in sc_encoder_stack;
 *   x1  = bf16(LayerNorm(res_scale x + gate1 * bf16(lin(o, O))) ln1_w + ln1_b)
 *   h   = bf16(GELU(lin(w1, x1)))
 *   x   = bf16(LayerNorm(res_scale x1 + gate2 * bf16(lin(w2, h))) ln2_w + ln2_b)
 *   layers  HOST array of n_layers; ffn_dim >= 1; res_scale finite.
 * bf16, not causal, D = H d <= 2048, ffn_dim <= 131072, B <= 8192 and n D <
 * 2^32 / 6, and the limits of sc_linear_i8 for every product, or
 * SC_EUNSUPPORTED.  Every other argument and error as for sc_encoder_stack;
 * x_out rows at or beyond final_len are left untouched, as there.
 */
sc_status sc_encoder_stack_i8(const sc_attn_desc *desc, int32_t n_layers, const int32_t *windows, const void *x_in,
                              const sc_layer_i8 *layers, int32_t ffn_dim, const float *thresholds,
                              int32_t keep_global, float ln_eps, float res_scale, void *x_out, int32_t *final_len,
                              int32_t *orig_idx, int32_t *kept_per_layer, void *workspace, size_t ws_bytes,
                              void *stream);

#ifdef __cplusplus
}
#endif
#endif /* SC_BLOCK_H_ */
