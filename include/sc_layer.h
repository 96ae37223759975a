/*
 * sc_layer.h - what a present-day encoder layer has beside its attention (sc.h)
 * and its block norms (sc_block.h), for serving and for training:
 *
 *   sc_rotary           rotary positions on queries and keys, with their norms per
 *                       head in the same pass, from the fused q|k|v rows of a
 *                       projection to the dense q, k, v of sc_window_attention;
 *   sc_rotary_backward  its gradients;
 *   sc_rotary_frequencies  the angles per position, scaled for long contexts;
 *   sc_gated_ffn        the gated feed-forward block y = (act(x Wg) * (x Wu)) Wd;
 *   sc_gated_ffn_backward  its gradients;
 *   sc_dropout          dropout with a residual sum, its mask made anew from a
 *                       counter wherever it is needed and never stored.
 *
 * The conventions of sc.h and sc_block.h hold: device tensors owned by the
 * caller, scratch memory from `workspace`, everything enqueued on `stream`
 * without synchronisation or allocation (all calls may be captured into a
 * graph), arguments checked on the host before anything is enqueued, no state
 * kept between calls.  Rows come as a padded batch: sequence b of B holds
 * valid_len[b] of n rows (device int32 [B]; values outside [0, n] are clamped),
 * or n without valid_len (NULL).  Output rows of padding are zero, and padding
 * rows of inputs are not read into any result.  Every result is deterministic.
 */
#ifndef SC_LAYER_H_
#define SC_LAYER_H_

#include "sc_block.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ------------------------------------------------------ rotary positions -- */

#define SC_ROTARY_HALF 0        /* pair i: dimensions i and i + rot_dim / 2 */
#define SC_ROTARY_INTERLEAVED 1 /* pair i: dimensions 2 i and 2 i + 1       */

#define SC_ROTARY_PLAIN 0  /* f_i = base^(-2 i / rot_dim)                                      */
#define SC_ROTARY_LINEAR 1 /* f_i / factor: positions interpolated                             */
#define SC_ROTARY_BASE 2   /* base * factor^(rot_dim / (rot_dim - 2)) in the place of base     */
#define SC_ROTARY_BANDS 3  /* by the turns t_i = f_i length / (2 pi) that a pair makes over the
                              length trained on: f_i where t_i >= fast, f_i / factor where
                              t_i <= slow, in between (linearly in t_i) a mixture of both;
                              amplitude 0.1 ln(factor) + 1                                     */

/*
 * Host: the angle per position of each pair, freq [rot_dim / 2], and the factor
 * on the rotated dimensions, *amplitude (1 but for SC_ROTARY_BANDS).
 *   base > 1; factor >= 1 (not read for SC_ROTARY_PLAIN); length >= 1 and
 *   fast > slow >= 0 for SC_ROTARY_BANDS (else not read); SC_ROTARY_BASE of one
 *   pair (rot_dim 2) is SC_ROTARY_PLAIN.
 * Errors: SC_EINVAL (null pointers, values not finite or outside the above,
 * rot_dim odd or below 2), SC_EUNSUPPORTED (rot_dim > 256).
 */
sc_status sc_rotary_frequencies(int32_t rot_dim, double base, int32_t scaling, double factor, double length,
                                double fast, double slow, double *freq, float *amplitude);

typedef struct sc_rotary_desc {
  int32_t B, n;             /* rows as above                                         */
  int32_t Hq, Hk, d;        /* query heads, key (and value) heads, size of a head: d even, 2 <= d <= 256 */
  const int32_t *valid_len; /* device int32 [B], or NULL                             */
  int32_t rot_dim;          /* dimensions rotated, the first of each head: even, 0 <= rot_dim <= d */
  int32_t layout;           /* SC_ROTARY_HALF or SC_ROTARY_INTERLEAVED               */
  int32_t norm;             /* 0 or 1: heads of q and k are normalised first         */
  int32_t kind;             /* SC_NORM_* of that norm                                */
  float eps;                /* > 0 (with norm)                                       */
  float amplitude;          /* finite: factor on the rotated dimensions              */
  int32_t dtype;            /* SC_F32 or SC_BF16: of all heads and gradients         */
  int64_t q_stride, k_stride, v_stride; /* elements between the tokens of q, k, v (and of dq, dk, dv) */
} sc_rotary_desc;

/*
 * For every token at position p and every head x of its queries and keys
 *   u = norm ? norm(x) * w : x                    over the d dimensions of the head
 *   (a, b) -> amplitude (a cos p f_i - b sin p f_i, a sin p f_i + b cos p f_i)
 * for the pairs (a, b) of u, pair i with frequency f_i; dimensions from rot_dim
 * on stay u.  Values are copied.  Float32 from the heads as read, rounded once;
 * angles are right to 2^-27 of a turn at any 32-bit position.
 *   freq     HOST float64 [rot_dim / 2], |f_i| < 2^20, read in the call (NULL
 *            without rot_dim).
 *   q, k, v  head h of token (b, j) at (b n + j) stride + h d: dense (stride =
 *            heads * d) or parts of fused rows.  k and v may be NULL.
 *   q_w, k_w float32 [d] or NULL (1), with norm only.
 *   positions  int32 [B, n] (e.g. the original positions orig_idx of a pruned
 *            batch), any value; NULL: j.
 *   q_out, k_out, v_out  dense [B, n, heads, d]; NULL where the input is.  An
 *            output may be its dense input (in place).
 * Errors: SC_EINVAL (null pointers, sizes, types, values as above, strides below
 * heads * d, overlaps), SC_EUNSUPPORTED (d > 256, B n >= 2^31, Hq + 2 Hk >= 2^15).
 */
sc_status sc_rotary(const sc_rotary_desc *desc, const double *freq, const void *q, const void *k, const void *v,
                    const float *q_w, const float *k_w, const int32_t *positions, void *q_out, void *k_out,
                    void *v_out, void *stream);

size_t sc_rotary_backward_workspace_size(const sc_rotary_desc *desc);

/*
 * Gradients of sc_rotary from those of its outputs, dense [B, n, heads, d].
 * The forward's inputs are read again (with norm), nothing of it has to be kept.
 *   dq_out, dk_out, dv_out  each with the gradient that it leads to, or NULL.
 *   q, k     as for sc_rotary, needed with norm for the parts asked for (not
 *            read without).
 *   dq, dk, dv  laid out as q, k, v (strides of desc), so that they may be parts
 *            of one fused row; only these parts are written.  At least one.
 *            Each may be its dense dq_out, dk_out, dv_out (in place).
 *   dq_w, dk_w  float32 [d], or NULL; with norm, and with dq, dk.  Sums over
 *            tokens and heads are float32 in a fixed order, without atomics.
 *   workspace  needed for dq_w or dk_w only; 16-byte aligned.
 * Errors: as sc_rotary, and SC_EWORKSPACE.
 */
sc_status sc_rotary_backward(const sc_rotary_desc *desc, const double *freq, const void *dq_out, const void *dk_out,
                             const void *dv_out, const void *q, const void *k, const float *q_w, const float *k_w,
                             const int32_t *positions, void *dq, void *dk, void *dv, float *dq_w, float *dk_w,
                             void *workspace, size_t ws_bytes, void *stream);

/* ----------------------------------------------------- gated feed-forward -- */

#define SC_ACT_SILU 2 /* v / (1 + exp(-v)) (beside SC_ACT_NONE and SC_ACT_GELU) */

typedef struct sc_ffn_desc {
  int32_t B, n, D, F;       /* rows as above, D channels, F gated channels   */
  const int32_t *valid_len; /* device int32 [B], or NULL                     */
  int32_t act;              /* SC_ACT_*                                      */
  int32_t dtype;            /* SC_BF16: of all tensors                       */
} sc_ffn_desc;

size_t sc_gated_ffn_workspace_size(const sc_ffn_desc *desc, int32_t save);

/* Bytes of what the backward needs of the forward, of the valid rows: h, and
 * act(g) and u act'(g) rounded to 24 bits, in a layout private to the library. */
size_t sc_gated_ffn_saved_size(const sc_ffn_desc *desc);

/*
 * The gated feed-forward block, per row,
 *   g = x . Wg, u = x . Wu;  h = bf16(act(g) * u);  y = bf16(h . Wd)
 * with float32 sums and activations.
 *   x, y     bf16 [B, n, D].   Wg, Wu  bf16 [D, F];  Wd  bf16 [F, D] (row-major).
 *   saved    sc_gated_ffn_saved_size() bytes for sc_gated_ffn_backward, or NULL.
 *   workspace  sc_gated_ffn_workspace_size(desc, saved != NULL) bytes.
 * Tensors, saved and workspace are aligned to 16 bytes.  A row's result does not
 * depend on the other rows' values or on valid_len; the order of its sums goes by
 * the sizes and, where B n <= 128, by whether `saved` is given too (y with and
 * without it may then differ in a rounding).
 * Errors: SC_EINVAL (null pointers, sizes, types, alignment, y, saved or
 * workspace overlapping anything), SC_EUNSUPPORTED (dtype SC_F32; B n >= 2^31;
 * with valid_len, B > 8192; tensors of 4 GiB: with D and F rounded up to 8,
 * 2 B n D, 2 B n F or 2 D F >= 2^32 - 4096), SC_EWORKSPACE.
 */
sc_status sc_gated_ffn(const sc_ffn_desc *desc, const void *x, const void *wg, const void *wu, const void *wd, void *y,
                       void *saved, void *workspace, size_t ws_bytes, void *stream);

size_t sc_gated_ffn_backward_workspace_size(const sc_ffn_desc *desc);

/*
 * Gradients of sc_gated_ffn from dy = dL/dy, bf16 [B, n, D]:
 *   dh = dy . Wd^T,  dg = bf16(dh (u act'(g))),  du = bf16(dh act(g)),
 *   dx = bf16(dg . Wg^T + du . Wu^T),
 *   dwg = bf16(x^T . dg),  dwu = bf16(x^T . du),  dwd = bf16(h^T . dy),
 * sums in float32 and in a fixed order, over rows too.
 *   saved    as the forward of the same desc, inputs and lengths left it (read
 *            only: any number of calls).
 *   dx  bf16 [B, n, D];  dwg, dwu  bf16 [D, F];  dwd  bf16 [F, D]; each may be
 *            NULL (not computed), at least one is not.
 * Alignment and errors as for sc_gated_ffn; outputs must not overlap each other,
 * the inputs or the workspace.
 */
sc_status sc_gated_ffn_backward(const sc_ffn_desc *desc, const void *x, const void *wg, const void *wu, const void *wd,
                                const void *saved, const void *dy, void *dx, void *dwg, void *dwu, void *dwd,
                                void *workspace, size_t ws_bytes, void *stream);

/* ---------------------------------------------------------------- dropout -- */

typedef struct sc_dropout_desc {
  int32_t B, n, D;          /* rows as above, D channels                           */
  const int32_t *valid_len; /* device int32 [B], or NULL                           */
  double p;                 /* 0 <= p, share that is dropped, to 2^-16 (below)     */
  float res_scale;          /* finite: of the residual                             */
  int32_t site;             /* number of this place in the model: its own mask     */
  int32_t dtype;            /* SC_F32 or SC_BF16                                   */
} sc_dropout_desc;

/*
 *   out = res_scale * residual + (r >= t ? x * 65536 / (65536 - t) : 0)
 * with t = p * 65536 rounded to an integer (halves to even; t <= 65535), float32
 * from the rows as read.  r are 16-bit random numbers of Philox4x32-10 (Salmon,
 * Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011): its
 * key is *seed (low word first), its counter (c / 8, j, b, site) for channel c
 * of row j of sequence b; the four words it gives, low half before high half,
 * are the r of channels 8 (c / 8) to 8 (c / 8) + 7.  The mask is a function of
 * these numbers alone: the gradient of x is the same call on the gradient of out
 * without the residual (that of the residual is res_scale times it), and a
 * token's mask depends neither on n, D or dtype nor on the batch.
 *   x, out     [B, n, D] in dtype; out may be x or residual (in place).
 *   residual   [B, n, D] in dtype, or NULL (0).
 *   seed       device int64 [1], 8-byte aligned: a captured graph draws new masks
 *              once the program writes another seed there.
 * A dropped element is 0 whatever x is, an infinity or a NaN too.
 * Errors: SC_EINVAL (null pointers, sizes, types, p not in [0, 65535.5 / 65536),
 * overlaps), SC_EUNSUPPORTED (B n >= 2^31).
 */
sc_status sc_dropout(const sc_dropout_desc *desc, const void *x, const int64_t *seed, const void *residual, void *out,
                     void *stream);

#ifdef __cplusplus
}
#endif
#endif /* SC_LAYER_H_ */
