/*
 * libonebitlamb -- the operators of a layer in 8 bits and of the flat gradient: the root-mean-square norm with the residual's
 * addition, the product of 8-bit matrices with a scale for each block of 128, and the gradient's norm with its clipping, as
 * hand-written HIP kernels for gfx950 (MI355X).  They work on the same flat buffers as onebitlamb.h and ob_matrix.h: weights may
 * lie in the parameters (or their 16-bit copy) that those steps write, weight gradients go into the flat gradient that they
 * read, and the gradient is clipped before them.
 *
 * Conventions, as in ob_matrix.h: device pointers are the caller's; every call validates its arguments on the host, enqueues
 * kernels on `hip_stream`, allocates nothing and returns without synchronising.  On error nothing is enqueued and a negative
 * ob_status is returned.  A context owns its workspace, on the device that was current at its creation (calls made with another
 * device current return OB_ERR_ARG); calls on one context must not overlap in time.  Pointers and the distances between rows may
 * be any multiple of the element's size unless a call says otherwise.  Results are reproducible from run to run: sums have one
 * order for given sizes.  An output may not overlap an input unless a call says otherwise.
 */
#ifndef OB_LAYER_H
#define OB_LAYER_H

#include "onebitlamb.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- numbers of 8 bits with a scale for each block of 128 -----------------------------------------------------------
 *
 * A matrix [rows, columns] is held as one byte a number, row r at data + r * ld, and a scale for each 128 columns of a row, or
 * of 128 rows (form OB_BLOCK_SQUARE): the byte scales[r * ld_scales + c / 128] (r / 128 for squares), a power of two
 * 2^(byte - 127) (E8M0), 255 for a NaN.  Its values are number times scale.  ld is a multiple of 128 and data lies at a multiple of
 * 16 bytes; the bytes of a row from `columns` up to the next multiple of 128 are zeros (every call here that writes such a matrix writes them).
 * ld_scales is a multiple of 4, and scales lie at a multiple of 4 bytes.
 *
 * A scale is the smallest power of two, from 2^-126 on, by which the block's largest magnitude is no more than the format's
 * largest number (448 or 57344), so that dividing by it rounds nothing and the matrix cores apply it themselves; the quotient is
 * rounded to nearest, ties to even.  A block with an infinity or a NaN is NaNs throughout.
 */
enum { OB_E4M3 = 0, /* 1.4.3, no infinities, largest 448 */
       OB_E5M2 = 1  /* 1.5.2, largest 57344 */ };
enum { OB_BLOCK_ROWS = 0, OB_BLOCK_SQUARE = 1 };

/* ---- root-mean-square norm with the residual's addition ---------------------------------------------------------------
 *
 *   forward    h = x + residual, rounded to h's type (or h = x, with residual NULL)
 *              rstd = 1 / sqrt(mean over the row of h^2 + eps)
 *              y = h rstd weight, rounded to x's type, and / or to 8 bits
 *   backward   g = dy weight, xhat = h rstd
 *              dh = dres + rstd (g - xhat mean(g xhat))          (dres NULL: 0), rounded to h's type
 *              dweight = sum over rows of dy xhat                 (+= with accumulate)
 * on rows of n numbers, in binary32, with y and xhat those of the rounded h.  Squares are summed in binary64 where their sum leaves binary32's
 * range, so that rows of any finite numbers have their norm.  dh is the gradient of x and of the residual.  A row of zeros with eps = 0 gives
 * NaNs, and one with a root mean square below 2^-128 an rstd, and numbers, of infinity; a row with an infinity has rstd 0, zeros, and a NaN where
 * the infinity was; one with a NaN gives NaNs.
 */
typedef struct ob_norm_ctx ob_norm_ctx; /* opaque */

typedef struct ob_norm_config {
  int64_t n;            /* 1 .. 16384 */
  int32_t dtype;        /* ob_dtype of x, y, dy */
  int32_t res_dtype;    /* of residual, h, dres, dh: dtype or OB_F32 */
  int32_t weight_dtype; /* of weight: any */
  float eps;            /* >= 0, finite */
} ob_norm_config;

ob_status ob_norm_create(const ob_norm_config* cfg, ob_norm_ctx** out);
void ob_norm_destroy(ob_norm_ctx* ctx);
size_t ob_norm_workspace_bytes(const ob_norm_ctx* ctx);
const char* ob_norm_last_hip_error(const ob_norm_ctx* ctx);

/* x [rows, n], residual and h [rows, n], y [rows, n], with rows ldx, ldr, ldh, ldy >= n elements apart (below 2^31; rows up to
 * 2^31 - 1); weight [n] or NULL (ones); rstd [rows] binary32, or NULL.  residual NULL: h is not written, and may be NULL.  h may be
 * residual itself, or x if their types are one (the same address and distance between rows).  y NULL: only in 8 bits; data NULL: not in 8 bits. */
ob_status ob_norm_forward(ob_norm_ctx* ctx, const void* x, int64_t ldx, const void* residual, int64_t ldr, const void* weight,
                          int64_t rows, void* h, int64_t ldh, void* y, int64_t ldy, void* data, int64_t ld, void* scales,
                          int64_t ld_scales, int32_t format, float* rstd, void* hip_stream);
/* h (x's own rows where there was no residual, if their types are one), rstd as forward left them.  dh [rows, n] or NULL, which may be dres
 * itself (or dy, if their types are one); dweight [n] binary32 or NULL. */
ob_status ob_norm_backward(ob_norm_ctx* ctx, const void* dy, int64_t lddy, const void* h, int64_t ldh, const float* rstd,
                           const void* weight, const void* dres, int64_t lddres, int64_t rows, void* dh, int64_t lddh, float* dweight,
                           int32_t accumulate, void* hip_stream);

/* ---- linear layer in 8 bits -------------------------------------------------------------------------------------------
 *
 *   forward      y [rows, n]  = x W^T          x [rows, k], W [n, k]
 *   input_grad   dx [rows, k] = dy W           dy [rows, n], with W's transpose [k, n]
 *   weight_grad  dW [n, k]    = dy^T x  (+=)    with the transposes of dy and x, [n, rows] and [k, rows]
 * Operands are matrices of 8 bits with scales as above: W in squares and e4m3, the transpose of x in e4m3, x and dy in either
 * format, with the scales of rows.  Products are summed in binary32 and each result is rounded once:
 *   OB_F32          exact products (an error of 7e-8 over a matrix of normal numbers, 8192 deep) of numbers, scale applied, from 2^-133 to below 2^128:
 *                   of all in a block whose scale is 2^-124 or more in e4m3, 2^-117 in e5m2.  Smaller numbers lose bits, or are zeros, and what is
 *                   2^128 in 8 bits is an infinity
 *   OB_F16, OB_BF16 at twice the rate: of eight adjacent products each is cut off 13 bits below the largest power of two among
 *                   them before they are summed, 1.5e-5 over such a matrix, where the result's rounding makes 2e-4 or 1.7e-3
 * quantize makes any of the operands, a matrix and its transpose in one pass.
 */
typedef struct ob_linear8_ctx ob_linear8_ctx; /* opaque */

typedef struct ob_linear8_config {
  int64_t k, n;      /* 1 .. 2^20 each */
  int64_t max_rows;  /* largest `rows` of a call: 0 .. 2^22 */
} ob_linear8_config;

ob_status ob_linear8_create(const ob_linear8_config* cfg, ob_linear8_ctx** out);
void ob_linear8_destroy(ob_linear8_ctx* ctx);
size_t ob_linear8_workspace_bytes(const ob_linear8_ctx* ctx);
const char* ob_linear8_last_hip_error(const ob_linear8_ctx* ctx);

/* src [rows, cols] of src_dtype, rows lds >= cols elements apart (below 2^22; rows and cols up to 2^22) -> data [rows, cols], with
 * scales, and / or data_t [cols, rows], with scales_t; a pointer NULL: not wanted.  `form` OB_BLOCK_SQUARE: both have the same scales,
 * of 128 x 128. */
ob_status ob_linear8_quantize(ob_linear8_ctx* ctx, const void* src, ob_dtype src_dtype, int64_t lds, int64_t rows, int64_t cols,
                              int32_t form, int32_t format, int32_t format_t, void* data, int64_t ld, void* scales, int64_t ld_scales,
                              void* data_t, int64_t ld_t, void* scales_t, int64_t ld_scales_t, void* hip_stream);
/* w, w_scales: [n, k]; w_t, w_t_scales of input_grad: its transpose [k, n].  Results are OB_F32, OB_F16 or OB_BF16. */
ob_status ob_linear8_forward(ob_linear8_ctx* ctx, const void* x, int64_t ldx, const void* x_scales, int64_t ldx_scales, int32_t x_format,
                             const void* w, int64_t ldw, const void* w_scales, int64_t ldw_scales, int64_t rows, void* y, int64_t ldy,
                             ob_dtype y_dtype, void* hip_stream);
/* forward of up to OB_LINEAR8_FEW_ROWS rows (more: OB_ERR_SIZE) from x itself, of x_dtype with rows ldx >= k elements apart: its numbers are made 8
 * bits of x_format on the way, the same as quantize makes.  For one trip to memory where rows are few or short; 16 long rows, and any
 * of 16384 numbers, are faster by the two calls. */
enum { OB_LINEAR8_FEW_ROWS = 16 };
ob_status ob_linear8_forward_few(ob_linear8_ctx* ctx, const void* x, ob_dtype x_dtype, int64_t ldx, int32_t x_format, const void* w, int64_t ldw,
                                 const void* w_scales, int64_t ldw_scales, int64_t rows, void* y, int64_t ldy, ob_dtype y_dtype, void* hip_stream);
ob_status ob_linear8_input_grad(ob_linear8_ctx* ctx, const void* dy, int64_t lddy, const void* dy_scales, int64_t lddy_scales, int32_t dy_format,
                                const void* w_t, int64_t ldw_t, const void* w_t_scales, int64_t ldw_t_scales, int64_t rows, void* dx,
                                int64_t lddx, ob_dtype dx_dtype, void* hip_stream);
/* dy_t [n, rows], x_t [k, rows], dw [n, k] with rows lddw >= k elements apart.  accumulate != 0: OB_F32 only. */
ob_status ob_linear8_weight_grad(ob_linear8_ctx* ctx, const void* dy_t, int64_t lddy_t, const void* dy_t_scales, int64_t lddy_t_scales,
                                 int32_t dy_format, const void* x_t, int64_t ldx_t, const void* x_t_scales, int64_t ldx_t_scales, int64_t rows,
                                 void* dw, int64_t lddw, ob_dtype dw_dtype, int32_t accumulate, void* hip_stream);

/* ---- norm of the flat gradient, and clipping ----------------------------------------------------------------------------
 *
 * A flat gradient of a list of tensors as in ob_lamb_config: layer_offsets [num_layers + 1], tightly packed (tensors may be empty).
 *   norm   layer_norms[l] = grad_scale ||g_l||_2, norm = grad_scale ||g||_2      squares summed in binary64, rounded once
 *   apply  out = g f, f = grad_scale min(1, max_norm / (norm + eps)) in binary32: norm is read on the device, formed by `norm` or
 *          elsewhere (for instance summed over ranks).  out == g with the same type: in place, and if f is 1 nothing is written.
 * A norm that is NaN makes every f NaN; an infinite one, which finite gradients have where theirs is beyond binary32, makes it 0 (finite
 * gradients become 0, others NaN), unless max_norm is infinite too.
 */
typedef struct ob_clip_ctx ob_clip_ctx; /* opaque */

typedef struct ob_clip_config {
  int64_t num_layers;            /* 1 .. 2^22 */
  const int64_t* layer_offsets;  /* HOST, copied; up to 2^35 elements */
  float eps;                     /* >= 0, finite */
  float grad_scale;              /* > 0, finite: the inverse loss scale */
} ob_clip_config;

ob_status ob_clip_create(const ob_clip_config* cfg, ob_clip_ctx** out);
void ob_clip_destroy(ob_clip_ctx* ctx);
size_t ob_clip_workspace_bytes(const ob_clip_ctx* ctx);
const char* ob_clip_last_hip_error(const ob_clip_ctx* ctx);

/* norm [1], layer_norms [num_layers] or NULL: binary32 on the device.  max_norm >= 0 (infinite: no clipping). */
ob_status ob_clip_norm(ob_clip_ctx* ctx, const void* grad, ob_dtype grad_dtype, float* norm, float* layer_norms, void* hip_stream);
ob_status ob_clip_apply(ob_clip_ctx* ctx, const void* grad, ob_dtype grad_dtype, const float* norm, float max_norm, void* out,
                        ob_dtype out_dtype, void* hip_stream);
/* both, one after the other, in fewer launches */
ob_status ob_clip_norm_apply(ob_clip_ctx* ctx, const void* grad, ob_dtype grad_dtype, float max_norm, float* norm, float* layer_norms,
                             void* out, ob_dtype out_dtype, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif
