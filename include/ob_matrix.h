/*
 * libonebitlamb -- the operators on matrices: the products of an expert layer, whose rows are grouped by expert, and the
 * orthogonalised update (Newton-Schulz products over the matrices of a flat list of tensors), as hand-written HIP kernels
 * for gfx950 (MI355X).  They work on the same flat buffers as onebitlamb.h: expert weights may lie in the 16-bit copy of the
 * parameters that its calls write, and their gradients go into the flat gradient that its calls read.
 *
 * Conventions, as there: device pointers are the caller's; every call validates its arguments on the host, enqueues kernels
 * on `hip_stream` (a hipStream_t passed as void*; NULL = the default stream), allocates nothing and returns without
 * synchronising.  On error nothing is enqueued and a negative ob_status is returned.  A context owns its workspace, on the
 * device that was current at its creation (calls made with another device current return OB_ERR_ARG); calls on one context
 * must not overlap in time.  Unlike there, tensors may start at any multiple of their element's size: they are as
 * densely packed as the flat list (OB_ERR_ALIGN only for a pointer that is no multiple of its element's size); rows that
 * start at multiples of 16 bytes are faster.
 */
#ifndef OB_MATRIX_H
#define OB_MATRIX_H

#include "onebitlamb.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- products of an expert layer ----------------------------------------------------------------------------------
 *
 * Rows are sorted by group (expert): group g has the rows offsets[g] <= r < offsets[g + 1] of x [rows, k] and y [rows, n].
 *   forward      y[r]  = x[r] W_g                for every row r of group g
 *   input_grad   dx[r] = dy[r] W_g^T
 *   weight_grad  dW_g  = x_g^T dy_g              (or dW_g += ...)
 * Operands are binary16 or bfloat16, products are summed in binary32, and each result is rounded once.
 * `offsets` [num_groups + 1] lies on the device and is not read by the host.  It has to be non-decreasing with values from
 * 0 to rows; values outside are brought into that range and a group that would end before it starts is empty (nothing is
 * read or written out of bounds; for a table that is not non-decreasing the results are not defined).  Groups may be empty:
 * forward and input_grad have nothing to do for them, and weight_grad writes zeros (or adds nothing).  Rows below
 * offsets[0] or from offsets[num_groups] on belong to no group: they are not read and what would be their results is not written.
 * Results are reproducible from run to run: sums have one order for given sizes and offsets.
 */
typedef struct ob_experts_ctx ob_experts_ctx; /* opaque */

enum { OB_EXPERTS_KN = 0, /* W_g is [k, n], rows of n */
       OB_EXPERTS_NK = 1  /* W_g is [n, k], rows of k */ };

typedef struct ob_experts_config {
  int32_t num_groups; /* 1 .. 65536 */
  int32_t dtype;      /* ob_dtype of x, dy and W: OB_F16 or OB_BF16 */
  int32_t w_layout;   /* OB_EXPERTS_KN or OB_EXPERTS_NK, of W and dW */
  int32_t reserved;   /* 0 */
  int64_t k, n;       /* 1 .. 2^20 each */
  int64_t max_rows;   /* largest `rows` of a call: 0 .. 2^26 */
  int64_t w_stride;   /* elements from W_g to W_(g+1), and from dW_g to dW_(g+1); >= k * n, or 0 for k * n */
} ob_experts_config;

ob_status ob_experts_create(const ob_experts_config* cfg, ob_experts_ctx** out);
void ob_experts_destroy(ob_experts_ctx* ctx);
size_t ob_experts_workspace_bytes(const ob_experts_ctx* ctx);
const char* ob_experts_last_hip_error(const ob_experts_ctx* ctx);

/* x [rows, k] with rows ldx >= k elements apart, y [rows, n] with ldy >= n (both below 2^22).  y_dtype / dx_dtype: the
 * configuration's dtype, or OB_F32.  An output may not overlap an input. */
ob_status ob_experts_forward(ob_experts_ctx* ctx, const void* x, int64_t ldx, const void* w, const int32_t* offsets,
                             int64_t rows, void* y, int64_t ldy, ob_dtype y_dtype, void* hip_stream);
ob_status ob_experts_input_grad(ob_experts_ctx* ctx, const void* dy, int64_t lddy, const void* w, const int32_t* offsets,
                                int64_t rows, void* dx, int64_t lddx, ob_dtype dx_dtype, void* hip_stream);
/* dw in the layout and stride of W; dw_dtype: the configuration's dtype or OB_F32.  accumulate != 0 adds to what dw holds
 * (OB_F32 only: a 16-bit sum would round at every call). */
ob_status ob_experts_weight_grad(ob_experts_ctx* ctx, const void* x, int64_t ldx, const void* dy, int64_t lddy,
                                 const int32_t* offsets, int64_t rows, void* dw, ob_dtype dw_dtype, int32_t accumulate,
                                 void* hip_stream);

/* ---- orthogonalised update --------------------------------------------------------------------------------------
 *
 * A list of tensors as in ob_lamb_config: layer_offsets [num_layers + 1], tightly packed, in flat buffers of
 * layer_offsets[num_layers] elements.  layer_rows[l] = 0 leaves tensor l out (vectors, embeddings: nothing of it is read or
 * written by these calls); otherwise it is a row-major matrix of layer_rows[l] rows, which must divide its size.
 *
 * orthogonalize: for each matrix G, with m <= n its smaller and larger side (a matrix of more rows than columns is taken
 * transposed),
 *     X = G / (||G||_F + eps),     `steps` times  X <- a X + (b S + c S S) X,  S = X X^T,
 * that is, each singular value s becomes p(p(..p(s))) of s / (||G||_F + eps), p(s) = a s + b s^3 + c s^5, and the
 * singular vectors stay.
 *
 * step: for each matrix, with element-wise binary32 operations in this order, one rounding each,
 *     m <- beta m + (1 - beta) (grad_scale g)
 *     u  = nesterov ? beta m + (1 - beta) (grad_scale g) : m
 *     x <- x (1 - lr weight_decay) - (lr layer_scale) O(u),    O as above
 * where 1 - beta is that of the binary32 number beta (0.05000001 for 0.95), as in the LAMB steps.
 * grad == NULL: m is taken as it is, formed elsewhere (for instance by ob_lamb_momentum_dense from the 1-bit momentum), and u = m.
 *
 * precision: the products are made of binary16 numbers and summed in binary32.
 *   OB_F32  every operand is a sum of two binary16 numbers (22 bits): 1e-6 to 3e-6 relative in the 2-norm over a matrix of normal
 *           numbers, 2e-5 at low numerical rank, about what binary32 products in the plain order make of them.  The numbers have
 *           fixed units, below which they lose digits: rows that are 1e-4, 1e-5 and 1e-6 of the others come out 5e-6, 5e-5 and
 *           5e-4 off themselves in a 64 x 200 matrix, up to 3e-3 in larger ones (binary32 products: 3e-7 to 2e-6), and a matrix whose norm
 *           is far below eps loses digits as a whole (1e-5 to 1e-4 off at a norm of 1.6e-12 with eps 1e-7, 1e-2 at 1e-14)
 *   OB_F16  X is a sum of two, S and the polynomial's matrix are one (11 bits): 1e-3 to 2e-3 relative in the 2-norm over the
 *           matrix, for matrices of low numerical rank as well; meant for 16-bit outputs.  Square matrices take 0.6 of OB_F32's
 *           time, a BERT-Large- or GPT-shaped list 0.75, lists whose matrices are all [3 m, m] or wider 0.8, small ones the same:
 *           wide matrices of large lists, and lists of no more than 64 x 512, are computed with 22 bits in both
 * Norms and the binary32 state are the same in both.
 * A matrix with an infinity or a NaN gives NaNs, and one with singular values that the polynomial takes beyond 3.9 may (from a
 * number beyond the working matrices' range: 3.9 where S is followed, near 16 otherwise, and which of the two a matrix takes goes by
 * the whole list's sizes); other matrices of the list are not touched by that.  A matrix of zeros gives zeros (eps > 0).
 */
typedef struct ob_muon_ctx ob_muon_ctx; /* opaque */

typedef struct ob_muon_config {
  int64_t num_layers;            /* >= 1 */
  const int64_t* layer_offsets;  /* HOST, copied */
  const int64_t* layer_rows;     /* HOST [num_layers], copied; at least one is not 0 */
  const float* layer_scale;      /* HOST [num_layers], copied; NULL: 0.2 sqrt(max(rows, columns)) */
  const float* coefficients;     /* HOST [3 * num_coefficients], copied: a, b, c of each step, the last ones for all that
                                    follow; |a| + |b| + |c| <= 100 */
  int32_t num_coefficients;      /* 1 .. steps */
  int32_t steps;                 /* 1 .. 64 */
  float eps;                     /* >= 0 */
  float beta;                    /* 0 <= beta < 1 */
  float weight_decay;            /* >= 0 */
  int32_t nesterov;
  int32_t precision;             /* OB_F32 or OB_F16 */
} ob_muon_config;

ob_status ob_muon_create(const ob_muon_config* cfg, ob_muon_ctx** out);
void ob_muon_destroy(ob_muon_ctx* ctx);
size_t ob_muon_workspace_bytes(const ob_muon_ctx* ctx);
const char* ob_muon_last_hip_error(const ob_muon_ctx* ctx);

/* src and out: flat buffers in the list's layout, of any ob_dtype each; they may not overlap. */
ob_status ob_muon_orthogonalize(ob_muon_ctx* ctx, const void* src, ob_dtype src_dtype, void* out, ob_dtype out_dtype,
                                void* hip_stream);

/* x, m: flat binary32 buffers.  grad (or NULL) of grad_dtype; grad_scale as in ob_lamb_compress_local_lp, used for
 * every grad_dtype.  x_lp: NULL, or a flat buffer of x_dtype (OB_F16, OB_BF16) that receives the rounded parameters of
 * the matrices.  No buffer may overlap another. */
ob_status ob_muon_step(ob_muon_ctx* ctx, float* x, float* m, const void* grad, ob_dtype grad_dtype, float grad_scale,
                       float lr, void* x_lp, ob_dtype x_dtype, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif
