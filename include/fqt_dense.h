/*
 * fqt_dense.h -- the dense operators around the binary layers of libfqt: the RMS norm of a
 * residual sum with 8-bit output, the matrix product with bias, activation and residual in its
 * epilogue, each with its backward pass, and the Newton-Schulz orthogonalisation of a matrix with
 * the optimizer step on latent weights that uses it.
 *
 * fqt.h holds the conventions (device pointers, streams, status codes, no allocation, no
 * synchronisation, host validation before any launch).  In addition:
 *  - A matrix [rows][cols] has unit stride along cols and a row stride `ld` in elements; ld = 0
 *    stands for cols, any other ld must be >= cols and at most FQT_MAX_LD.
 *  - x and w of a product start on 16 bytes, every other matrix and vector on its element size,
 *    workspaces on 256 bytes (FQT_E_ALIGN otherwise).  Operand rows of a
 *    product that are not multiples of 16 bytes long and apart cost a copy, except in a forward of up
 *    to four rows.
 *  - A row or column count of zero is no error: nothing is launched but what an output needs (the
 *    gradient of a parameter over no rows is zero, a product over no columns is its bias).
 *  - Optional pointers may be NULL.  Outputs must not overlap inputs or each other unless a
 *    declaration says that they may.
 *  - Inputs are expected to be finite.  Infinities and NaN stay in the rows (or, in a product, the
 *    rows and columns) that they enter, and a row with one in it gets a scale that is not finite.
 *  - Sums are taken in float32 or wider (int32 for int8 products), in an order that depends only
 *    on the sizes: equal calls give equal bits.
 */
#ifndef FQT_DENSE_H
#define FQT_DENSE_H

#include "fqt.h"

#ifdef __cplusplus
extern "C" {
#endif

/* 8-bit element types, beside FQT_F32 and FQT_BF16: signed integers of -127 ... 127, and the
 * 8-bit float with 4 exponent and 3 mantissa bits (largest value 448, no infinities).  Both come
 * with one float32 scale per row; a code stands for code * scale. */
#define FQT_I8 2
#define FQT_E4M3 3
#define FQT_NO_CODES (-1)

#define FQT_MAX_LD (INT64_C(1) << 22)
#define FQT_MAX_ROWS (INT64_C(1) << 31)   /* rows of any matrix here stay below this */

/* ------------------------------------------------------------------ RMS norm of a residual sum
 *   h = x + residual                       (float32 sum; stored rounded to x_dtype)
 *   rstd = 1 / sqrt(mean over cols of h^2 + eps)
 *   y = h * rstd * g                       (from the unrounded sum; stored rounded to y_dtype)
 *   scale = max over cols of |y| / T       (T = 127 for FQT_I8, 448 for FQT_E4M3)
 *   q = y / scale rounded to nearest even  (0 where scale is 0)
 * The quotient is taken as h g (T / max over cols of |h g|), a few float32 roundings off y / scale, so a tie
 * may go to either neighbour.  h^2 is summed in float32: a row whose sum passes 3.4e38 has rstd, y,
 * scale and q 0.
 * x, residual, h: x_dtype; g [cols]: float32; y: y_dtype; q: q_dtype; scale, rstd: float32 [rows]. */
typedef struct {
  int64_t rows, cols;
  int64_t ldx, ldr, ldh, ldy, ldq;    /* x and dx; residual and dres; h; y and dy; q             */
  int32_t x_dtype, y_dtype;           /* FQT_F32 or FQT_BF16                                     */
  int32_t q_dtype;                    /* FQT_I8, FQT_E4M3 or FQT_NO_CODES                        */
  float eps;                          /* > 0                                                     */
} fqt_norm_desc;

/* residual, h, y, q (with scale), rstd are optional.  h may be x or residual (same ld). */
int fqt_rmsnorm_forward(const fqt_norm_desc *desc, const void *x, const void *residual,
                        const float *g, void *h, void *y, void *q, float *scale, float *rstd,
                        void *hip_stream);

/* Gradients of y for dL/dy, with t = h * rstd and u = dy * g:
 *   dx = rstd * (u - t * mean over cols of u t) + dres      (x_dtype; the gradient of x and of the
 *                                                            residual alike)
 *   dg = sum over rows of dy * t                            (float32 [cols])
 * The codes pass their gradient through (y, not q, is what dy belongs to).  h: x_dtype with ldh;
 * dres: x_dtype, optional, the gradient that reaches h past the norm; dx may be dres.
 * ws: >= fqt_norm_workspace_size bytes, no initialisation. */
int fqt_norm_workspace_size(const fqt_norm_desc *desc, size_t *bytes);
int fqt_rmsnorm_backward(const fqt_norm_desc *desc, const void *h, const float *g,
                         const float *rstd, const void *dy, const void *dres, void *dx, float *dg,
                         void *ws, size_t ws_bytes, void *hip_stream);

/* Codes and scales of the rows of x (a weight matrix, a batch): scale = max |x| / T, q = x / scale
 * rounded to nearest even.  Uses rows, cols, ldx, ldq, x_dtype and q_dtype of desc. */
int fqt_quantize_rows(const fqt_norm_desc *desc, const void *x, void *q, float *scale,
                      void *hip_stream);

/* ------------------------------------------------------------------ product with its epilogue
 *   z[m][n] = x_scale[m] * w_scale[n] * sum over k of x[m][k] w[n][k] + bias[n]
 *   y = act(z) + residual
 * x [M][K] and w [N][K] of x_dtype; the scales (float32 [M], [N]) belong to the 8-bit types and are
 * NULL for FQT_BF16.  bias float32 [N], residual, z, y [M][N] of y_dtype; bias, residual and z are
 * optional.  z is stored rounded; y comes from the unrounded z.  y may be residual (same ld).
 * FQT_I8 sums are exact in int32, so K <= 133144 there; fewer than 2^23 tiles of 256 x 256 cover
 * M x N, M x K and N x K each (FQT_E_SHAPE).  FQT_E4M3 sums have the precision of their matrix instruction, 1e-5 to 6e-5 of their
 * norm, where y is FQT_BF16, and float32's (through bf16 copies of the codes) where it is FQT_F32.  Up to four
 * rows, the form for single tokens, are summed on the vector units, in float32 for every type. */
#define FQT_ACT_NONE 0
#define FQT_ACT_RELU 1
#define FQT_ACT_GELU 2                    /* z * Phi(z), Phi the normal distribution
                                           * function, to 2.5e-7               */
#define FQT_ACT_SILU 3                    /* z / (1 + exp(-z))                     */
#define FQT_ACT_HARDTANH 4                /* z clamped to [-1, 1]                  */
typedef struct {
  int64_t M, N, K;
  int64_t ldx, ldw, ldr, ldy, ldz;    /* ldy: y and dy                                           */
  int64_t lddx, lddw;
  int32_t x_dtype;                    /* x and w: FQT_BF16, FQT_I8 or FQT_E4M3                    */
  int32_t y_dtype;                    /* y, residual, z, dy: FQT_F32 or FQT_BF16                  */
  int32_t dx_dtype, dw_dtype;         /* FQT_F32 or FQT_BF16                                      */
  int32_t act;
} fqt_linear_desc;

/* How a call lays out a matrix product, from its sizes alone (nothing is launched): the edge of the
 * output tiles and the workgroups of each launch (a second one takes the last tiles in smaller ones),
 * and the pieces that the contraction is split into.  No launches: the sizes take a form without
 * tiles (forwards of up to four rows, orthogonalisations of up to 64). */
typedef struct {
  int32_t launches, splits;
  int32_t tile[2], threads[2];
  int64_t workgroups[2];
} fqt_product_plan;
#define FQT_PRODUCT_FORWARD 0
#define FQT_PRODUCT_DX 1
#define FQT_PRODUCT_DW 2
int fqt_linear_plan(const fqt_linear_desc *desc, int32_t product, fqt_product_plan *plan);

int fqt_linear_workspace_size(const fqt_linear_desc *desc, int32_t backward, size_t *bytes);
int fqt_linear_forward(const fqt_linear_desc *desc, const void *x, const void *w,
                       const float *x_scale, const float *w_scale, const float *bias,
                       const void *residual, void *z, void *y, void *ws, size_t ws_bytes,
                       void *hip_stream);

/* Gradients for dy = dL/dy (the residual's is dy itself), with dz = dy * act'(z) in float32:
 *   dx[m][k] = sum over n of dz[m][n] w_scale[n] w[n][k]
 *   dw[n][k] = sum over m of dz[m][n] x_scale[m] x[m][k]   (the gradient of w_scale[n] w[n][k])
 *   dbias[n] = sum over m of dz[m][n]                       (float32)
 * z: the pre-activation that the forward stored, required unless act is FQT_ACT_NONE.  act' is 0
 * at the corners of relu and hardtanh.  dx, dw, dbias are optional, each given one is computed.
 * The matrix cores take dz (times w_scale or x_scale) rounded once to bf16; 8-bit codes are exact in
 * bf16.  ws: >= fqt_linear_workspace_size(desc, 1) bytes. */
int fqt_linear_backward(const fqt_linear_desc *desc, const void *x, const void *w,
                        const float *x_scale, const float *w_scale, const void *z, const void *dy,
                        void *dx, void *dw, float *dbias, void *ws, size_t ws_bytes,
                        void *hip_stream);

/* ------------------------------------------------------------------ orthogonalised update
 *   X_0 = u / (|u| + eps)                      (Frobenius norm, summed in float64)
 *   X_{i+1} = a X_i + (b P + c P^2) X_i,  P = X_i X_i^T,  (a, b, c) = (3.4445, -4.7750, 2.0315)
 * taken on the short side of u; steps of them bring the singular values of u near 1.  The products
 * run on the 16-bit matrix cores from operands split in two (22 bits and their rounding), with
 * float32 sums: results as from float32 products.  The shorter side is at most 65536, rows times cols
 * (in eights) below 2^34 (FQT_E_SHAPE otherwise). */
typedef struct {
  int64_t rows, cols;
  int64_t ldg, ldo, ldm;              /* g; o and w; m                                           */
  int32_t g_dtype, o_dtype;           /* FQT_F32 or FQT_BF16 (fqt_muon_step: o_dtype FQT_F32)    */
  int32_t steps;                      /* 1 ... 32                                                */
  float eps;                          /* > 0                                                     */
} fqt_ortho_desc;

/* The step of an optimizer that orthogonalises its momentum:
 *   m = momentum * m + g;  u = nesterov ? g + momentum * m : m;
 *   w = (1 - lr * weight_decay) * w - lr * scale * X_steps(u). */
typedef struct {
  float lr, momentum, weight_decay, scale;
  int32_t nesterov;
} fqt_muon_cfg;

/* The plans of P = X X^T, of b P + c P^2 (both symmetric) and of its product with X. */
#define FQT_PRODUCT_GRAM 0
#define FQT_PRODUCT_POLY 1
#define FQT_PRODUCT_APPLY 2
int fqt_ortho_plan(const fqt_ortho_desc *desc, int32_t product, fqt_product_plan *plan);
int fqt_ortho_workspace_size(const fqt_ortho_desc *desc, size_t *bytes);
/* o = X_steps(g).  o may be g where both have one type and stride. */
int fqt_orthogonalize(const fqt_ortho_desc *desc, const void *g, void *o, void *ws,
                      size_t ws_bytes, void *hip_stream);
/* w and m (float32) are updated in place. */
int fqt_muon_step(const fqt_ortho_desc *desc, const fqt_muon_cfg *cfg, const void *g, float *m,
                  float *w, void *ws, size_t ws_bytes, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* FQT_DENSE_H */
