/*
 * fqt_step.h -- what stands between the last layer of a network and its updated weights: the softmax
 * cross entropy of a linear layer's outputs without keeping them, with its gradients, the norm of all
 * gradients, and AdamW over all tensors of a model with states in float32 or in 8 bits.
 *
 * fqt.h and fqt_dense.h hold the conventions (device pointers, streams, status codes, matrices with a row
 * stride, 8-bit operands with a scale for each row, workspaces on 256 bytes, no allocation, no
 * synchronisation, host validation before any launch, sums in an order that depends only on the sizes:
 * equal calls give equal bits).
 */
#ifndef FQT_STEP_H
#define FQT_STEP_H

#include "fqt_dense.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ------------------------------------------------------------------ loss of a linear layer
 *   z[m][n] = x_scale[m] * w_scale[n] * sum over k of x[m][k] w[n][k] + bias[n]
 *   lse[m]  = log of the sum over n of exp(z[m][n])
 *   loss[m] = lse[m] - (1 - smoothing) z[m][target[m]] - smoothing * mean over n of z[m][n]
 * z is never stored as a matrix of M x N (of up to four rows, or where its contraction is split, it passes
 * through the workspace).  x [M][K] and w [N][K] of x_dtype; the scales (float32 [M], [N]) belong to the
 * 8-bit types and are NULL for FQT_BF16; bias float32 [N], optional; target int64 [M]; loss and lse float32
 * [M].  Row m is left out where target[m] is `ignore`: its loss is 0, its lse as ever.  Any other target that
 * is no class makes the row's loss NaN, and its gradients (nothing outside the arrays is read for it).  A
 * bias of minus infinity takes a class out (not with smoothing, whose mean is over all).  The loss holds its relative precision also where it is
 * small (the largest z is left out of the sum that is added to it).
 * mean, float32 [2], optional: the mean loss over the rows that count, and 1 / their number; both 0 if none
 * does.
 * Sums are exact in int32 for FQT_I8 (K <= 133144), float32 otherwise (of FQT_E4M3 too: the matrix cores take
 * its codes widened to bf16).  N >= 1; sizes as in fqt_linear_forward. */
typedef struct {
  int64_t M, N, K;                    /* rows, classes, features                                 */
  int64_t ldx, ldw, lddx, lddw;
  int64_t ignore;                     /* target of the rows that are left out                    */
  int32_t x_dtype;                    /* x and w: FQT_BF16, FQT_I8 or FQT_E4M3                   */
  int32_t dx_dtype, dw_dtype;         /* FQT_F32 or FQT_BF16                                     */
  float smoothing;                    /* 0 ... 1                                                 */
} fqt_loss_desc;

int fqt_loss_workspace_size(const fqt_loss_desc *desc, int32_t backward, size_t *bytes);
int fqt_loss_forward(const fqt_loss_desc *desc, const void *x, const void *w, const float *x_scale,
                     const float *w_scale, const float *bias, const int64_t *target, float *loss,
                     float *lse, float *mean, void *ws, size_t ws_bytes, void *hip_stream);

/* Gradients, with z computed again in pieces of the classes (dz of a piece lies in the workspace in bf16, twice for the 8-bit
 * types: about 256 MB, or 4096 classes of all rows where that is more; up to 5120 classes are one piece):
 *   dz[m][n] = c[m] (exp(z[m][n] - lse[m]) - (1 - smoothing) [n = target[m]] - smoothing / N)
 *   dx[m][k] = sum over n of dz[m][n] w_scale[n] w[n][k]
 *   dw[n][k] = sum over m of dz[m][n] x_scale[m] x[m][k]   (the gradient of w_scale[n] w[n][k])
 *   dbias[n] = sum over m of dz[m][n]                       (float32)
 * c is dloss[m] (float32 [M], the gradient of each row's loss) or dmean[0] * mean[1] (dmean float32 [1],
 * the gradient of the forward's mean; mean as the forward left it): one of the two is given, the other
 * is NULL.  dz is 0 in rows that are left out, whatever z is there; but x has to be finite there too for dw
 * (0 times infinity).  dx, dw, dbias are optional, each given one is computed.  The matrix cores take dz
 * (times w_scale or x_scale) rounded once to bf16, and sum in float32; dbias sums it unrounded.
 * At a target whose probability is over 1/2 dz is c (expm1(log p) + smoothing - smoothing / N), with log p = z - lse from a z
 * summed in float64: p - 1 keeps its precision relative to itself for the lse that is given.  But an lse in float32 is
 * itself off by 2^-25 of its size, which is more than p - 1 of a well fitted row: the functions below pass log p on. */
int fqt_loss_backward(const fqt_loss_desc *desc, const void *x, const void *w, const float *x_scale,
                      const float *w_scale, const float *bias, const int64_t *target,
                      const float *lse, const float *dloss, const float *dmean, const float *mean,
                      void *dx, void *dw, float *dbias, void *ws, size_t ws_bytes,
                      void *hip_stream);

/* The same with log p of the targets, float32 [M], which the forward leaves (0 in rows that are left out, NaN where the
 * target is no class) and the backward takes instead of computing it: gradients of rows whose loss is small then
 * keep the relative precision that the loss has.  logp NULL: as the functions above. */
int fqt_loss_forward_logp(const fqt_loss_desc *desc, const void *x, const void *w, const float *x_scale,
                          const float *w_scale, const float *bias, const int64_t *target, float *loss,
                          float *lse, float *logp, float *mean, void *ws, size_t ws_bytes, void *hip_stream);
int fqt_loss_backward_logp(const fqt_loss_desc *desc, const void *x, const void *w, const float *x_scale,
                           const float *w_scale, const float *bias, const int64_t *target,
                           const float *lse, const float *logp, const float *dloss, const float *dmean,
                           const float *mean, void *dx, void *dw, float *dbias, void *ws, size_t ws_bytes,
                           void *hip_stream);

/* ------------------------------------------------------------------ lists of tensors
 * One tensor of a list, n contiguous elements.  Lists are read by the host during the call: they may
 * change or go afterwards, also when the call was captured into a graph.  Tensors must not overlap. */
typedef struct {
  const void *g;                      /* gradient, g_dtype                                       */
  float *p;                           /* weight                                                  */
  void *m, *v;                        /* states: float32, or e4m3 codes (a byte each)            */
  float *m_scale, *v_scale;           /* of 8-bit states: float32 [ceil(n / FQT_STATE_BLOCK)]    */
  int64_t n;
  int64_t first;                      /* its place in the random sequence, a multiple of 4       */
  int32_t g_dtype;                    /* FQT_F32 or FQT_BF16                                     */
} fqt_param;
#define FQT_STATE_BLOCK 256
#define FQT_MAX_PARAMS 65536          /* tensors of a list                                       */

/* out[0] = the norm of all gradients, sqrt of the sum of g^2 over all tensors (summed in float64);
 * out[1] = min(1, max_norm / (out[0] + 1e-6)), what clipping multiplies them by.  out: float32 [2].  A norm
 * that is not finite shows in out: infinity gives the factor 0, NaN is NaN.  max_norm > 0, infinity for no
 * clipping.  Uses g, n and g_dtype of the list. */
int fqt_grad_norm_workspace_size(const fqt_param *params, int32_t count, size_t *bytes);
int fqt_grad_norm(const fqt_param *params, int32_t count, float max_norm, float *out, void *ws,
                  size_t ws_bytes, void *hip_stream);

/* A step of AdamW, for every element of every tensor, with s = grad_scale[0] (1 if NULL) and t = step:
 *   m = beta1 m + (1 - beta1) s g;  v = beta2 v + (1 - beta2) (s g)^2
 *   p = p - lr weight_decay p - lr / (1 - beta1^t) * m / (sqrt(v / (1 - beta2^t)) + eps)
 * in float32, the factors in float64.  t is `step`, or *step_dev (device memory, read as the kernel runs: for
 * captured graphs) where that is given; t >= 1 (a smaller *step_dev counts as 1).  With eps = 0 an element whose m and v
 * are 0 becomes NaN; so does one whose gradient is infinite, also where s is 0.
 *
 * States of 8 bits (state_dtype FQT_E4M3): m and sqrt(v) are held as e4m3 codes, with one float32 scale for
 * each block of FQT_STATE_BLOCK elements of a tensor: scale = max of the block / 448, and a code stands for
 * code * scale.  p is updated from the float32 values; what is stored is rounded stochastically: down to a code
 * plus, with the probability of the remainder, one step, so that slow averages move as they should where
 * rounding to nearest would hold them.  sqrt(v) > 0 never becomes 0 (the smallest code instead), since
 * its m may not.  A block whose maximum is below 2^-100 is stored as zeros.  A value that is not finite
 * makes its block's scale so, and with the next step the block.
 * The random bits are those of Philox4x32-10 with the key `seed` and the counter
 * ((first + i) / 4 (64 bits, 3 << 30 in the upper word), 0, t modulo 2^32): word (first + i) % 4 belongs to element i, its lower
 * 16 bits to m, the upper to v. */
typedef struct {
  double lr, beta1, beta2, eps, weight_decay;   /* lr, eps, weight_decay and lr weight_decay 0 ... 1e30, 0 <= beta < 1 */
  uint64_t seed;
  int32_t state_dtype;                          /* FQT_F32 or FQT_E4M3                              */
} fqt_adamw_cfg;
int fqt_adamw_step(const fqt_adamw_cfg *cfg, const fqt_param *params, int32_t count, int64_t step,
                   const int64_t *step_dev, const float *grad_scale, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* FQT_STEP_H */
