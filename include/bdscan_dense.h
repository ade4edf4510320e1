/*
 * bdscan_dense.h -- the dense operators either side of the mixers of BDLM
 * Mamba-H (arXiv 2607.02805) on NVIDIA GB300 (sm_103a):
 *   - the linear layer with bias, activation and residual in one product (the
 *     MLP of a block, Appendix C: ratio 4; the projections around a mixer; the
 *     logits of single tokens), forward and backward;
 *   - the weighted softmax cross entropy of the language-model head over the
 *     vocabulary (the masked objective, Sec. 3; Sec. 4.1), at the rows that
 *     count, without keeping the logits, forward and backward.
 * Both run on the tcgen05 tensor cores (bf16 operands, fp32 accumulation in
 * TMEM); fp32 inputs are computed to fp32 accuracy from three bf16 pieces per
 * value.
 *
 * Conventions of bdscan.h: device pointers, 16-byte aligned, caller-owned
 * memory with a caller workspace (sizes from the *_workspace_size queries; a
 * query that returns 0 for valid dims needs none, and the workspace may then
 * be NULL), asynchronous on `stream`, gradients overwritten, return codes and
 * bdscan_last_error(). A wait on tensor-core work that gives up sets the flag
 * of bdscan_ssd_wait_flag(). Calls need the driver's tensor-map encoder and
 * return BDSCAN_ERR_UNSUPPORTED without it. A value that is not finite makes
 * every output that reads it non-finite (with fp32 inputs: NaN where the exact
 * value is infinite).
 */
#ifndef BDSCAN_DENSE_H
#define BDSCAN_DENSE_H

#include <stddef.h>
#include <stdint.h>

#include "bdscan.h"

#ifdef __cplusplus
extern "C" {
#endif

#define BDSCAN_ACT_NONE 0
#define BDSCAN_ACT_SILU 1 /* z / (1 + exp(-z)) */
#define BDSCAN_ACT_GELU 2 /* z (1 + tanh(sqrt(2/pi) (z + 0.044715 z^3))) / 2 */

/* y = residual + act(x w^T + bias).
 * Layouts: x [rows][d_in] (row stride ld_x), w [d_out][d_in], bias [d_out],
 * residual [rows][d_out] (row stride ld_res), y [rows][d_out] (row stride
 * ld_y). Strides are in elements, 0 stands for the row length.
 * Types: x, w, bias, pre and the gradients have `dtype`; y, residual and dy
 * have `out_dtype`: (f32,f32), (bf16,bf16) or (bf16,f32). Sums are fp32 and
 * rounded once. Any sizes: rows >= 0, d_in and d_out >= 1. */
typedef struct bdscan_linear_dims {
  int64_t rows;
  int64_t d_in;
  int64_t d_out;
  int64_t ld_x;
  int64_t ld_res;
  int64_t ld_y; /* of y, and of dy in the backward */
  int32_t act;  /* BDSCAN_ACT_* */
  int32_t dtype;
  int32_t out_dtype;
} bdscan_linear_dims;

/* bias, residual and pre are nullable. pre [rows][d_out] receives x w^T + bias
 * (before the activation, rounded to `dtype`), which the backward of an
 * activation reads. y may be the residual itself (same stride), no other
 * input. */
size_t bdscan_linear_forward_workspace_size(const bdscan_linear_dims* dims);
int bdscan_linear_forward(const bdscan_linear_dims* dims, const void* x, const void* w, const void* bias,
                          const void* residual, void* pre, void* y, void* workspace, size_t workspace_bytes,
                          void* stream);

/* Gradients of <dy, y>: with dz = dy act'(pre), dx = dz w [rows][d_in],
 * dw = dz^T x [d_out][d_in], dbias = column sums of dz [d_out] (the residual's
 * gradient is dy itself). Each of dx, dw, dbias is nullable and then not
 * computed. pre is not read (nullable) without an activation. dz enters the
 * two products rounded to `dtype` (fp32: three pieces), and dbias unrounded. */
size_t bdscan_linear_backward_workspace_size(const bdscan_linear_dims* dims);
int bdscan_linear_backward(const bdscan_linear_dims* dims, const void* x, const void* w, const void* pre,
                           const void* dy, void* dx, void* dw, void* dbias, void* workspace, size_t workspace_bytes,
                           void* stream);

/* loss[t] = weight[t] (lse[t] - z[t][target[t]]), lse[t] = log sum_v exp(z[t][v]),
 * z = h w^T, at the rows that count: target inside 0 .. vocab - 1 and weight
 * not zero. The others (the tokens that a masked objective left visible,
 * padding) get loss = lse = 0 and no gradient, whatever h holds there, and
 * cost no product.
 * `excluded` names a vocabulary entry whose probability is zero (the mask
 * token, which a denoiser never predicts): its logit counts as minus infinity
 * and its row of w gets no gradient; -1 for none. A row whose target is the
 * excluded entry has loss +infinity (times its weight).
 * Layouts: h [rows][d_model] (row stride ld_h, 0: d_model), w [vocab][d_model],
 * both of `dtype` (f32 or bf16); target [rows] int64; weight, loss, lse,
 * dloss [rows] fp32. */
typedef struct bdscan_lm_loss_dims {
  int64_t rows;
  int64_t d_model;
  int64_t vocab;
  int64_t ld_h;
  int64_t excluded;
  int32_t dtype;
} bdscan_lm_loss_dims;

/* weight is nullable (ones). */
size_t bdscan_lm_loss_forward_workspace_size(const bdscan_lm_loss_dims* dims);
int bdscan_lm_loss_forward(const bdscan_lm_loss_dims* dims, const void* h, const void* w, const int64_t* target,
                           const float* weight, float* loss, float* lse, void* workspace, size_t workspace_bytes,
                           void* stream);

/* Gradients of <dloss, loss> (dloss nullable: ones) with respect to h
 * [rows][d_model] and w [vocab][d_model], of `dtype`. lse is the forward's. The
 * logits are computed again, in pieces of the vocabulary whose gradient (rounded
 * to `dtype`; fp32: three pieces) the workspace holds, 512 MiB at most (256 entries at
 * least). The product for dw reads h times weight and dloss, rounded likewise. */
size_t bdscan_lm_loss_backward_workspace_size(const bdscan_lm_loss_dims* dims);
int bdscan_lm_loss_backward(const bdscan_lm_loss_dims* dims, const void* h, const void* w, const int64_t* target,
                            const float* weight, const float* lse, const float* dloss, void* dh, void* dw,
                            void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* BDSCAN_DENSE_H */
