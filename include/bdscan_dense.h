/*
 * bdscan_dense.h -- the dense operators either side of the mixers of BDLM
 * Mamba-H (arXiv 2607.02805) on NVIDIA GB300 (sm_103a):
 *   - the linear layer with bias, activation and residual in one product (the
 *     MLP of a block, Appendix C: ratio 4; the projections around a mixer; the
 *     logits of single tokens), forward and backward;
 *   - the gated linear layer: both projections of a gated feed-forward block,
 *     the activation and the product in one, forward and backward;
 *   - the weighted softmax cross entropy of the language-model head over the
 *     vocabulary (the masked objective, Sec. 3; Sec. 4.1), at the rows that
 *     count, without keeping the logits, forward and backward;
 *   - the distillation loss: how far the head's distribution is from a
 *     teacher's, of which the likeliest entries are known, the same way;
 *   - token scores of given logits: log probabilities of tokens, entropies and
 *     the likeliest entries (what a denoising step chooses its tokens by, and
 *     what a teacher hands on), forward and backward.
 * The products run on the tcgen05 tensor cores (bf16 operands, fp32 accumulation in
 * TMEM); fp32 inputs are computed to fp32 accuracy from three bf16 pieces per
 * value.
 *
 * Conventions of bdscan.h: device pointers, 16-byte aligned, caller-owned
 * memory with a caller workspace (sizes from the *_workspace_size queries; a
 * query that returns 0 for valid dims needs none, and the workspace may then
 * be NULL), asynchronous on `stream`, gradients overwritten, return codes and
 * bdscan_last_error(). An output that shares memory with an input is refused
 * where the two are not one operand computed in place, said so below; columns
 * side by side in a wider buffer share none. (Not checked by the linear
 * layer's and the vocabulary loss's backward and the loss's forward.) A wait on tensor-core work that gives up sets the flag
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

/* y = act(x wg^T + bg) * (x wu^T + bu), elementwise product.
 * Layouts: x [rows][d_in] (row stride ld_x), w [2 d_hidden][d_in]: the rows of
 * wg, then those of wu; bias [2 d_hidden] likewise (nullable), y
 * [rows][d_hidden] (row stride ld_y). All have `dtype` (f32 or bf16). Sums,
 * activation and product are fp32, y is rounded once. rows >= 0, d_in and
 * d_hidden >= 1. */
typedef struct bdscan_gated_linear_dims {
  int64_t rows;
  int64_t d_in;
  int64_t d_hidden;
  int64_t ld_x;
  int64_t ld_y; /* of y, and of dy in the backward */
  int32_t act;  /* BDSCAN_ACT_* */
  int32_t dtype;
} bdscan_gated_linear_dims;

size_t bdscan_gated_linear_forward_workspace_size(const bdscan_gated_linear_dims* dims);
int bdscan_gated_linear_forward(const bdscan_gated_linear_dims* dims, const void* x, const void* w, const void* bias,
                                void* y, void* workspace, size_t workspace_bytes, void* stream);

/* Gradients of <dy, y>: with g = x wg^T + bg and u = x wu^T + bu, computed
 * again, dz = [dy u act'(g), dy act(g)] [rows][2 d_hidden], dx = dz w
 * [rows][d_in], dw = dz^T x [2 d_hidden][d_in], dbias = column sums of dz
 * [2 d_hidden]. Each of dx, dw, dbias is nullable and then not computed; bias
 * is the forward's. dz enters the products rounded to `dtype` (fp32: three
 * pieces), and dbias unrounded. */
size_t bdscan_gated_linear_backward_workspace_size(const bdscan_gated_linear_dims* dims);
int bdscan_gated_linear_backward(const bdscan_gated_linear_dims* dims, const void* x, const void* w, const void* bias,
                                 const void* dy, void* dx, void* dw, void* dbias, void* workspace,
                                 size_t workspace_bytes, void* stream);

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

/* loss[t] = weight[t] sum_v q_tv (log q_tv - log p_tv), the divergence of the
 * student's p_t = softmax(h w^T / temperature) over the whole vocabulary from the
 * teacher's q_t = softmax(teacher[t] / temperature) over the row's known entries:
 * those whose id is inside 0 .. vocab - 1 and not `excluded`, with a teacher's
 * logit above minus infinity. An id that comes twice has both shares.
 * lse[t] = log sum_v exp(z[t][v] / temperature). A row counts where its weight is
 * not zero and an entry is known; the others get loss = lse = 0 and no gradient,
 * whatever h holds there, and cost no product. `excluded` as in the vocabulary
 * loss.
 * Layouts: h, w, weight, loss, lse, dloss as in the vocabulary loss; ids
 * [rows][top] int64, teacher [rows][top] fp32, top 1 .. 64; z [rows][top] fp32
 * receives h w^T at the known entries of the rows that count, else 0, which the
 * backward reads. temperature 2^-20 .. 2^20. */
typedef struct bdscan_distill_loss_dims {
  int64_t rows;
  int64_t d_model;
  int64_t vocab;
  int64_t ld_h;
  int64_t excluded;
  int32_t top;
  int32_t dtype;
  float temperature;
} bdscan_distill_loss_dims;

/* weight is nullable (ones). */
size_t bdscan_distill_loss_forward_workspace_size(const bdscan_distill_loss_dims* dims);
int bdscan_distill_loss_forward(const bdscan_distill_loss_dims* dims, const void* h, const void* w, const int64_t* ids,
                                const float* teacher, const float* weight, float* loss, float* lse, float* z,
                                void* workspace, size_t workspace_bytes, void* stream);

/* Gradients of <dloss, loss> (dloss nullable: ones) with respect to h
 * [rows][d_model] and w [vocab][d_model], of `dtype`, as in the vocabulary loss
 * with p - q at the logits, over the temperature. lse and z are the forward's. */
size_t bdscan_distill_loss_backward_workspace_size(const bdscan_distill_loss_dims* dims);
int bdscan_distill_loss_backward(const bdscan_distill_loss_dims* dims, const void* h, const void* w,
                                 const int64_t* ids, const float* teacher, const float* weight, const float* lse,
                                 const float* z, const float* dloss, void* dh, void* dw, void* workspace,
                                 size_t workspace_bytes, void* stream);

/* Scores of rows of logits z, with p = softmax(z / temperature):
 *   logp[t] = log p[token[t]],  entropy[t] = -sum_v p_v log p_v,
 *   top_ids, top_logp [rows][top]: the `top` entries of the largest
 *   probability, largest first, of equal logits the lower index first, and
 *   their log probabilities.
 * `excluded` names an entry of probability zero, whatever its logit (-1: none);
 * a logit of minus infinity is one too. Such entries are never among the
 * likeliest (places left over hold -1 and minus infinity), and as a token have
 * logp minus infinity. A row without any other entry has entropy 0, no likeliest
 * entries and no gradient. A row whose token is outside 0 .. vocab - 1 does not
 * count: its logits are not read, logp, entropy and gradient are 0, and it has
 * no likeliest entries. A row with NaN or plus infinity at an entry that
 * is not excluded has NaN everywhere and -1 for the likeliest entries.
 * Layouts: logits [rows][vocab] (row stride ld_logits) and dlogits (ld_dlogits)
 * of `dtype` (f32 or bf16); token [rows] int64; stats [rows][2]: the largest
 * logit and the logarithm of the sum of exponentials relative to it, which the
 * backward reads (minus infinity first: no gradient). Everything else fp32,
 * top_ids int64. top 0 .. 64, temperature 2^-20 .. 2^20. No workspace. */
typedef struct bdscan_token_scores_dims {
  int64_t rows;
  int64_t vocab;
  int64_t ld_logits;
  int64_t ld_dlogits;
  int64_t excluded;
  int32_t top;
  int32_t dtype;
  float temperature;
} bdscan_token_scores_dims;

/* token and logp are nullable together, entropy and stats each, top_ids and
 * top_logp where top is 0. */
int bdscan_token_scores_forward(const bdscan_token_scores_dims* dims, const void* logits, const int64_t* token,
                                float* logp, float* entropy, float* stats, int64_t* top_ids, float* top_logp,
                                void* stream);

/* dlogits: gradient of <dlogp, logp> + <dentropy, entropy> at the logits. dlogp
 * and dentropy are nullable (zero); token is the forward's, nullable where dlogp
 * is; stats and entropy (read where dentropy is given) are the forward's.
 * dlogits may be the logits themselves; another stride is then refused. */
int bdscan_token_scores_backward(const bdscan_token_scores_dims* dims, const void* logits, const int64_t* token,
                                 const float* stats, const float* entropy, const float* dlogp, const float* dentropy,
                                 void* dlogits, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* BDSCAN_DENSE_H */
