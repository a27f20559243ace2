/*
 * acdc_train.h -- C ABI of the operators on either side of a cascade's
 * forward and backward pass (acdc.h) in a training step: losses that turn
 * rows of logits (a cascade's y) into a gradient (its grad_y), and the
 * optimiser's step that turns parameter gradients into new parameters.
 *
 * Every pointer is a device pointer on the current HIP device unless stated
 * otherwise; every call is enqueued on the given stream without host
 * synchronisation; nothing is allocated.  Checks run on the host before any
 * HIP call, and on error nothing is launched.  Status codes, their strings
 * and acdc_last_hip_error are those of acdc.h.  Results are bitwise
 * reproducible on one device: sums run in a fixed order, without atomics.
 * Sums, softmax statistics and moments are held in 32 bits or more.
 *
 * Logits.  rows x classes values of type `dtype`, row r at logits + r *
 * stride (in elements, stride >= classes), so that the first classes
 * columns of wider rows can be read in place.  Pointers need the alignment
 * of their element only.  targets: one class per row, int32 or int64
 * (target_bits 32 or 64).  A negative target marks a row that takes no part:
 * its logits do not matter and may hold anything, its outputs are 0 and its
 * gradient is written as 0.  A target >= classes gives NaN for its row.
 * Logits of -inf are classes of probability 0; a row that has only such
 * classes has no distribution and gives NaN, as does one that holds NaN or
 * +inf.  grad_logits has rows grad_stride apart and the logits' dtype; it
 * may be the logits' own memory (same pointer and stride) or other columns of
 * the same wider rows (same stride), otherwise it must not overlap them.
 */
#ifndef ACDC_TRAIN_H_
#define ACDC_TRAIN_H_

#include "acdc.h"

#ifdef __cplusplus
extern "C" {
#endif

enum acdc_dtype { ACDC_F32 = 0, ACDC_BF16 = 1 };

/* ------------------------------------------------------------- the losses */

/* Per row, with M = max_j x_j, S = sum_j exp(x_j - M), p_j = exp(x_j - M) / S:
 *   logp    = x_t - M - log S                      log-probability of the target t
 *   entropy = log S - sum_j p_j (x_j - M)          H (optional, may be null)
 *   saved   = (M, S, H, logp), [rows][4] float     for acdc_logprob_backward (optional) */
int acdc_logprob_forward(const void* logits, int32_t dtype, int64_t stride, const void* targets, int32_t target_bits,
                         int64_t rows, int32_t classes, float* logp, float* entropy, float* saved, void* workspace,
                         size_t workspace_bytes, acdc_stream_t stream);
size_t acdc_logprob_workspace_size(int64_t rows, int32_t classes, int32_t dtype);

/* dL/dx_j = c (g ([j = t] - p_j) - h p_j (log p_j + H)) for each row, with
 * g = grad_logp[r] = dL/dlogp, h = grad_entropy[r] = dL/dH (may be null: 0)
 * and c = *scale (device, may be null: 1).  `saved` as acdc_logprob_forward or
 * a loss below filled it for the same logits and targets.  A row with
 * g = h = 0 gets zeros. */
int acdc_logprob_backward(const void* logits, int32_t dtype, int64_t stride, const void* targets, int32_t target_bits,
                          const float* saved, const float* grad_logp, const float* grad_entropy, const float* scale,
                          void* grad_logits, int64_t grad_stride, int64_t rows, int32_t classes,
                          acdc_stream_t stream);

/* Clipped policy loss with a KL term and an entropy bonus.  Per row with
 * ratio = exp(logp - logp_old), advantage a, k = logp_ref - logp:
 *   policy = -min(ratio a, clamp(ratio, 1 - clip_low, 1 + clip_high) a)
 *   kl     = exp(k) - k - 1
 *   loss   = policy + kl_coef kl - entropy_coef H
 * and the total sum_r w_r loss_r / W, W = sum_r w_r (with mean = 0: not
 * divided).  weights >= 0 (null: 1 each); a row of weight 0 takes no part,
 * like one with a negative target.  W = 0 gives a loss and gradients of 0.
 * logp_ref may be null when kl_coef = 0 (kl is then 0); where it is given all the
 * same, it serves the stats alone.
 *
 * stats, 6 floats: the total, and the weighted sums (means with mean != 0) of
 * policy, kl, H, the share of rows whose ratio was clipped away, and ratio.
 * logp [rows].  Optional (may be null):
 *   grad_logits  grad_scale * dL/dlogits
 *   saved        as in acdc_logprob_forward, with
 *   row_grads    [2][rows]: dL/dlogp and dL/dH (without grad_scale), what
 *                acdc_logprob_backward takes. */
typedef struct acdc_policy_params {
  float clip_low, clip_high, kl_coef, entropy_coef, grad_scale;
  int32_t mean;
} acdc_policy_params;
int acdc_policy_loss(const void* logits, int32_t dtype, int64_t stride, const void* targets, int32_t target_bits,
                     const float* logp_old, const float* logp_ref, const float* advantages, const float* weights,
                     int64_t rows, int32_t classes, const acdc_policy_params* params /* host */, float* stats,
                     float* logp, void* grad_logits, int64_t grad_stride, float* saved, float* row_grads,
                     void* workspace, size_t workspace_bytes, acdc_stream_t stream);
size_t acdc_policy_workspace_size(int64_t rows, int32_t classes, int32_t dtype);

/* Preference loss over pairs of sequences.  Sequence s is the rows
 * offsets[s] .. offsets[s+1] - 1 (offset_bits 32 or 64; 2 * pairs + 1
 * non-decreasing values in 0 .. rows); sequence 2p is the preferred one of
 * pair p and 2p + 1 the other.  With the reference's log-probabilities
 * logp_ref [rows] of the same targets:
 *   reward_s = beta sum of (logp - logp_ref) over the sequence's rows with a target
 *   margin_p = reward_2p - reward_2p+1
 *   loss     = mean over pairs of -(1 - e) log sigmoid(margin) - e log sigmoid(-margin)
 * with label smoothing e.  An empty sequence has reward 0.  Rows outside
 * every sequence get a zero gradient; offsets outside 0 .. rows are clamped.
 *
 * stats, 5 floats: loss, share of pairs with margin > 0, mean margin, mean
 * reward of the preferred and of the other sequences.  The rest as in
 * acdc_policy_loss. */
typedef struct acdc_preference_params {
  float beta, label_smoothing, grad_scale;
} acdc_preference_params;
int acdc_preference_loss(const void* logits, int32_t dtype, int64_t stride, const void* targets, int32_t target_bits,
                         const void* offsets, int32_t offset_bits, const float* logp_ref, int64_t rows,
                         int32_t classes, int64_t pairs, const acdc_preference_params* params /* host */,
                         float* stats, float* logp, void* grad_logits, int64_t grad_stride, float* saved,
                         float* row_grads, void* workspace, size_t workspace_bytes, acdc_stream_t stream);
size_t acdc_preference_workspace_size(int64_t rows, int32_t classes, int32_t dtype, int64_t pairs);

/* ---------------------------------------------------------- the optimiser */

/* One tensor of an AdamW step: n contiguous elements (0 <= n < 2^34 - 1024).
 * Moments in 32 bits (m_scale = v_scale = null): m and v are float [n].
 * Moments in 8 bits: m and v are codes, uint8 [n], each an OCP e4m3 value q;
 * elements 256 b .. 256 b + 255 share the scales m_scale[b] and v_scale[b]
 * (ceil(n / 256) floats each): m = q m_scale, sqrt(v) = q v_scale.  A scale is
 * the block's largest magnitude / 448, so that the largest element keeps its
 * value and the block follows its decay; a positive v never becomes 0.  A NaN or
 * infinite moment is a NaN code and does not count for its block's scale.
 * Pointers need the alignment of their element only. */
typedef struct acdc_adamw_tensor {
  void* param;        /* param_type */
  float* master;      /* float copy that is updated and rounded into param; null: param itself (BF16 only) */
  const void* grad;   /* grad_type */
  void *m, *v;
  float *m_scale, *v_scale;
  int64_t n;
  float lr, weight_decay;
  int32_t param_type, grad_type; /* enum acdc_dtype */
} acdc_adamw_tensor;

/* For every tensor, with g = grad * *grad_scale (device float, may be null: 1):
 *   m = beta1 m + (1 - beta1) g,  v = beta2 v + (1 - beta2) g^2
 *   w = w (1 - lr weight_decay) - lr m / (1 - beta1^step) / (sqrt(v / (1 - beta2^step)) + eps)
 * in 32 bits, w the master or the parameter; step counts from 1.  A grad_scale
 * that is not finite, or is -0, leaves every tensor as it is: what acdc_grad_norm
 * gives for gradients that hold a NaN or an infinity.  `tensors` is a host array
 * that is read before the call returns; no two tensors may overlap.  Its numbers
 * and step travel in the launches' arguments: captured into a graph, every replay
 * is the step that was captured, with its lr and its bias correction. */
int acdc_adamw_step(const acdc_adamw_tensor* tensors, int32_t count, double beta1, double beta2, double eps,
                    int64_t step, const float* grad_scale, acdc_stream_t stream);

/* out[0] = 2-norm of all gradients together, out[1] = min(1, max_norm /
 * (out[0] + 1e-6)), or 1 with max_norm <= 0 (no clipping): a grad_scale for
 * acdc_adamw_step.  The norm is computed in 64 bits, as is the quotient.  An
 * infinite gradient gives inf and -0, a NaN gives NaN twice, so that the step
 * with that scale changes nothing (with 1, without clipping, it spoils the
 * elements in question).  `grads`, `sizes`, `types` are host arrays of `count`. */
int acdc_grad_norm(const void* const* grads, const int64_t* sizes, const int32_t* types, int32_t count,
                   float max_norm, float* out, void* workspace, size_t workspace_bytes, acdc_stream_t stream);
size_t acdc_grad_norm_workspace_size(const int64_t* sizes, int32_t count);

#ifdef __cplusplus
}
#endif

#endif /* ACDC_TRAIN_H_ */
