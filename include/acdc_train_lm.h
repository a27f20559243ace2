/*
 * acdc_train_lm.h -- C ABI of the operators that make a language model of a
 * cascade (acdc.h): the way from tokens to rows, the normalisation of rows,
 * and a loss over a vocabulary that is wider than a row.
 *
 * Pointers, streams, checks, status codes and reproducibility are those of
 * acdc_train.h: device pointers unless stated otherwise, work enqueued without
 * host synchronisation, nothing allocated, everything checked on the host
 * before the first launch, sums in a fixed order and without atomics on
 * values.  An output overlaps no input and no other output, unless stated
 * otherwise, and the workspace none of them.  A workspace belongs to one call
 * at a time.
 */
#ifndef ACDC_TRAIN_LM_H_
#define ACDC_TRAIN_LM_H_

#include "acdc_train.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ------------------------------------------------- the vocabulary's losses
 *
 * Logits x_rv = sum_k hidden[r][k] weight[v][k] that are never stored as a
 * whole: they are computed in pieces of the vocabulary, and for the gradient
 * once more.  Per row with M = max_v x_rv, S = sum_v exp(x_rv - M):
 *   logp = x_rt - M - log S
 * bfloat16 values are multiplied exactly and summed in 32 bits; float32
 * values in products as exact as 32-bit ones.  Before the products that give
 * the two gradients dL/dx is rounded: for float32 inputs to 24 bits, for
 * bfloat16 ones to 16 or, in large products of 1024 rows and 1024 classes or
 * more, to 8 (where acdc_vocab_loss may round the exponentials in it to 8 bits
 * as well).
 *
 * hidden: rows x width, weight: classes x width, both of type `dtype`, rows
 * hidden_stride and weight_stride apart (in elements, >= width).  targets as in
 * acdc_train.h: a negative one marks a row that takes no part (its hidden
 * values may hold anything; its outputs and gradient are 0), one >= classes
 * makes its row NaN, and with it the weight's gradient.  hidden and weight
 * are finite; a row of hidden that is not gives NaN for itself and for the
 * weight's gradient.  1 <= width <= 2^17, 1 <= classes <= 2^27, rows <= 2^24.
 * bfloat16 weights are read where they lie if they begin at 16 bytes and width
 * and weight_stride are multiples of 8, weight_stride below 2^22; any other
 * weight is copied into the workspace, piece by piece. */
typedef struct acdc_vocab_head {
  const void* hidden;
  const void* weight;
  const void* targets;
  int64_t hidden_stride, weight_stride, rows;
  int32_t width, classes, dtype, target_bits;
} acdc_vocab_head;

/* Where the gradients go; a null pointer: not wanted.  hidden: rows x width
 * of the head's dtype.  weight: classes x width of weight_type (ACDC_F32, or
 * the head's dtype); with accumulate != 0 the gradient is added to what is
 * there (the sum rounded once). */
typedef struct acdc_vocab_grads {
  void* hidden;
  void* weight;
  int64_t hidden_stride, weight_stride;
  int32_t weight_type, accumulate;
} acdc_vocab_grads;

/* logp [rows]; saved [rows][2] = (M, S), 8-byte aligned, for acdc_vocab_backward
 * (optional, may be null). */
int acdc_vocab_logprob(const acdc_vocab_head* head /* host */, float* logp, float* saved, void* workspace,
                       size_t workspace_bytes, acdc_stream_t stream);

/* dL/dx_rv = c g_r ([v = t] - p_rv) with g = grad_logp = dL/dlogp and c =
 * *scale (device, may be null: 1), and from it dL/dhidden and dL/dweight.  A
 * row with g = 0 takes no part.  `saved` as acdc_vocab_logprob or
 * acdc_vocab_loss filled it for the same head. */
int acdc_vocab_backward(const acdc_vocab_head* head /* host */, const float* saved, const float* grad_logp,
                        const float* scale, const acdc_vocab_grads* grads /* host */, void* workspace,
                        size_t workspace_bytes, acdc_stream_t stream);

/* Cross entropy: -sum_r w_r logp_r / W, W = sum_r w_r (with mean = 0: not
 * divided).  weights (null: 1 each); a row of weight 0 takes no part.  W = 0
 * gives a loss and gradients of 0.  stats, 2 floats: the loss and W.
 * Optional: saved, row_grads [rows] (dL/dlogp without grad_scale, what
 * acdc_vocab_backward takes), and the gradients (grads may be null), which
 * grad_scale multiplies. */
typedef struct acdc_vocab_params {
  float grad_scale;
  int32_t mean;
} acdc_vocab_params;
int acdc_vocab_loss(const acdc_vocab_head* head /* host */, const float* weights,
                    const acdc_vocab_params* params /* host */, float* stats, float* logp, float* saved,
                    float* row_grads, const acdc_vocab_grads* grads /* host */, void* workspace,
                    size_t workspace_bytes, acdc_stream_t stream);

/* Bytes for any of the calls; `gradient` 0: for calls without gradients. */
size_t acdc_vocab_workspace_size(int64_t rows, int32_t width, int32_t classes, int32_t dtype, int32_t gradient);

/* ------------------------------------------------------------- layer norm
 *
 * Per row, with mean and variance (divided by width) of its values:
 *   rstd = 1 / sqrt(variance + eps),  y = (x - mean) rstd weight + bias
 * x: rows x width of x_type, y of y_type, rows x_stride and y_stride apart.
 * weight and bias: width values of vector_type (either may be null: 1 and 0).
 * saved [rows][2] = (mean, rstd), 8-byte aligned (optional).  1 <= width <=
 * 2^24, rows < 2^30. */
int acdc_norm_forward(const void* x, int32_t x_type, int64_t x_stride, const void* weight, const void* bias,
                      int32_t vector_type, float eps, void* y, int32_t y_type, int64_t y_stride, float* saved, int64_t rows,
                      int32_t width, acdc_stream_t stream);

/* With u = (x - mean) rstd and a = grad_y weight:
 *   grad_x = rstd (a - mean(a) - u mean(a u))
 *   grad_weight = sum over rows of grad_y u,  grad_bias = sum over rows of grad_y
 * grad_y is of y_type, grad_x of x_type, grad_weight and grad_bias of
 * grads_type; each may be null (not wanted), and with accumulate != 0 the two
 * sums are added to what is there.  grad_x may be grad_y's own memory (same
 * type, pointer and stride).  The sums run in 32 bits over 1024 parts of the
 * rows at the most and then over the parts.  A workspace size of 256 stands for
 * none: the workspace may be null. */
int acdc_norm_backward(const void* x, int32_t x_type, int64_t x_stride, const void* grad_y, int32_t y_type,
                       int64_t grad_y_stride, const void* weight, int32_t vector_type, const float* saved, void* grad_x,
                       int64_t grad_x_stride, void* grad_weight, void* grad_bias, int32_t grads_type, int32_t accumulate,
                       int64_t rows, int32_t width, void* workspace, size_t workspace_bytes, acdc_stream_t stream);
size_t acdc_norm_workspace_size(int64_t rows, int32_t width);

/* -------------------------------------------------------------- embedding
 *
 * out[r] = scale * weight[tokens[r]]: weight classes x width of weight_type,
 * out rows x width of out_type, rows weight_stride and out_stride apart.
 * A negative token gives a row of zeros, one >= classes a row of NaN.
 * 1 <= width <= 2^20, 1 <= classes <= 2^30, rows <= 2^28 - 64, and
 * (rows / 64 + 1) (width / 512 + 1) <= 2^22, here and below. */
int acdc_embedding_forward(const void* tokens, int32_t token_bits, const void* weight, int32_t weight_type,
                           int64_t weight_stride, float scale, void* out, int32_t out_type, int64_t out_stride, int64_t rows,
                           int32_t width, int32_t classes, acdc_stream_t stream);

/* grad_weight[v] = scale * sum of grad_out[r] over the rows r with token v, in
 * the order of the rows (long sums in pieces of 16 to 64 sorted rows, by the
 * sizes alone), 0 for a class without rows; with accumulate != 0 added to what is there.  Rows whose token is
 * negative or >= classes take no part and are not read. */
int acdc_embedding_backward(const void* tokens, int32_t token_bits, const void* grad_out, int32_t out_type,
                            int64_t out_stride, float scale, void* grad_weight, int32_t weight_type, int64_t weight_stride,
                            int32_t accumulate, int64_t rows, int32_t width, int32_t classes, void* workspace,
                            size_t workspace_bytes, acdc_stream_t stream);
size_t acdc_embedding_workspace_size(int64_t rows, int32_t width, int32_t classes);

#ifdef __cplusplus
}
#endif

#endif /* ACDC_TRAIN_LM_H_ */
