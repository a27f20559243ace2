// Losses over rows of logits (acdc_train.h): token log-probabilities, the
// clipped policy loss and the preference loss, with their gradients.
//
// Mathematics.  All three see a row of logits x only through logp = x_t - M -
// log S and H = log S - U / S, with M = max_j x_j, S = sum_j e_j, U = sum_j
// e_j (x_j - M), e_j = exp(x_j - M).  With g = dL/dlogp and h = dL/dH,
//   dL/dx_j = g [j = t] - p_j (g + h (log p_j + H)),   p_j = e_j / S.
// (M, S) rather than log S is kept per row: p_j from x_j - log S would carry
// the rounding of log S, 2^-24 |log S| relative.
#include <hip/hip_runtime.h>

#include <cmath>

#include "acdc_train.hpp"

namespace acdc {
namespace {

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kNegMax = -3.402823466e38f;

__device__ __forceinline__ float exp_of(float d) { return __builtin_amdgcn_exp2f(d * kLog2e); }

// Class of row r's target; -1: the row takes no part.
__device__ __forceinline__ long long target_of(const void* targets, int bits, long long r) {
  return bits == 64 ? static_cast<const long long*>(targets)[r] : (long long)static_cast<const int*>(targets)[r];
}

// Running (M, S, U) of a softmax row: M the maximum so far, S and U relative to it.
struct Run {
  float m, s, u;
};
__device__ __forceinline__ Run empty_run() { return {kNegMax, 0.f, 0.f}; }
// x - m, kept above -1e30 so that a class of probability 0 (-inf, or a finite
// lowest value) adds 0 and not 0 * inf to U.  NaN stays.
__device__ __forceinline__ float below(float x, float m) {
  const float d = x - m;
  return d < -1e30f ? -1e30f : d;
}
__device__ __forceinline__ Run merge(const Run& a, const Run& b) {
  Run r;
  r.m = fmaxf(a.m, b.m);
  const float da = below(a.m, r.m), db = below(b.m, r.m);
  const float fa = exp_of(da), fb = exp_of(db);
  r.s = a.s * fa + b.s * fb;
  r.u = fa * (a.u + da * a.s) + fb * (b.u + db * b.s);
  return r;
}

constexpr int kThreads = 256;

__device__ __forceinline__ Run merge_wave(Run r) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    const Run b{__shfl_xor(r.m, o), __shfl_xor(r.s, o), __shfl_xor(r.u, o)};
    r = merge(r, b);
  }
  return r;
}

// One workgroup per row: (M, S, H, logp).
template <class T>
__global__ __launch_bounds__(kThreads) void k_row_stats(const typename T::Elem* __restrict__ x, long long stride,
                                                        const void* __restrict__ targets, int bits, int classes,
                                                        float4* __restrict__ stat) {
  __shared__ Run part[kThreads / 64];
  const long long r = blockIdx.x;
  const long long t = target_of(targets, bits, r);
  if (t < 0) {
    if (threadIdx.x == 0) stat[r] = make_float4(0.f, 1.f, 0.f, 0.f);
    return;
  }
  const typename T::Elem* row = x + r * stride;
  Run run = empty_run();
  const int full = classes / T::kPer;
  for (int c = threadIdx.x; c < full; c += kThreads) {
    const auto raw = load_chunk<T>(row + (long long)c * T::kPer);
    Run b = empty_run();
#pragma unroll
    for (int i = 0; i < T::kPer; ++i) b.m = fmaxf(b.m, T::get(raw, i));
#pragma unroll
    for (int i = 0; i < T::kPer; ++i) {
      const float d = below(T::get(raw, i), b.m), e = exp_of(d);
      b.s += e;
      b.u += e * d;
    }
    run = merge(run, b);
  }
  for (int j = full * T::kPer + threadIdx.x; j < classes; j += kThreads) {
    const float v = T::one(row[j]);
    Run b = empty_run();
    b.m = fmaxf(b.m, v);
    const float d = below(v, b.m), e = exp_of(d);
    b.s = e;
    b.u = e * d;
    run = merge(run, b);
  }
  run = merge_wave(run);
  if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = run;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < kThreads / 64; ++w) run = merge(run, part[w]);
    const float xt = t < classes ? T::one(row[t]) : __builtin_nanf("");
    const float log_s = logf(run.s);
    // a row of zero-probability classes only: S = 0
    const float nan = run.s > 0.f ? 0.f : __builtin_nanf("");
    stat[r] = make_float4(run.m, run.s, log_s - run.u / run.s + nan, (xt - run.m) - log_s + nan);
  }
}

// dL/dlogits of one row per workgroup from its (M, S, H, logp), g and h.
template <class T>
__global__ __launch_bounds__(kThreads) void k_row_grad(const typename T::Elem* x, long long stride,
                                                       const void* __restrict__ targets, int bits, int classes,
                                                       const float4* __restrict__ stat,
                                                       const float* __restrict__ grad_logp,
                                                       const float* __restrict__ grad_entropy,
                                                       const float* __restrict__ scale, float scale_host,
                                                       typename T::Elem* grad, long long grad_stride) {
  const long long r = blockIdx.x;
  const long long t = target_of(targets, bits, r);
  typename T::Elem* out = grad + r * grad_stride;
  const typename T::Elem* row = x + r * stride;
  const float c = scale_host * (scale != nullptr ? *scale : 1.f);
  float g = 0.f, h = 0.f;
  if (t >= 0) {
    g = grad_logp[r];
    h = grad_entropy != nullptr ? grad_entropy[r] : 0.f;
  }
  const int full = classes / T::kPer;
  if (g == 0.f && h == 0.f) {
    float zero[T::kPer] = {};
    for (int k = threadIdx.x; k < full; k += kThreads) store_chunk<T>(out + (long long)k * T::kPer, T::pack(zero));
    for (int j = full * T::kPer + threadIdx.x; j < classes; j += kThreads) out[j] = T::to(0.f);
    return;
  }
  g *= c;
  h *= c;
  const float4 st = stat[r];
  const float inv = 1.f / st.y;
  // log p_j + H = d_j + (H - log S)
  const float k0 = g + h * (st.z - logf(st.y)) + (t < classes ? 0.f : __builtin_nanf(""));
  auto value = [&](float v, long long j) {
    const float d = below(v, st.x);
    const float y = -(exp_of(d) * inv) * (k0 + h * d);
    return j == t ? y + g : y;
  };
  for (int k = threadIdx.x; k < full; k += kThreads) {
    const auto raw = load_chunk<T>(row + (long long)k * T::kPer);
    float y[T::kPer];
#pragma unroll
    for (int i = 0; i < T::kPer; ++i) y[i] = value(T::get(raw, i), (long long)k * T::kPer + i);
    store_chunk<T>(out + (long long)k * T::kPer, T::pack(y));
  }
  for (int j = full * T::kPer + threadIdx.x; j < classes; j += kThreads) out[j] = T::to(value(T::one(row[j]), j));
}

// logp and entropy of every row out of its statistics.
__global__ __launch_bounds__(kThreads) void k_row_values(const float4* __restrict__ stat, long long rows,
                                                         float* __restrict__ logp, float* __restrict__ entropy) {
  const long long r = (long long)blockIdx.x * kThreads + threadIdx.x;
  if (r >= rows) return;
  logp[r] = stat[r].w;
  if (entropy != nullptr) entropy[r] = stat[r].z;
}

// Sum of v over the workgroup in a fixed order, for every thread.
template <int THREADS>
__device__ __forceinline__ double total_of(double v, double* part) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
  __syncthreads();
  if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = v;
  __syncthreads();
  double s = part[0];
#pragma unroll
  for (int w = 1; w < THREADS / 64; ++w) s += part[w];
  return s;
}

// The policy loss of all rows: one workgroup.  Writes stats, logp and
// row_grads = (dL/dlogp, dL/dH).
constexpr int kWide = 1024;
struct PolicyArgs {
  const void* targets;
  int bits;
  const float *old, *ref, *advantages, *weights;
  long long rows;
  acdc_policy_params p;
};
__device__ __forceinline__ float weight_of(const PolicyArgs& a, long long r) {
  if (target_of(a.targets, a.bits, r) < 0) return 0.f;
  return a.weights != nullptr ? a.weights[r] : 1.f;
}
__global__ __launch_bounds__(kWide) void k_policy_rows(PolicyArgs a, const float4* __restrict__ stat,
                                                       float* __restrict__ stats, float* __restrict__ logp,
                                                       float* __restrict__ grads) {
  __shared__ double part[kWide / 64];
  double w = 0.0;
  for (long long r = threadIdx.x; r < a.rows; r += kWide) w += weight_of(a, r);
  const double total = total_of<kWide>(w, part);
  const float norm = !a.p.mean ? 1.f : total != 0.0 ? float(1.0 / total) : 0.f;
  double sum[6] = {};
  for (long long r = threadIdx.x; r < a.rows; r += kWide) {
    const float wr = weight_of(a, r) * norm;
    float g = 0.f, h = 0.f, lp = 0.f;
    if (wr != 0.f) {
      const float4 st = stat[r];
      lp = st.w;
      const float adv = a.advantages[r], ratio = expf(lp - a.old[r]);
      const float lo = 1.f - a.p.clip_low, hi = 1.f + a.p.clip_high;
      const float free_ = ratio * adv, bounded = (ratio < lo ? lo : ratio > hi ? hi : ratio) * adv;
      const bool cut = bounded < free_;
      const float policy = -(cut ? bounded : free_);
      float em = 0.f, kl = 0.f;
      if (a.ref != nullptr) {
        const float k = a.ref[r] - lp;
        em = expm1f(k);
        kl = em - k;
      }
      g = wr * ((cut ? 0.f : -free_) - a.p.kl_coef * em);
      h = -a.p.entropy_coef * wr;
      const float loss = policy + a.p.kl_coef * kl - a.p.entropy_coef * st.z;
      const float v[6] = {loss, policy, kl, st.z, cut ? 1.f : 0.f, ratio};
#pragma unroll
      for (int i = 0; i < 6; ++i) sum[i] += double(wr) * double(v[i]);
    }
    logp[r] = lp;
    grads[r] = g;
    grads[a.rows + r] = h;
  }
#pragma unroll
  for (int i = 0; i < 6; ++i) {
    const double s = total_of<kWide>(sum[i], part);
    if (threadIdx.x == 0) stats[i] = float(s);
  }
}

__device__ __forceinline__ long long offset_of(const void* offsets, int bits, long long s, long long rows) {
  const long long o = bits == 64 ? static_cast<const long long*>(offsets)[s]
                                 : (long long)static_cast<const int*>(offsets)[s];
  return o < 0 ? 0 : o > rows ? rows : o;
}

// reward of every sequence: one workgroup per sequence.
__global__ __launch_bounds__(kThreads) void k_rewards(const void* __restrict__ targets, int bits,
                                                      const void* __restrict__ offsets, int offset_bits,
                                                      const float* __restrict__ ref, long long rows, float beta,
                                                      const float4* __restrict__ stat, float* __restrict__ reward) {
  __shared__ double part[kThreads / 64];
  const long long s = blockIdx.x;
  const long long a = offset_of(offsets, offset_bits, s, rows), b = offset_of(offsets, offset_bits, s + 1, rows);
  double v = 0.0;
  for (long long r = a + threadIdx.x; r < b; r += kThreads)
    if (target_of(targets, bits, r) >= 0) v += double(stat[r].w) - double(ref[r]);
  v = total_of<kThreads>(v, part);
  if (threadIdx.x == 0) reward[s] = float(beta * v);
}

// log(1 + exp(z))
__device__ __forceinline__ float softplus(float z) { return fmaxf(z, 0.f) + log1pf(expf(-fabsf(z))); }

// Losses and slopes dL/dlogp of every sequence's rows: one workgroup.
__global__ __launch_bounds__(kWide) void k_pairs(const float* __restrict__ reward, long long pairs, float beta, float e,
                                                 float* __restrict__ stats, float* __restrict__ slope) {
  __shared__ double part[kWide / 64];
  double sum[5] = {};
  for (long long p = threadIdx.x; p < pairs; p += kWide) {
    const float good = reward[2 * p], bad = reward[2 * p + 1], m = good - bad;
    const float loss = (1.f - e) * softplus(-m) + e * softplus(m);
    // NaN margins are not counted as wins, and give NaN slopes
    const float s = (e / (1.f + expf(-m)) - (1.f - e) / (1.f + expf(m))) * (beta / float(pairs));
    slope[2 * p] = s;
    slope[2 * p + 1] = -s;
    const float v[5] = {loss, m > 0.f ? 1.f : 0.f, m, good, bad};
#pragma unroll
    for (int i = 0; i < 5; ++i) sum[i] += double(v[i]);
  }
#pragma unroll
  for (int i = 0; i < 5; ++i) {
    const double s = total_of<kWide>(sum[i], part);
    if (threadIdx.x == 0) stats[i] = pairs > 0 ? float(s / double(pairs)) : 0.f;
  }
}

// logp and row_grads of the preference loss.
__global__ __launch_bounds__(kThreads) void k_preference_rows(const void* __restrict__ targets, int bits,
                                                              const void* __restrict__ offsets, int offset_bits,
                                                              long long rows, long long pairs,
                                                              const float4* __restrict__ stat,
                                                              const float* __restrict__ slope, float* __restrict__ logp,
                                                              float* __restrict__ grads) {
  const long long r = (long long)blockIdx.x * kThreads + threadIdx.x;
  if (r >= rows) return;
  const bool on = target_of(targets, bits, r) >= 0;
  // the sequence s with offsets[s] <= r < offsets[s + 1], if any
  long long lo = 0, hi = 2 * pairs;  // offsets[lo] <= r < offsets[hi] once both ends hold
  float g = 0.f;
  if (on && pairs > 0 && offset_of(offsets, offset_bits, 0, rows) <= r && r < offset_of(offsets, offset_bits, hi, rows)) {
    while (hi - lo > 1) {
      const long long mid = (lo + hi) / 2;
      if (offset_of(offsets, offset_bits, mid, rows) <= r) lo = mid;
      else hi = mid;
    }
    g = slope[lo];
  }
  logp[r] = on ? stat[r].w : 0.f;
  grads[r] = g;
  grads[rows + r] = 0.f;
}

// ------------------------------------------------------------------ host side

bool logits_ok(const void* logits, int32_t dtype, int64_t stride, const void* targets, int32_t bits, int64_t rows,
               int32_t classes, int* status) {
  const size_t eb = dtype_bytes(dtype);
  *status = ACDC_ERR_INVALID_ARG;
  if (eb == 0 || (bits != 32 && bits != 64) || rows < 0 || rows > 0x7fffffff || classes < 1) return false;
  if (stride < classes || stride > (int64_t(1) << 40)) return false;
  if (rows > 0 && (logits == nullptr || targets == nullptr)) return false;
  if (!aligned_to(logits, eb) || !aligned_to(targets, size_t(bits) / 8)) return false;
  *status = ACDC_OK;
  return true;
}

struct Span {
  uintptr_t a, b;
};
Span span_of(const void* p, int64_t rows, int64_t stride, int32_t classes, size_t eb) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(p);
  return {a, rows > 0 ? a + uintptr_t((rows - 1) * stride + classes) * eb : a};
}
// grad_logits: the logits themselves, or memory apart from them.
bool grad_ok(const void* logits, int64_t stride, const void* grad, int64_t grad_stride, int32_t dtype, int64_t rows,
             int32_t classes) {
  const size_t eb = dtype_bytes(dtype);
  if (grad_stride < classes || grad_stride > (int64_t(1) << 40) || !aligned_to(grad, eb)) return false;
  if (grad == logits) return grad_stride == stride;
  const Span x = span_of(logits, rows, stride, classes, eb), g = span_of(grad, rows, grad_stride, classes, eb);
  return x.b <= g.a || g.b <= x.a;
}
bool floats_ok(std::initializer_list<const void*> must, std::initializer_list<const void*> may) {
  for (const void* p : must)
    if (p == nullptr || !aligned_to(p, 4)) return false;
  for (const void* p : may)
    if (!aligned_to(p, 4)) return false;
  return true;
}

size_t up256(size_t b) { return (b + 255) & ~size_t(255); }
struct Workspace {
  size_t stat, grads, reward, slope, total;
};
Workspace layout(int64_t rows, int64_t pairs) {
  Workspace w{};
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t o = at;
    at += up256(bytes);
    return o;
  };
  w.stat = take(size_t(rows) * sizeof(float4));
  w.grads = take(size_t(rows) * 2 * sizeof(float));
  w.reward = take(size_t(pairs) * 2 * sizeof(float));
  w.slope = take(size_t(pairs) * 2 * sizeof(float));
  w.total = at;
  return w;
}
bool sizes_ok(int64_t rows, int32_t classes, int32_t dtype) {
  return dtype_bytes(dtype) != 0 && rows >= 0 && rows <= 0x7fffffff && classes >= 1;
}

int done() {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? ACDC_OK : hip_fail(e);
}

template <class F>
void with_type(int32_t dtype, F&& f) {
  if (dtype == ACDC_F32) f.template operator()<F32>();
  else f.template operator()<BF16>();
}

int launch_stats(const void* logits, int32_t dtype, int64_t stride, const void* targets, int32_t bits, int64_t rows,
                 int32_t classes, float4* stat, hipStream_t s) {
  with_type(dtype, [&]<class T>() {
    hipLaunchKernelGGL(k_row_stats<T>, dim3(unsigned(rows)), dim3(kThreads), 0, s,
                       static_cast<const typename T::Elem*>(logits), (long long)stride, targets, bits, classes, stat);
  });
  return done();
}
int launch_grad(const void* logits, int32_t dtype, int64_t stride, const void* targets, int32_t bits, int64_t rows,
                int32_t classes, const float4* stat, const float* g, const float* h, const float* scale, float scale_host,
                void* grad, int64_t grad_stride, hipStream_t s) {
  with_type(dtype, [&]<class T>() {
    hipLaunchKernelGGL(k_row_grad<T>, dim3(unsigned(rows)), dim3(kThreads), 0, s,
                       static_cast<const typename T::Elem*>(logits), (long long)stride, targets, bits, classes, stat, g,
                       h, scale, scale_host, static_cast<typename T::Elem*>(grad), (long long)grad_stride);
  });
  return done();
}

unsigned blocks_for(int64_t rows) { return unsigned((rows + kThreads - 1) / kThreads); }

}  // namespace
}  // namespace acdc

using namespace acdc;

extern "C" size_t acdc_logprob_workspace_size(int64_t rows, int32_t classes, int32_t dtype) {
  return sizes_ok(rows, classes, dtype) ? layout(rows, 0).total : 0;
}

extern "C" int acdc_logprob_forward(const void* logits, int32_t dtype, int64_t stride, const void* targets,
                                    int32_t target_bits, int64_t rows, int32_t classes, float* logp, float* entropy,
                                    float* saved, void* workspace, size_t workspace_bytes, acdc_stream_t stream) {
  int rc;
  if (!logits_ok(logits, dtype, stride, targets, target_bits, rows, classes, &rc)) return rc;
  if (rows == 0) return ACDC_OK;
  if (!floats_ok({logp}, {entropy}) || !aligned_to(saved, 16) || !aligned_to(workspace, 16)) return ACDC_ERR_INVALID_ARG;
  const Workspace w = layout(rows, 0);
  if (workspace == nullptr || workspace_bytes < w.total) return ACDC_ERR_WORKSPACE;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  float4* stat = reinterpret_cast<float4*>(saved != nullptr ? saved : workspace);
  rc = launch_stats(logits, dtype, stride, targets, target_bits, rows, classes, stat, s);
  if (rc != ACDC_OK) return rc;
  hipLaunchKernelGGL(k_row_values, dim3(blocks_for(rows)), dim3(kThreads), 0, s, stat, (long long)rows, logp, entropy);
  return done();
}

extern "C" int acdc_logprob_backward(const void* logits, int32_t dtype, int64_t stride, const void* targets,
                                     int32_t target_bits, const float* saved, const float* grad_logp,
                                     const float* grad_entropy, const float* scale, void* grad_logits,
                                     int64_t grad_stride, int64_t rows, int32_t classes, acdc_stream_t stream) {
  int rc;
  if (!logits_ok(logits, dtype, stride, targets, target_bits, rows, classes, &rc)) return rc;
  if (rows == 0) return ACDC_OK;
  if (saved == nullptr || grad_logits == nullptr || !aligned_to(saved, 16) ||
      !floats_ok({grad_logp}, {grad_entropy, scale}) ||
      !grad_ok(logits, stride, grad_logits, grad_stride, dtype, rows, classes))
    return ACDC_ERR_INVALID_ARG;
  return launch_grad(logits, dtype, stride, targets, target_bits, rows, classes, reinterpret_cast<const float4*>(saved),
                     grad_logp, grad_entropy, scale, 1.f, grad_logits, grad_stride,
                     reinterpret_cast<hipStream_t>(stream));
}

extern "C" size_t acdc_policy_workspace_size(int64_t rows, int32_t classes, int32_t dtype) {
  return sizes_ok(rows, classes, dtype) ? layout(rows, 0).total : 0;
}

extern "C" int acdc_policy_loss(const void* logits, int32_t dtype, int64_t stride, const void* targets,
                                int32_t target_bits, const float* logp_old, const float* logp_ref,
                                const float* advantages, const float* weights, int64_t rows, int32_t classes,
                                const acdc_policy_params* params, float* stats, float* logp, void* grad_logits,
                                int64_t grad_stride, float* saved, float* row_grads, void* workspace,
                                size_t workspace_bytes, acdc_stream_t stream) {
  int rc;
  if (!logits_ok(logits, dtype, stride, targets, target_bits, rows, classes, &rc)) return rc;
  if (params == nullptr || !floats_ok({stats}, {logp_old, logp_ref, advantages, weights, logp, row_grads}) ||
      !aligned_to(saved, 16) || !aligned_to(workspace, 16))
    return ACDC_ERR_INVALID_ARG;
  const acdc_policy_params p = *params;
  if (!(p.clip_low >= 0.f) || !(p.clip_high >= 0.f) || !(p.kl_coef - p.kl_coef == 0.f) ||
      !(p.entropy_coef - p.entropy_coef == 0.f) || !(p.grad_scale - p.grad_scale == 0.f))
    return ACDC_ERR_INVALID_ARG;
  if (p.kl_coef != 0.f && logp_ref == nullptr) return ACDC_ERR_INVALID_ARG;
  if (rows > 0 && (logp_old == nullptr || advantages == nullptr || logp == nullptr)) return ACDC_ERR_INVALID_ARG;
  if (grad_logits != nullptr && !grad_ok(logits, stride, grad_logits, grad_stride, dtype, rows, classes))
    return ACDC_ERR_INVALID_ARG;
  const Workspace w = layout(rows, 0);
  if (w.total > 0 && (workspace == nullptr || workspace_bytes < w.total)) return ACDC_ERR_WORKSPACE;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  char* ws = static_cast<char*>(workspace);
  float4* stat = saved != nullptr ? reinterpret_cast<float4*>(saved) : reinterpret_cast<float4*>(ws + w.stat);
  float* grads = row_grads != nullptr ? row_grads : reinterpret_cast<float*>(ws + w.grads);
  if (rows > 0) {
    rc = launch_stats(logits, dtype, stride, targets, target_bits, rows, classes, stat, s);
    if (rc != ACDC_OK) return rc;
  }
  const PolicyArgs a{targets, target_bits, logp_old, logp_ref, advantages, weights, rows, p};
  hipLaunchKernelGGL(k_policy_rows, dim3(1), dim3(kWide), 0, s, a, stat, stats, logp, grads);
  rc = done();
  if (rc != ACDC_OK || rows == 0 || grad_logits == nullptr) return rc;
  return launch_grad(logits, dtype, stride, targets, target_bits, rows, classes, stat, grads, grads + rows, nullptr,
                     p.grad_scale, grad_logits, grad_stride, s);
}

extern "C" size_t acdc_preference_workspace_size(int64_t rows, int32_t classes, int32_t dtype, int64_t pairs) {
  if (!sizes_ok(rows, classes, dtype) || pairs < 0 || pairs > 0x3fffffff) return 0;
  return layout(rows, pairs).total;
}

extern "C" int acdc_preference_loss(const void* logits, int32_t dtype, int64_t stride, const void* targets,
                                    int32_t target_bits, const void* offsets, int32_t offset_bits,
                                    const float* logp_ref, int64_t rows, int32_t classes, int64_t pairs,
                                    const acdc_preference_params* params, float* stats, float* logp, void* grad_logits,
                                    int64_t grad_stride, float* saved, float* row_grads, void* workspace,
                                    size_t workspace_bytes, acdc_stream_t stream) {
  int rc;
  if (!logits_ok(logits, dtype, stride, targets, target_bits, rows, classes, &rc)) return rc;
  if (params == nullptr || pairs < 0 || pairs > 0x3fffffff || (offset_bits != 32 && offset_bits != 64) ||
      !aligned_to(offsets, size_t(offset_bits) / 8) || (pairs > 0 && offsets == nullptr) ||
      !floats_ok({stats}, {logp_ref, logp, row_grads}) || !aligned_to(saved, 16) || !aligned_to(workspace, 16))
    return ACDC_ERR_INVALID_ARG;
  const acdc_preference_params p = *params;
  if (!(p.beta - p.beta == 0.f) || !(p.grad_scale - p.grad_scale == 0.f) || !(p.label_smoothing >= 0.f) ||
      !(p.label_smoothing <= 1.f))
    return ACDC_ERR_INVALID_ARG;
  if (rows > 0 && (logp_ref == nullptr || logp == nullptr)) return ACDC_ERR_INVALID_ARG;
  if (grad_logits != nullptr && !grad_ok(logits, stride, grad_logits, grad_stride, dtype, rows, classes))
    return ACDC_ERR_INVALID_ARG;
  const Workspace w = layout(rows, pairs);
  if (w.total > 0 && (workspace == nullptr || workspace_bytes < w.total)) return ACDC_ERR_WORKSPACE;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  char* ws = static_cast<char*>(workspace);
  float4* stat = saved != nullptr ? reinterpret_cast<float4*>(saved) : reinterpret_cast<float4*>(ws + w.stat);
  float* grads = row_grads != nullptr ? row_grads : reinterpret_cast<float*>(ws + w.grads);
  float* reward = reinterpret_cast<float*>(ws + w.reward);
  float* slope = reinterpret_cast<float*>(ws + w.slope);
  if (rows > 0) {
    rc = launch_stats(logits, dtype, stride, targets, target_bits, rows, classes, stat, s);
    if (rc != ACDC_OK) return rc;
  }
  if (pairs > 0)
    hipLaunchKernelGGL(k_rewards, dim3(unsigned(2 * pairs)), dim3(kThreads), 0, s, targets, target_bits, offsets,
                       offset_bits, logp_ref, (long long)rows, p.beta, stat, reward);
  hipLaunchKernelGGL(k_pairs, dim3(1), dim3(kWide), 0, s, reward, (long long)pairs, p.beta, p.label_smoothing, stats,
                     slope);
  if (rows > 0)
    hipLaunchKernelGGL(k_preference_rows, dim3(blocks_for(rows)), dim3(kThreads), 0, s, targets, target_bits, offsets,
                       offset_bits, (long long)rows, (long long)pairs, stat, slope, logp, grads);
  rc = done();
  if (rc != ACDC_OK || rows == 0 || grad_logits == nullptr) return rc;
  return launch_grad(logits, dtype, stride, targets, target_bits, rows, classes, stat, grads, grads + rows, nullptr,
                     p.grad_scale, grad_logits, grad_stride, s);
}
