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

#include <algorithm>
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
constexpr int kAhead = 4;  // chunks that a thread of the streaming kernels asks for at a time

__device__ __forceinline__ Run merge_wave(Run r) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    const Run b{__shfl_xor(r.m, o), __shfl_xor(r.s, o), __shfl_xor(r.u, o)};
    r = merge(r, b);
  }
  return r;
}

// (M, S, H, logp) of a row from its whole run and its target's logit.
__device__ __forceinline__ float4 stat_of(const Run& run, float xt) {
  const float log_s = logf(run.s);
  // a row of zero-probability classes only has S = 0
  const float nan = run.s > 0.f ? 0.f : __builtin_nanf("");
  return make_float4(run.m, run.s, log_s - run.u / run.s + nan, (xt - run.m) - log_s + nan);
}
// The logit of target t >= 0; NaN past the classes.
template <class T>
__device__ __forceinline__ float target_logit(const typename T::Elem* row, long long t, int classes) {
  return t < classes ? T::one(row[t]) : __builtin_nanf("");
}

// A row as chunks at aligned addresses and the elements around them: `head`
// elements before the first chunk, `full` chunks, and `extra` elements in all
// outside of them (fewer than 2 kPer), one for each of the first lanes.  A
// chunk that lies across two cache lines costs both: rows of 65535 bfloat16
// ran 20 % slower as chunks from the row's first element.
template <class T, bool UNIFORM = true>
struct Cut {
  int head, full, extra;
  __device__ __forceinline__ Cut(const typename T::Elem* row, int classes) {
    const unsigned off = unsigned(reinterpret_cast<uintptr_t>(row)) & 15u;
    int h = off != 0u ? int((16u - off) / sizeof(typename T::Elem)) : 0;
    if (h > classes) h = classes;
    head = UNIFORM ? uniform(h) : h;
    full = (classes - head) / T::kPer;
    extra = classes - full * T::kPer;
  }
  // the element outside of the chunks that is lane's (lane < extra)
  __device__ __forceinline__ int element(int lane) const { return lane < head ? lane : full * T::kPer + lane; }
  // class t's chunk, or -1 if it lies outside of them (then it is lane_of(t)'s)
  __device__ __forceinline__ int chunk_of(int t) const {
    const int i = t - head;
    return i >= 0 && i < full * T::kPer ? i / T::kPer : -1;
  }
  __device__ __forceinline__ int lane_of(int t) const { return t < head ? t : t - full * T::kPer; }
};

// Chunks (16 bytes) that one of `split` workgroups of a row takes: from, to.
__device__ __forceinline__ void chunks_of(int full, int split, int k, int& from, int& to) {
  const int per = (full + split - 1) / split;
  from = min(full, k * per);
  to = min(full, from + per);
}

// What a row leaves besides its gradient (null: not wanted).
struct RowOut {
  float* logp;
  float* entropy;
  float4* stat;
  float *g, *h;
};
__device__ __forceinline__ void put_row(const RowOut& o, long long r, const float4& st, float g, float h) {
  if (o.logp != nullptr) o.logp[r] = st.w;
  if (o.entropy != nullptr) o.entropy[r] = st.z;
  if (o.stat != nullptr) o.stat[r] = st;
  if (o.g != nullptr) {
    o.g[r] = g;
    o.h[r] = h;
  }
}

// f.template operator()<N, ALL>(c) for the chunks c, c + step, ... below `to`, AHEAD
// at a time; what is left at the end (fewer, ALL false) is asked for together too.
template <int AHEAD, class F>
__device__ __forceinline__ void stream(int c, int to, int step, F&& f) {
  for (; c + (AHEAD - 1) * step < to; c += AHEAD * step) f.template operator()<AHEAD, true>(c);
  if (c < to) f.template operator()<AHEAD - 1, false>(c);
}
// The run of N chunks c, c + step, ...; without ALL only of those below `to`.
template <class T, int N, bool ALL>
__device__ __forceinline__ Run run_of(const typename T::Elem* body, int c, int step, int to) {
  typename T::Raw raw[N];
#pragma unroll
  for (int q = 0; q < N; ++q)
    if (ALL || c + q * step < to) raw[q] = load_chunk<T>(body + (long long)(c + q * step) * T::kPer);
  Run b = empty_run();
#pragma unroll
  for (int q = 0; q < N; ++q)
    if (ALL || c + q * step < to) {
#pragma unroll
      for (int i = 0; i < T::kPer; ++i) b.m = fmaxf(b.m, T::get(raw[q], i));
    }
#pragma unroll
  for (int q = 0; q < N; ++q)
    if (ALL || c + q * step < to) {
#pragma unroll
      for (int i = 0; i < T::kPer; ++i) {
        const float d = T::get(raw[q], i) - b.m, e = exp_of(d);
        b.s += e;
        b.u += e * fmaxf(d, -1e30f);
      }
    }
  return b;
}

// Over a row that THREADS lanes share: 16 or a wave (64), which need no barrier,
// or the workgroup.
template <int THREADS>
struct Group {
  float* slots;  // 3 * THREADS / 64 floats of LDS
  __device__ __forceinline__ float max(float v) {
    if constexpr (THREADS == 16) return over_16(v, [](float p, float q) { return fmaxf(p, q); });
    v = wave_max(v);
    if constexpr (THREADS > 64) {
      if (threadIdx.x % 64 == 0) slots[threadIdx.x / 64] = v;
      __syncthreads();
#pragma unroll
      for (int w = 0; w < THREADS / 64; ++w) v = fmaxf(v, slots[w]);
    }
    return v;
  }
  // s and u over the group; the slots are those that max does not use, so that
  // a barrier a call is enough (the next row's max comes after this one's barrier)
  __device__ __forceinline__ void sum(float& s, float& u) {
    if constexpr (THREADS == 16) {
      s = over_16(s, [](float p, float q) { return p + q; });
      u = over_16(u, [](float p, float q) { return p + q; });
      return;
    }
    s = wave_sum(s);
    u = wave_sum(u);
    if constexpr (THREADS > 64) {
      constexpr int W = THREADS / 64;
      if (threadIdx.x % 64 == 0) {
        slots[W + threadIdx.x / 64] = s;
        slots[2 * W + threadIdx.x / 64] = u;
      }
      __syncthreads();
      s = u = 0.f;
#pragma unroll
      for (int w = 0; w < W; ++w) {
        s += slots[W + w];
        u += slots[2 * W + w];
      }
    }
  }
};

// Rows that LANES lanes share, several to a workgroup where those are few.
template <int LANES>
struct Share {
  static constexpr int WG = LANES < kThreads ? kThreads : LANES, ROWS = WG / LANES;
  static __device__ __forceinline__ int lane() { return ROWS == 1 ? int(threadIdx.x) : int(threadIdx.x) % LANES; }
  static __device__ __forceinline__ unsigned first() {
    if constexpr (ROWS == 1) return blockIdx.x;
    const int row = int(threadIdx.x) / LANES;
    return blockIdx.x * ROWS + unsigned(LANES == 64 ? uniform(row) : row);
  }
};

// A part of a row, streamed: every thread keeps a run of its own.
// Item r * split + k is part k of row r; with split = 1 its lanes write the
// row's (M, S, H, logp), otherwise the runs of the parts.  Bound by HBM: 19.9 k
// rows of 32768 bfloat16, 1.3 GB, in 220 us (5.9 TB/s; the vector unit 81 % busy).
template <class T, int LANES>
__global__ __launch_bounds__(Share<LANES>::WG) void k_row_stats(const typename T::Elem* __restrict__ x,
                                                                long long stride, const void* __restrict__ targets,
                                                                int bits, int classes, int split, unsigned items,
                                                                RowOut out, float4* __restrict__ parts) {
  __shared__ float slots[3 * Share<LANES>::WG / 64];
  Group<LANES> group{slots};
  const int lane = Share<LANES>::lane();
  for (unsigned item = Share<LANES>::first(); item < items; item += gridDim.x * Share<LANES>::ROWS) {
    const int k = item % unsigned(split);
    const long long r = item / unsigned(split);
    const long long t = target_of(targets, bits, r);
    if (t < 0) {
      if (lane == 0 && k == 0) put_row(out, r, make_float4(0.f, 1.f, 0.f, 0.f), 0.f, 0.f);
      continue;
    }
    const typename T::Elem* row = x + r * stride;
    const float xt = split == 1 ? target_logit<T>(row, t, classes) : 0.f;
    Run run = empty_run();
    const Cut<T, (LANES >= 64)> cut(row, classes);
    int from, to;
    chunks_of(cut.full, split, k, from, to);
    const typename T::Elem* body = row + cut.head;
    stream<kAhead>(from + lane, to, LANES, [&]<int N, bool ALL>(int c) {
      run = merge(run, run_of<T, N, ALL>(body, c, LANES, to));
    });
    if (k == split - 1 && lane < cut.extra) {
      const float v = T::one(row[cut.element(lane)]);
      Run b = empty_run();
      b.m = fmaxf(b.m, v);
      const float d = v - b.m, e = exp_of(d);
      b.s = e;
      b.u = e * fmaxf(d, -1e30f);
      run = merge(run, b);
    }
    const float m = group.max(run.m), d = below(run.m, m), f = exp_of(d);
    float s = run.s * f, u = f * (run.u + d * run.s);
    group.sum(s, u);
    if (lane == 0) {
      if (split == 1) put_row(out, r, stat_of(Run{m, s, u}, xt), 0.f, 0.f);
      else parts[r * split + k] = make_float4(m, s, u, 0.f);
    }
  }
}

// The row's statistics out of its parts, by one thread.
__device__ __forceinline__ float4 join_alone(const float4* __restrict__ parts, int split, long long r, float xt) {
  const float4* p = parts + r * split;
  float m = kNegMax, s = 0.f, u = 0.f;
#pragma unroll 8
  for (int k = 0; k < split; ++k) m = fmaxf(m, p[k].x);
#pragma unroll 8
  for (int k = 0; k < split; ++k) {
    const float4 v = p[k];
    const float d = below(v.x, m), f = exp_of(d);
    s += v.y * f;
    u += f * (v.z + d * v.y);
  }
  return stat_of(Run{m, s, u}, xt);
}

// The row's statistics out of its parts (at most 64), for a whole wave.
template <class T>
__device__ __forceinline__ float4 join_parts(const float4* __restrict__ parts, int split, long long r, float xt) {
  const int lane = threadIdx.x % 64;
  Run run = empty_run();
  if (lane < split) {
    const float4 p = parts[r * split + lane];
    run = Run{p.x, p.y, p.z};
  }
  return stat_of(merge_wave(run), xt);
}

// Statistics of rows in parts: one wave per row; logp and entropy too.  2 us, which
// is what a launch takes.
template <class T>
__global__ __launch_bounds__(kThreads) void k_row_join(const typename T::Elem* __restrict__ x, long long stride,
                                                       const void* __restrict__ targets, int bits, int classes,
                                                       const float4* __restrict__ parts, int split, long long rows,
                                                       RowOut out) {
  const long long r = (long long)blockIdx.x * (kThreads / 64) + threadIdx.x / 64;
  if (r >= rows) return;
  const long long t = target_of(targets, bits, r);
  float4 st = make_float4(0.f, 1.f, 0.f, 0.f);
  if (t >= 0) st = join_parts<T>(parts, split, r, target_logit<T>(x + r * stride, t, classes));
  if (threadIdx.x % 64 == 0) put_row(out, r, st, 0.f, 0.f);
}

// What turns a logit into its gradient: y_j = e_j (a + b d_j), d_j = x_j - M,
// and g more for the target.
struct Slope {
  float m, a, b;
};
__device__ __forceinline__ Slope slope_of(float m, float s, float h_row, float g, float h) {
  const float inv = 1.f / s;
  return {m, -inv * (g + h * (h_row - logf(s))), -inv * h};
}
__device__ __forceinline__ float slope_value(const Slope& k, float x) {
  const float d = x - k.m;
  // a class of probability 0 has d = -inf or nearly: its 0 is not to meet an infinity
  return exp_of(d) * (k.a + k.b * fmaxf(d, -1e30f));
}

// The gradients of N chunks c, c + step, ... as in run_of.  Their loads stand before their
// stores: the gradient may be the logits' own memory, so that the compiler
// would not move a load ahead of an earlier store by itself.
template <class T, int N, bool ALL>
__device__ __forceinline__ void slopes(const Slope& sl, const typename T::Elem* body, typename T::Elem* out, int c, int step,
                                       int to) {
  typename T::Raw raw[N];
#pragma unroll
  for (int q = 0; q < N; ++q)
    if (ALL || c + q * step < to) raw[q] = load_chunk<T>(body + (long long)(c + q * step) * T::kPer);
#pragma unroll
  for (int q = 0; q < N; ++q)
    if (ALL || c + q * step < to) {
      float y[T::kPer];
#pragma unroll
      for (int i = 0; i < T::kPer; ++i) y[i] = slope_value(sl, T::get(raw[q], i));
      store_chunk<T>(out + (long long)(c + q * step) * T::kPer, T::pack(y));
    }
}

// dL/dlogits from each row's (M, S, H, logp), g and h; items as in k_row_stats,
// the last rows first: what a forward read last is what the cache still holds.
// Bound by HBM: 26.4 k rows of 32768 bfloat16, a quarter of them idle, read 1.3
// and write 1.73 GB in 545 us (5.6 TB/s).
template <class T, int LANES>
__global__ __launch_bounds__(kThreads) void k_row_grad(const typename T::Elem* x, long long stride,
                                                       const void* __restrict__ targets, int bits, int classes,
                                                       const float4* __restrict__ stat,
                                                       const float* __restrict__ grad_logp,
                                                       const float* __restrict__ grad_entropy,
                                                       const float* __restrict__ scale, float scale_host,
                                                       typename T::Elem* grad, long long grad_stride, int split,
                                                       unsigned items) {
  static_assert(LANES <= kThreads);
  const int lane = Share<LANES>::lane();
  for (unsigned item = Share<LANES>::first(); item < items; item += gridDim.x * Share<LANES>::ROWS) {
    const unsigned at = items - 1 - item;
    const int k = at % unsigned(split);
    const long long r = at / unsigned(split);
    const long long t = target_of(targets, bits, r);
    typename T::Elem* out = grad + r * grad_stride;
    const typename T::Elem* row = x + r * stride;
    const float c = scale_host * (scale != nullptr ? *scale : 1.f);
    const float4 st = stat[r];
    float g = grad_logp[r], h = grad_entropy != nullptr ? grad_entropy[r] : 0.f;  // (asked for along with the target)
    if (t < 0) g = h = 0.f;
    const Cut<T, (LANES >= 64)> cut(row, classes);
    int from, to;
    chunks_of(cut.full, split, k, from, to);
    const int one = cut.element(lane);
    const bool has_one = k == split - 1 && lane < cut.extra;
    const typename T::Elem* body = row + cut.head;
    typename T::Elem* out_body = out + cut.head;
    if (g == 0.f && h == 0.f) {
      float zero[T::kPer] = {};
      for (int i = from + lane; i < to; i += LANES)
        store_chunk<T>(out_body + (long long)i * T::kPer, T::pack(zero));
      if (has_one) out[one] = T::to(0.f);
      continue;
    }
    g *= c;
    h *= c;
    Slope sl = slope_of(st.x, st.y, st.z, g, h);
    if (t >= classes) sl.a = __builtin_nanf("");
    // the thread that writes the target's chunk writes the target again, with its g
    bool mine = false;
    if (t < classes) {
      const int tc = cut.chunk_of(int(t));
      mine = tc >= 0 ? tc >= from && tc < to && (tc - from) % LANES == lane
                     : has_one && cut.lane_of(int(t)) == lane;
    }
    const float yt = mine ? slope_value(sl, T::one(row[t])) + g : 0.f;
    stream<kAhead>(from + lane, to, LANES, [&]<int N, bool ALL>(int i) {
      slopes<T, N, ALL>(sl, body, out_body, i, LANES, to);
    });
    if (has_one) out[one] = T::to(slope_value(sl, T::one(row[one])));
    if (mine) out[t] = T::to(yt);
  }
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

// --------------------------------------------------------- the policy loss
constexpr int kWide = 1024;
struct PolicyArgs {
  const void* targets;
  int bits;
  const float *old, *ref, *advantages, *weights;
  long long rows;
  acdc_policy_params p;
};
__device__ __forceinline__ float weight_of(const PolicyArgs& a, long long r) {
  const float w = a.weights != nullptr ? a.weights[r] : 1.f;  // (asked for along with the target)
  return target_of(a.targets, a.bits, r) < 0 ? 0.f : w;
}
__device__ __forceinline__ float norm_of(const PolicyArgs& a, double total) {
  return !a.p.mean ? 1.f : total != 0.0 ? float(1.0 / total) : 0.f;
}

constexpr int kStats = 6;
struct PolicyRow {
  float g, h;        // dL/dlogp, dL/dH
  float v[kStats];   // what the row adds to the stats
};
// One row that takes part, of normalised weight w.
__device__ __forceinline__ PolicyRow policy_row(const acdc_policy_params& p, float w, float logp, float entropy,
                                                float old, float adv, bool has_ref, float ref) {
  const float ratio = expf(logp - old), lo = 1.f - p.clip_low, hi = 1.f + p.clip_high;
  const float free_ = ratio * adv, bounded = (ratio < lo ? lo : ratio > hi ? hi : ratio) * adv;
  const bool cut = bounded < free_;
  const float policy = -(cut ? bounded : free_);
  float em = 0.f, kl = 0.f;
  if (has_ref) {
    const float k = ref - logp;
    em = expm1f(k);  // exp(k) - 1 - k of policies close to each other is a small difference
    kl = k < __builtin_inff() ? em - k : em;  // (a token of probability 0: infinite, not inf - inf)
  }
  PolicyRow r;
  // (a coefficient of 0, with the reference's values for the stats alone, leaves
  // them out: far from the reference they are infinite)
  const bool counts = p.kl_coef != 0.f;
  r.g = w * ((cut ? 0.f : -free_) - (counts ? p.kl_coef * em : 0.f));
  r.h = -p.entropy_coef * w;
  r.v[0] = w * (policy + (counts ? p.kl_coef * kl : 0.f) - p.entropy_coef * entropy);
  r.v[1] = w * policy;
  r.v[2] = w * kl;
  r.v[3] = w * entropy;
  r.v[4] = cut ? w : 0.f;
  r.v[5] = w * ratio;
  return r;
}

// Sums of the weights, for the kernels that need 1 / W: rows in at most
// kWeightSums groups, a workgroup each.  (One workgroup of 1024 for up to 16384
// rows, and one number for the others to read, took 3 us longer with the kernel
// after it at 8192 rows and 4 at 16384.)
constexpr int kWeightSums = 256;
__host__ __device__ inline long long weight_group(long long rows) {
  const long long per = (rows + kWeightSums - 1) / kWeightSums;
  return per > kThreads ? per : kThreads;
}
__global__ __launch_bounds__(kThreads) void k_weight_sums(PolicyArgs a, double* __restrict__ sums) {
  __shared__ float part[kThreads / 64];
  const long long per = weight_group(a.rows), from = blockIdx.x * per;
  const long long to = from + per < a.rows ? from + per : a.rows;
  double w = 0.0;
#pragma unroll 4
  for (long long r = from + threadIdx.x; r < to; r += kThreads) w += double(weight_of(a, r));
  const float wave = wave_sum(float(w));
  if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = wave;
  __syncthreads();
  if (threadIdx.x == 0) {
    double total = 0.0;
#pragma unroll
    for (int k = 0; k < kThreads / 64; ++k) total += double(part[k]);
    sums[blockIdx.x] = total;
  }
}
// W summed by every workgroup itself, which saves the launch before it: while
// all of them together read no more than kOwnWeights weights.  2000 rows of 1000
// floats (125 workgroups) 14 -> 11.6 us, 8000 of 100 bfloat16 (250) 14 -> 11.6,
// 1000 of 2000 floats (250) 14.1 -> 11.8; but 2000 of 20000 bfloat16 (2000) 41 ->
// 44, 4000 of 4096 floats (4000) 32 -> 39.
constexpr long long kOwnWeights = 1 << 21;
template <int WG>
__device__ __forceinline__ double weight_all(const PolicyArgs& a, float* part) {
  double w = 0.0;
#pragma unroll 4
  for (long long r = threadIdx.x; r < a.rows; r += WG) w += double(weight_of(a, r));
  const float wave = wave_sum(float(w));
  if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = wave;
  __syncthreads();
  double total = 0.0;
#pragma unroll
  for (int k = 0; k < WG / 64; ++k) total += double(part[k]);
  return total;
}
// W out of the sums, for a whole wave.
__device__ __forceinline__ double weight_total(const double* __restrict__ sums, int groups) {
  double w = 0.0;
  for (int i = threadIdx.x % 64; i < groups; i += 64) w += sums[i];
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) w += __shfl_xor(w, o);
  return w;
}

// The policy loss of rows whose statistics stand in `stat` (in parts of
// `split`, where that is more than 1): one thread per row, or a wave for each
// of up to 16 rows in parts.  With one workgroup it sums the weights and writes
// the stats itself; with more, `sums` holds the weights' sums and `partial` gets
// each workgroup's stats.  A few us of latency: what it reads is nothing beside
// the logits.
template <class T>
__global__ __launch_bounds__(kWide) void k_policy_rows(PolicyArgs a, const typename T::Elem* __restrict__ x,
                                                       long long stride, int classes, const float4* __restrict__ parts,
                                                       int split, const double* __restrict__ sums, int groups,
                                                       const float4* stat, RowOut out, float* __restrict__ partial) {
  __shared__ double part[kWide / 64];
  __shared__ float waves[kWide / 64][kStats];
  float norm = 1.f;
  if (a.p.mean) {
    if (gridDim.x == 1) {
      double w = 0.0;
      for (long long r = threadIdx.x; r < a.rows; r += kWide) w += double(weight_of(a, r));
      norm = norm_of(a, total_of<kWide>(w, part));
    } else {
      norm = norm_of(a, weight_total(sums, groups));
    }
  }
  double sum[kStats] = {};
  const bool by_wave = split > 1 && a.rows <= kWide / 64;
  const int per = by_wave ? kWide / 64 : kWide, me = by_wave ? threadIdx.x / 64 : threadIdx.x;
  for (long long r = (long long)blockIdx.x * per + me; r < a.rows; r += (long long)gridDim.x * per) {
    const float w = weight_of(a, r) * norm;
    float4 st = make_float4(0.f, 1.f, 0.f, 0.f);
    PolicyRow row{};
    if (w != 0.f) {
      if (split > 1) {
        const long long t = target_of(a.targets, a.bits, r);
        const float xt = target_logit<T>(x + r * stride, t, classes);
        st = by_wave ? join_parts<T>(parts, split, r, xt) : join_alone(parts, split, r, xt);
      } else {
        st = stat[r];
      }
      row = policy_row(a.p, w, st.w, st.z, a.old[r], a.advantages[r], a.ref != nullptr, a.ref != nullptr ? a.ref[r] : 0.f);
    }
    if (!by_wave || threadIdx.x % 64 == 0) {
      put_row(out, r, st, row.g, row.h);
#pragma unroll
      for (int i = 0; i < kStats; ++i) sum[i] += double(row.v[i]);
    }
  }
#pragma unroll
  for (int i = 0; i < kStats; ++i) {
    const float v = wave_sum(float(sum[i]));
    if (threadIdx.x % 64 == 0) waves[threadIdx.x / 64][i] = v;
  }
  __syncthreads();
  if (threadIdx.x < kStats) {
    double s = 0.0;
#pragma unroll
    for (int k = 0; k < kWide / 64; ++k) s += double(waves[k][threadIdx.x]);
    partial[(long long)threadIdx.x * gridDim.x + blockIdx.x] = float(s);
  }
}

// stats[i] = factor times the sum of partial[i][0 .. n - 1]: one workgroup, two
// waves a stat.  (A launch this small takes about as long as its instructions
// take to be fetched: 50 ns for each 64 bytes of them.  So no lane handles more
// than one stat, and the small kernels here keep their loops rolled.)
template <int STATS>
__global__ __launch_bounds__(128 * STATS) void k_total(const float* __restrict__ partial, int n, float factor,
                                                       float* __restrict__ stats) {
  __shared__ float part[2 * STATS];
  const int wave = threadIdx.x / 64, lane = threadIdx.x % 64;
  typedef float Four __attribute__((ext_vector_type(4), aligned(4)));
  const float* p = partial + (long long)(wave / 2) * n;
  const int quads = n / 4, me = wave % 2 * 64 + lane;
  double sum = 4 * quads + me < n ? double(p[4 * quads + me]) : 0.0;
#pragma unroll 8
  for (int j = me; j < quads; j += 128) {
    const Four v = reinterpret_cast<const Four*>(p)[j];
    sum += double((v[0] + v[1]) + (v[2] + v[3]));
  }
  const float v = wave_sum(float(sum));
  if (lane == 0) part[wave] = v;
  __syncthreads();
  if (threadIdx.x < STATS) stats[threadIdx.x] = (part[2 * threadIdx.x] + part[2 * threadIdx.x + 1]) * factor;
}

// The policy loss and its gradient in one pass over the logits: a row stays in
// the registers of its THREADS lanes, NC chunks each, from its load to its
// gradient's store.  Rows blockIdx, blockIdx + gridDim, ... of a workgroup;
// its rows' stats go into partial[.][blockIdx].  LONG: what the registers do
// not hold of a row is streamed for the statistics and read again (out of the
// Infinity Cache, which a row a CU fits) for the gradient.
//
// Bound by HBM, each logit read once and its gradient written once: 8192 rows of
// 4096 floats, 255 MB, in 49 us (5.2 TB/s), of 65536 bfloat16, 2.04 GB, in 380
// us (5.4 TB/s); statistics and gradient as two passes took 61 and 640 us.  The
// vector unit is 54 and 67 % busy.  So many chunks a lane as a row needs, that
// the loads of a whole row are in flight together; several workgroups a CU, so
// that one loads while another stores.
constexpr int fused_waves(int nc) { return nc <= 4 ? 8 : nc <= 8 ? 6 : nc <= 12 ? 5 : 4; }
template <class T, int WG, int THREADS, int NC, bool LONG, bool NT>
__global__ __launch_bounds__(WG) __attribute__((amdgpu_waves_per_eu(LONG ? 4 : fused_waves(NC)))) void k_policy_fused(
    PolicyArgs a, const typename T::Elem* x, long long stride, int classes, const double* __restrict__ sums, int groups,
    typename T::Elem* grad, long long grad_stride, RowOut out, float* __restrict__ partial) {
  constexpr int ROWS = WG / THREADS;
  __shared__ float slots[3 * (WG / 64)];
  __shared__ double acc[ROWS][kStats];  // each row's stats: too seldom to hold registers
  Group<THREADS> group{slots};
  const int lane = threadIdx.x % THREADS;
  const int sub = ROWS > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x / THREADS) : 0;
  // a row's target and weight, asked for while the last row (or the weights' sum) is worked on
  long long target = -1;
  float weight = 0.f;
  auto head = [&](long long r) {
    if (r >= a.rows) return;
    target = target_of(a.targets, a.bits, r);
    weight = a.weights != nullptr ? a.weights[r] : 1.f;
  };
  head((long long)blockIdx.x * ROWS + sub);
  __shared__ float own[WG / 64];
  float norm = 1.f;
  if (a.p.mean) norm = norm_of(a, sums != nullptr ? weight_total(sums, groups) : weight_all<WG>(a, own));
  if (threadIdx.x < ROWS * kStats) (&acc[0][0])[threadIdx.x] = 0.0;
  __syncthreads();
  const unsigned at = unsigned(lane) * 16u;
  for (long long r = (long long)blockIdx.x * ROWS + sub; r < a.rows; r += (long long)gridDim.x * ROWS) {
    const int t = uniform(target < 0 ? -1 : target < classes ? int(target) : classes);
    const float w = uniform(t < 0 ? 0.f : weight * norm);
    const typename T::Elem* row = x + r * stride;
    typename T::Elem* to = grad + r * grad_stride;
    head(r + (long long)gridDim.x * ROWS);
    const Cut<T> cut(row, classes);
    const typename T::Elem* body = row + cut.head;
    typename T::Elem* to_body = to + cut.head;
    const int one = cut.element(lane);
    const bool has_one = lane < cut.extra;
    auto chunk = [&](int c) { return c * THREADS + lane < cut.full; };
    if (w == 0.f) {
      float zero[T::kPer] = {};
#pragma unroll
      for (int c = 0; c < NC; ++c)
        if (chunk(c)) store_chunk_at<T>(to_body, c * THREADS * 16u, at, T::pack(zero));
      if constexpr (LONG)
        for (int c = NC * THREADS + lane; c < cut.full; c += THREADS)
          store_chunk<T>(to_body + (long long)c * T::kPer, T::pack(zero));
      if (has_one) to[one] = T::to(0.f);
      if (lane == 0) put_row(out, r, make_float4(0.f, 1.f, 0.f, 0.f), 0.f, 0.f);
      continue;
    }
    typename T::Raw raw[NC];
    // between two passes over the registers: without it the compiler keeps every
    // value's difference and exponential from one pass for the next, two or three
    // registers a value, and spills
    auto forget = [&] {
#pragma unroll
      for (int c = 0; c < NC; ++c) asm volatile("" : "+v"(raw[c]));
    };
#pragma unroll
    for (int c = 0; c < NC; ++c) raw[c] = typename T::Raw{};
#pragma unroll
    for (int c = 0; c < NC; ++c)
      if (chunk(c)) raw[c] = load_chunk_at<T, NT>(body, c * THREADS * 16u, at);
    const float last = has_one ? T::one(row[one]) : kNegMax;
    const float xt = uniform(target_logit<T>(row, t, classes));
    const float old = uniform(a.old[r]), adv = uniform(a.advantages[r]);
    const float ref = uniform(a.ref != nullptr ? a.ref[r] : 0.f);
    Run run = empty_run();  // of what is streamed
    if constexpr (LONG)
      stream<kAhead>(NC * THREADS + lane, cut.full, THREADS, [&]<int N, bool ALL>(int c) {
        run = merge(run, run_of<T, N, ALL>(body, c, THREADS, cut.full));
      });
    float m = fmaxf(run.m, last);
#pragma unroll
    for (int c = 0; c < NC; ++c)
      if (chunk(c)) {
#pragma unroll
        for (int i = 0; i < T::kPer; ++i) m = fmaxf(m, T::get(raw[c], i));
      }
    forget();
    m = uniform(group.max(m));
    float s = 0.f, u = 0.f;
    if constexpr (LONG) {
      const float d = below(run.m, m), f = exp_of(d);
      s = run.s * f;
      u = f * (run.u + d * run.s);
    }
    auto add = [&](float v) {
      const float d = v - m, e = exp_of(d);
      s += e;
      u += e * fmaxf(d, -1e30f);
    };
#pragma unroll
    for (int c = 0; c < NC; ++c)
      if (chunk(c)) {
#pragma unroll
        for (int i = 0; i < T::kPer; ++i) add(T::get(raw[c], i));
      }
    if (has_one) add(last);
    forget();
    group.sum(s, u);
    const float4 st = stat_of(Run{m, s, u}, xt);
    const PolicyRow p = policy_row(a.p, w, st.w, st.z, old, adv, a.ref != nullptr, ref);
    const float g = uniform(p.g * a.p.grad_scale);
    Slope sl = slope_of(m, s, st.z, g, p.h * a.p.grad_scale);
    sl.a = uniform(sl.a);
    sl.b = uniform(sl.b);
#pragma unroll
    for (int c = 0; c < NC; ++c)
      if (chunk(c)) {
        float y[T::kPer];
#pragma unroll
        for (int i = 0; i < T::kPer; ++i) y[i] = slope_value(sl, T::get(raw[c], i));
        store_chunk_at<T>(to_body, c * THREADS * 16u, at, T::pack(y));
      }
    if constexpr (LONG)
      stream<kAhead>(NC * THREADS + lane, cut.full, THREADS, [&]<int N, bool ALL>(int c) {
        slopes<T, N, ALL>(sl, body, to_body, c, THREADS, cut.full);
      });
    if (has_one) to[one] = T::to(slope_value(sl, last));
    // the lane that wrote the target's chunk writes the target again, with its g
    const int tc = cut.chunk_of(t);
    if (t < classes && (tc >= 0 ? tc % THREADS : cut.lane_of(t)) == lane) to[t] = T::to(slope_value(sl, xt) + g);
    if (lane == 0) {
      put_row(out, r, st, p.g, p.h);
#pragma unroll
      for (int i = 0; i < kStats; ++i) acc[sub][i] += double(p.v[i]);
    }
  }
  __syncthreads();
  if (threadIdx.x < kStats) {
    double v = 0.0;
#pragma unroll
    for (int q = 0; q < ROWS; ++q) v += acc[q][threadIdx.x];
    partial[(long long)threadIdx.x * gridDim.x + blockIdx.x] = float(v);
  }
}

// What one wave does for the rows of a tile (up to 64), a lane for each: the
// row's loss out of its (M, S, U, x_t), its slope, and the stats.  Left to every
// wave for its own row, that arithmetic (two exponentials, two logarithms, three
// quotients) is most of its work: 20000 rows of 257 bfloat16 classes took 33 us
// with a wave per row.
struct RowIn {
  float w, old, adv, ref;
};
__device__ __forceinline__ RowIn row_in(const PolicyArgs& a, long long r, bool any) {
  RowIn v{0.f, 0.f, 0.f, 0.f};
  if (any) {
    v.w = weight_of(a, r);
    v.old = a.old[r];
    v.adv = a.advantages[r];
    if (a.ref != nullptr) v.ref = a.ref[r];
  }
  return v;
}
__device__ __forceinline__ void tile_rows(const PolicyArgs& a, long long base, int rows, int lane, float norm, RowIn in,
                                          const float4* stat, float4* slope, int* target, const RowOut& out,
                                          double& acc) {
  if (gridDim.x == 1 && a.p.mean) {  // these are all rows
    double total = double(in.w);
#pragma unroll 1
    for (int o = 32; o > 0; o >>= 1) total += __shfl_xor(total, o);
    norm = norm_of(a, total);
  }
  const float w = in.w * norm;
  float4 st = make_float4(0.f, 1.f, 0.f, 0.f), sl = make_float4(0.f, 0.f, 0.f, 0.f);
  PolicyRow p{};
  if (w != 0.f) {
    const float4 z = stat[lane];
    st = stat_of(Run{z.x, z.y, z.z}, z.w);
    p = policy_row(a.p, w, st.w, st.z, in.old, in.adv, a.ref != nullptr, in.ref);
    const float g = p.g * a.p.grad_scale;
    const Slope k = slope_of(st.x, st.y, st.z, g, p.h * a.p.grad_scale);
    sl = make_float4(k.a, k.b, g, 0.f);
  }
  if (lane < rows) {
    put_row(out, base + lane, st, p.g, p.h);
    slope[lane] = sl;
    if (w == 0.f) target[lane] = -1;
  }
#pragma unroll
  for (int i = 0; i < kStats; ++i) {
    const float v = wave_sum(p.v[i]);
    if (lane == i) acc += double(v);
  }
}

// One pass over rows of at most 64 chunks: 16 lanes a row, NC chunks each, four
// rows a wave.  A wave for a row would spend its instructions on lanes that have
// nothing to do and on reductions over 64 lanes: 64 rows of 256 floats, which
// one workgroup takes (a launch instead of three), took 9.3 us that way, bound by
// the one CU's vector unit, and take 5.4 this way.
template <class T, int WAVES, int NC>
__global__ __launch_bounds__(64 * WAVES) void k_policy_short(
    PolicyArgs a, const typename T::Elem* x, long long stride, int classes, const double* __restrict__ sums, int groups,
    typename T::Elem* grad, long long grad_stride, RowOut out, float* __restrict__ partial) {
  constexpr int ROWS = WAVES * 4;
  __shared__ float4 stat[ROWS];   // M, S, U, x_t
  __shared__ float4 slope[ROWS];  // a, b, g
  __shared__ int target[ROWS];    // -1: the row takes no part
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int mine = threadIdx.x / 16, part = threadIdx.x % 16;
  float norm = 1.f;
  __shared__ float own[WAVES];
  if (gridDim.x > 1 && a.p.mean) norm = norm_of(a, sums != nullptr ? weight_total(sums, groups) : weight_all<64 * WAVES>(a, own));
  double acc = 0.0;  // lane i of wave 0: stat i
  for (long long base = (long long)blockIdx.x * ROWS; base < a.rows; base += (long long)gridDim.x * ROWS) {
    const int rows = a.rows - base < ROWS ? int(a.rows - base) : ROWS;
    RowIn in{};
    if (wave == 0) in = row_in(a, base + lane, lane < rows);
    const bool any = mine < rows;
    const long long r = any ? base + mine : base;
    const typename T::Elem* row = x + r * stride;
    const Cut<T, false> cut(row, classes);
    const float weight = a.weights != nullptr ? a.weights[r] : 1.f;
    const long long tt = target_of(a.targets, a.bits, r);
    const int t = any && tt >= 0 && weight != 0.f ? (tt < classes ? int(tt) : classes) : -1;
    // the one workgroup of a small call does not wait for the targets before it
    // asks for the logits; what it gets of an idle row is not looked at
    const bool ask = WAVES > 8 ? any : t >= 0;
    const bool has_one = part < cut.extra;
    typename T::Raw raw[NC];
    float one = kNegMax, xt = __builtin_nanf("");
    if (ask) {
#pragma unroll
      for (int c = 0; c < NC; ++c)
        if (c * 16 + part < cut.full) raw[c] = load_chunk<T>(row + cut.head + (c * 16 + part) * T::kPer);
      if (has_one) one = T::one(row[cut.element(part)]);
    }
    if (t >= 0 && t < classes) xt = T::one(row[t]);
    if (part == 0 && any) target[mine] = t;
    if (t >= 0) {
      float m = fmaxf(one, kNegMax);
#pragma unroll
      for (int c = 0; c < NC; ++c)
        if (c * 16 + part < cut.full) {
#pragma unroll
          for (int e = 0; e < T::kPer; ++e) m = fmaxf(m, T::get(raw[c], e));
        }
      m = over_16(m, [](float p, float q) { return fmaxf(p, q); });
      float s = 0.f, u = 0.f;
      auto add = [&](float z) {
        const float d = z - m, e = exp_of(d);
        s += e;
        u += e * fmaxf(d, -1e30f);
      };
#pragma unroll
      for (int c = 0; c < NC; ++c)
        if (c * 16 + part < cut.full) {
#pragma unroll
          for (int e = 0; e < T::kPer; ++e) add(T::get(raw[c], e));
        }
      if (has_one) add(one);
      s = over_16(s, [](float p, float q) { return p + q; });
      u = over_16(u, [](float p, float q) { return p + q; });
      if (part == 0) stat[mine] = make_float4(m, s, u, xt);
    }
    __syncthreads();
    if (wave == 0) tile_rows(a, base, rows, lane, norm, in, stat, slope, target, out, acc);
    __syncthreads();
    if (any) {
      const bool on = target[mine] >= 0;
      typename T::Elem* to = grad + r * grad_stride;
      const float4 k = slope[mine], z = stat[mine];
      const Slope sl{z.x, k.x, k.y};
#pragma unroll
      for (int c = 0; c < NC; ++c)
        if (c * 16 + part < cut.full) {
          float y[T::kPer] = {};
          if (on) {
#pragma unroll
            for (int e = 0; e < T::kPer; ++e) y[e] = slope_value(sl, T::get(raw[c], e));
          }
          store_chunk<T>(to + cut.head + (c * 16 + part) * T::kPer, T::pack(y));
        }
      if (has_one) to[cut.element(part)] = T::to(on ? slope_value(sl, one) : 0.f);
      // the lane that wrote the target's chunk writes the target again, with its g
      if (on && t < classes) {
        const int tc = cut.chunk_of(t);
        if ((tc >= 0 ? tc % 16 : cut.lane_of(t)) == part) to[t] = T::to(slope_value(sl, z.w) + k.z);
      }
    }
    __syncthreads();  // before the next tile's rows
  }
  if (wave == 0 && lane < kStats) partial[(long long)lane * gridDim.x + blockIdx.x] = float(acc);
}

// The same for rows of 65 to 256 chunks: WAVES waves hold RPW rows each in LDS.
template <class T, int WAVES, int RPW, int NC>
__global__ __launch_bounds__(64 * WAVES) void k_policy_tile(
    PolicyArgs a, const typename T::Elem* x, long long stride, int classes, const double* __restrict__ sums, int groups,
    typename T::Elem* grad, long long grad_stride, RowOut out, float* __restrict__ partial) {
  constexpr int ROWS = WAVES * RPW;
  typedef typename T::Raw Slot __attribute__((aligned(16)));
  __shared__ Slot held[ROWS][NC][64];
  __shared__ float rest[ROWS][64];  // the element outside of the chunks that is a lane's
  __shared__ float4 stat[ROWS];     // M, S, U, x_t
  __shared__ float4 slope[ROWS];    // a, b, g
  __shared__ int target[ROWS];      // -1: the row takes no part
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const unsigned at = unsigned(lane) * 16u;
  float norm = 1.f;
  __shared__ float own[WAVES];
  if (gridDim.x > 1 && a.p.mean) norm = norm_of(a, sums != nullptr ? weight_total(sums, groups) : weight_all<64 * WAVES>(a, own));
  double acc = 0.0;  // lane i of wave 0: stat i
  for (long long base = (long long)blockIdx.x * ROWS; base < a.rows; base += (long long)gridDim.x * ROWS) {
    const int rows = a.rows - base < ROWS ? int(a.rows - base) : ROWS;
    const int first = wave * RPW, last = min(first + RPW, rows);
    RowIn in{};  // asked for ahead of the rows' arithmetic
    if (wave == 0) in = row_in(a, base + lane, lane < rows);
    // the wave's rows' targets, a lane for each
    int own = -1;
    if (first + lane < last) {
      const float weight = a.weights != nullptr ? a.weights[base + first + lane] : 1.f;
      const long long tt = target_of(a.targets, a.bits, base + first + lane);
      if (tt >= 0 && weight != 0.f) own = tt < classes ? int(tt) : classes;
    }
    typename T::Raw raw[RPW][NC];
    float extra[RPW];
#pragma unroll
    for (int q = 0; q < RPW; ++q) {
      // the one workgroup of a small call does not wait for the targets before it
      // asks for the logits; what it gets of an idle row is not looked at
      if (first + q < last && (WAVES > 8 || __builtin_amdgcn_readlane(own, q) >= 0)) {
        const typename T::Elem* row = x + (base + first + q) * stride;
        const Cut<T> cut(row, classes);
#pragma unroll
        for (int c = 0; c < NC; ++c)
          if (c * 64 + lane < cut.full) raw[q][c] = load_chunk_at<T>(row + cut.head, c * 1024u, at);
        if (lane < cut.extra) extra[q] = T::one(row[cut.element(lane)]);
      }
    }
    if (first + lane < last) target[first + lane] = own;
#pragma unroll
    for (int q = 0; q < RPW; ++q) {
      if (first + q >= last) continue;
#pragma unroll
      for (int c = 0; c < NC; ++c) held[first + q][c][lane] = raw[q][c];
      rest[first + q][lane] = extra[q];
    }
    wave_sync();  // the rows' targets and a target's logit are other lanes'
#pragma unroll 1
    for (int i = first; i < last; ++i) {
      const int t = uniform(target[i]);
      if (t < 0) continue;
      const typename T::Elem* row = x + (base + i) * stride;
      const Cut<T> cut(row, classes);
      const bool has_one = lane < cut.extra;
      const float one = has_one ? rest[i][lane] : kNegMax;
      const int tc = cut.chunk_of(t);
      const typename T::Elem* held_row = reinterpret_cast<const typename T::Elem*>(held[i]);
      const float xt = t >= classes ? __builtin_nanf("") : tc >= 0 ? T::one(held_row[t - cut.head]) : rest[i][cut.lane_of(t)];
      typename T::Raw v[NC];
      float m = fmaxf(one, kNegMax);
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        v[c] = held[i][c][lane];
        if (c * 64 + lane < cut.full) {
#pragma unroll
          for (int e = 0; e < T::kPer; ++e) m = fmaxf(m, T::get(v[c], e));
        }
      }
      m = wave_max(m);
      float s = 0.f, u = 0.f;
      auto add = [&](float z) {
        const float d = z - m, e = exp_of(d);
        s += e;
        u += e * fmaxf(d, -1e30f);
      };
#pragma unroll
      for (int c = 0; c < NC; ++c)
        if (c * 64 + lane < cut.full) {
#pragma unroll
          for (int e = 0; e < T::kPer; ++e) add(T::get(v[c], e));
        }
      if (has_one) add(one);
      s = wave_sum(s);
      u = wave_sum(u);
      if (lane == 0) stat[i] = make_float4(m, s, u, xt);
    }
    __syncthreads();
    if (wave == 0) tile_rows(a, base, rows, lane, norm, in, stat, slope, target, out, acc);
    __syncthreads();
#pragma unroll 1
    for (int i = first; i < last; ++i) {
      const int t = uniform(target[i]);
      typename T::Elem* to = grad + (base + i) * grad_stride;
      const Cut<T> cut(x + (base + i) * stride, classes);
      const float4 k = slope[i], z = stat[i];
      const Slope sl{z.x, k.x, k.y};
      // of a row that takes no part nothing but its length is looked at
#pragma unroll
      for (int c = 0; c < NC; ++c)
        if (c * 64 + lane < cut.full) {
          float y[T::kPer] = {};
          if (t >= 0) {
            const typename T::Raw v = held[i][c][lane];
#pragma unroll
            for (int e = 0; e < T::kPer; ++e) y[e] = slope_value(sl, T::get(v, e));
          }
          store_chunk_at<T>(to + cut.head, c * 1024u, at, T::pack(y));
        }
      if (lane < cut.extra) to[cut.element(lane)] = T::to(t >= 0 ? slope_value(sl, rest[i][lane]) : 0.f);
      if (t >= 0 && t < classes) {
        const int tc = cut.chunk_of(t);
        if ((tc >= 0 ? tc % 64 : cut.lane_of(t)) == lane) to[t] = T::to(slope_value(sl, z.w) + k.z);
      }
    }
    __syncthreads();  // before the next tile's rows
  }
  if (wave == 0 && lane < kStats) partial[(long long)lane * gridDim.x + blockIdx.x] = float(acc);
}

// ----------------------------------------------------- the preference loss
__device__ __forceinline__ long long offset_of(const void* offsets, int bits, long long s, long long rows) {
  const long long o = bits == 64 ? static_cast<const long long*>(offsets)[s]
                                 : (long long)static_cast<const int*>(offsets)[s];
  return o < 0 ? 0 : o > rows ? rows : o;
}

constexpr int kPairStats = 5;
struct PairArgs {
  const void *targets, *offsets;
  int bits, offset_bits;
  const float* ref;
  long long rows, pairs;
  float beta, smoothing;
};

// Sum of logp - logp_ref over rows from .. to - 1, by a group of n threads.
__device__ __forceinline__ double excess(const PairArgs& a, const float4* __restrict__ stat, long long from, long long to,
                                         int lane, int n) {
  double v = 0.0;
#pragma unroll 4
  for (long long r = from + lane; r < to; r += n) {
    const double d = double(stat[r].w) - double(a.ref[r]);  // (asked for along with the target)
    v += target_of(a.targets, a.bits, r) >= 0 ? d : 0.0;
  }
  return v;
}

// Rewards, margin and loss of pairs, and dL/dlogp of their rows, whose g and h
// are 0 before it: 5 to 7 us of latency, beside passes over the logits.  WG / GROUP pairs a workgroup at a time: a wave each in the
// one workgroup of a call with few pairs, which writes the stats itself, else
// a workgroup each, whose sums go into partial[.][blockIdx].
template <int WG, int GROUP>
__global__ __launch_bounds__(WG) void k_pairs(PairArgs a, const float4* __restrict__ stat, float* __restrict__ g,
                                              float* __restrict__ partial) {
  constexpr int PAIRS = WG / GROUP;
  __shared__ double acc[PAIRS][kPairStats];
  __shared__ double part[WG / 64];
  const int lane = threadIdx.x % GROUP, mine = threadIdx.x / GROUP;
  double sum[kPairStats] = {};
  for (long long p = (long long)blockIdx.x * PAIRS + mine; p < a.pairs; p += (long long)gridDim.x * PAIRS) {
    const long long o0 = offset_of(a.offsets, a.offset_bits, 2 * p, a.rows);
    const long long o1 = offset_of(a.offsets, a.offset_bits, 2 * p + 1, a.rows);
    const long long o2 = offset_of(a.offsets, a.offset_bits, 2 * p + 2, a.rows);
    double v0 = excess(a, stat, o0, o1, lane, GROUP), v1 = excess(a, stat, o1, o2, lane, GROUP);
    if constexpr (GROUP == 64) {
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) {
        v0 += __shfl_xor(v0, o);
        v1 += __shfl_xor(v1, o);
      }
    } else {
      v0 = total_of<WG>(v0, part);
      v1 = total_of<WG>(v1, part);
    }
    const float good = float(a.beta * v0), bad = float(a.beta * v1), m = float(a.beta * (v0 - v1)), e = a.smoothing;
    // -log sigmoid(+-m) and sigmoid(+-m) out of one exponential, z = exp(-|m|) <= 1.
    // A NaN margin is no win, and gives NaN slopes.  An infinite one (a token of
    // probability 0) costs nothing on the side that the smoothing leaves out.
    const float z = expf(-fabsf(m)), q = 1.f / (1.f + z);
    const float share = m < 0.f ? 1.f - e : e;
    const float loss = log1pf(z) + (share > 0.f ? share * fabsf(m) : 0.f);
    const float up = m < 0.f ? z * q : q, down = m < 0.f ? q : z * q;
    const float slope = (e * up - (1.f - e) * down) * (a.beta / float(a.pairs));
#pragma unroll 4
    for (long long r = o0 + lane; r < o2; r += GROUP)
      if (target_of(a.targets, a.bits, r) >= 0) g[r] = r < o1 ? slope : -slope;
    const float v[kPairStats] = {loss, m > 0.f ? 1.f : 0.f, m, good, bad};
#pragma unroll
    for (int i = 0; i < kPairStats; ++i) sum[i] += double(v[i]);
  }
  if (lane == 0)
#pragma unroll
    for (int i = 0; i < kPairStats; ++i) acc[mine][i] = sum[i];
  __syncthreads();
  if (threadIdx.x < kPairStats) {
    double s = 0.0;
#pragma unroll
    for (int w = 0; w < PAIRS; ++w) s += acc[w][threadIdx.x];
    if (PAIRS > 1) s = a.pairs > 0 ? s / double(a.pairs) : 0.0;
    partial[(long long)threadIdx.x * gridDim.x + blockIdx.x] = float(s);
  }
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
// grad_logits: the logits themselves, or memory apart from them: before or after
// them, or other columns of the same wider rows.
bool grad_ok(const void* logits, int64_t stride, const void* grad, int64_t grad_stride, int32_t dtype, int64_t rows,
             int32_t classes) {
  const size_t eb = dtype_bytes(dtype);
  if (grad_stride < classes || grad_stride > (int64_t(1) << 40) || !aligned_to(grad, eb)) return false;
  if (grad == logits) return grad_stride == stride;
  const Span x = span_of(logits, rows, stride, classes, eb), g = span_of(grad, rows, grad_stride, classes, eb);
  if (x.b <= g.a || g.b <= x.a) return true;
  if (grad_stride != stride) return false;
  const uintptr_t row = uintptr_t(stride) * eb, width = uintptr_t(classes) * eb;
  const uintptr_t at = g.a >= x.a ? (g.a - x.a) % row : (row - (x.a - g.a) % row) % row;
  return at >= width && at + width <= row;
}
bool floats_ok(std::initializer_list<const void*> must, std::initializer_list<const void*> may) {
  for (const void* p : must)
    if (p == nullptr || !aligned_to(p, 4)) return false;
  for (const void* p : may)
    if (!aligned_to(p, 4)) return false;
  return true;
}

size_t up256(size_t b) { return (b + 255) & ~size_t(255); }
// Workgroups that share a row.  One, but for few long rows, which are cut into
// parts of at least 4096 values, up to about four workgroups a CU.  Parts cost
// a launch that joins them and a second pass over the logits: 80 rows of 20000
// floats take 14 us whole and 20 in parts, 40 rows of 100000 24 and 25, 40 rows
// of 200000 bfloat16 39 and 25; past the 256 KB that a CU's registers hold of a
// row, 80 rows of 200000 41 and 30, 160 rows 44 and 45.
int split_of(int64_t rows, int32_t classes, int32_t dtype) {
  const int64_t few = int64_t(classes) * int64_t(dtype_bytes(dtype)) > 262144 ? 128 : 64;
  if (rows < 1 || rows >= few) return 1;
  const int64_t parts = std::min<int64_t>({64, 1024 / rows, classes / 4096});
  return int(std::max<int64_t>(1, parts));
}
// Workgroups (and so partial stats) of the kernels that sum the policy's stats.
constexpr int64_t kMaxPartials = 8192;
// Bytes of logits from which on the one pass over them reads them with the hint
// that no cache need keep them (they are past half of the Infinity Cache, and
// nothing reads them again): 8192 rows of 65536 bfloat16 394 us instead of 400,
// 2048 rows of 4096 floats, 34 MB, 20 us without it and 22 with it.  Gradients
// are always written with the hint: 8192 rows of 4096 61 -> 57 us, 2048 rows
// 23 -> 20 us; the cascade's backward that reads them next takes as much
// longer, so that the two together are the same within 2 % at any size.
constexpr double kKeepBytes = 128e6;

struct Workspace {
  size_t stat, grads, parts, sums, partial, total;
};
Workspace layout(int64_t rows, int32_t classes, int32_t dtype, int64_t pairs) {
  Workspace w{};
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t o = at;
    at += up256(bytes);
    return o;
  };
  const int split = split_of(rows, classes, dtype);
  w.stat = take(size_t(rows) * sizeof(float4));
  w.grads = take(size_t(rows) * 2 * sizeof(float));
  w.parts = take(split > 1 ? size_t(rows) * split * sizeof(float4) : 0);
  w.sums = take(kWeightSums * sizeof(double));
  w.partial = take(size_t(std::min(std::max(rows, pairs), kMaxPartials)) * kStats * sizeof(float));
  w.total = at;
  return w;
}
// Of the log-probabilities alone: the parts of rows, where they come in parts.
size_t logprob_bytes(int64_t rows, int32_t classes, int32_t dtype) {
  const int split = split_of(rows, classes, dtype);
  return up256(std::max<size_t>(1, split > 1 ? size_t(rows) * split * sizeof(float4) : 0));
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

// The logits as every launch takes them.
struct Logits {
  const void* x;
  int32_t dtype;
  int64_t stride;
  const void* targets;
  int32_t bits;
  int64_t rows;
  int32_t classes;
};

// Workgroups of a launch over `items`: a grid holds fewer than 2^32 lanes.
unsigned grid_for(unsigned items) { return std::min(items, 1u << 22); }

// Chunks up to which a wave takes a row in the passes over logits; up to a round of
// 16 lanes those do.  A workgroup a row is bound by how fast workgroups begin, some
// 700 a us: 40000 rows, statistics and gradient, of 78 floats take 16 us for 95, of
// 600 47 for 99, of 1500 104 for 117, 10000 of 78 14 for 28, of 2040 42 for 41.
constexpr int64_t kWaveChunks = 512;

// Row statistics into `out`; rows in parts (split > 1) leave their parts only.
int launch_stats(const Logits& l, int split, const RowOut& out, float4* parts, hipStream_t s) {
  with_type(l.dtype, [&]<class T>() {
    auto go = [&]<int LANES>() {
      const unsigned items = unsigned(l.rows * split);
      using Rows = Share<LANES>;
      hipLaunchKernelGGL((k_row_stats<T, LANES>), dim3(grid_for((items + Rows::ROWS - 1) / Rows::ROWS)), dim3(Rows::WG), 0, s,
                         static_cast<const typename T::Elem*>(l.x), (long long)l.stride, l.targets, l.bits, l.classes,
                         split, items, out, parts);
    };
    // as many lanes as ask for a part of a row in one or two rounds of kAhead chunks
    // (19.9 k rows of 32768 bfloat16: 250 us with 256 lanes, 238 with 512)
    const int64_t chunks = l.classes / T::kPer / split;
    if (chunks <= 16 * kAhead) go.template operator()<16>();
    else if (chunks <= kWaveChunks) go.template operator()<64>();
    else if (chunks <= 2 * kAhead * kThreads) go.template operator()<kThreads>();
    else go.template operator()<512>();
  });
  return done();
}
// The same, joined where they came in parts.
int launch_values(const Logits& l, const RowOut& out, float4* parts, hipStream_t s) {
  const int split = split_of(l.rows, l.classes, l.dtype);
  const int rc = launch_stats(l, split, out, parts, s);
  if (rc != ACDC_OK || split == 1) return rc;
  with_type(l.dtype, [&]<class T>() {
    constexpr int per = kThreads / 64;
    hipLaunchKernelGGL(k_row_join<T>, dim3(unsigned((l.rows + per - 1) / per)), dim3(kThreads), 0, s,
                       static_cast<const typename T::Elem*>(l.x), (long long)l.stride, l.targets, l.bits, l.classes,
                       parts, split, (long long)l.rows, out);
  });
  return done();
}
int launch_grad(const Logits& l, const float4* stat, const float* g, const float* h, const float* scale,
                float scale_host, void* grad, int64_t grad_stride, hipStream_t s) {
  const int split = split_of(l.rows, l.classes, l.dtype);
  with_type(l.dtype, [&]<class T>() {
    const unsigned items = unsigned(l.rows * split);
    auto go = [&]<int LANES>() {
      constexpr unsigned per = Share<LANES>::ROWS;
      hipLaunchKernelGGL((k_row_grad<T, LANES>), dim3(grid_for((items + per - 1) / per)), dim3(kThreads), 0, s,
                         static_cast<const typename T::Elem*>(l.x), (long long)l.stride, l.targets, l.bits, l.classes,
                         stat, g, h, scale, scale_host, static_cast<typename T::Elem*>(grad), (long long)grad_stride,
                         split, items);
    };
    const int64_t chunks = l.classes / T::kPer / split;
    if (chunks <= 16 * kAhead) go.template operator()<16>();
    else if (chunks <= kWaveChunks) go.template operator()<64>();
    else go.template operator()<kThreads>();
  });
  return done();
}

// f.template operator()<THREADS, NC, LONG>() for the fewest lanes and registers
// that hold a row of `chunks` chunks; LONG where none do.  A workgroup of 1024
// lanes has a CU for itself, so that nothing else runs while it loads or stores.
// Rows of bfloat16, with twice the values to work on for each byte, are better
// off with two workgroups of 512 and a part of the row read twice: 4096 rows of
// 131072 take 438 us against 485, 3000 rows of 70000 185 against 224.  Rows of
// floats are not: 2048 of 65536 216 against 205, 512 of 300000 341 against 288.
template <class T, class F>
void with_row_shape(int chunks, F&& f) {
  if (chunks <= 16) f.template operator()<16, 1, false>();
  else if (chunks <= 32) f.template operator()<16, 2, false>();
  else if (chunks <= 64) f.template operator()<16, 4, false>();
  else if (chunks <= 128) f.template operator()<64, 2, false>();
  else if (chunks <= 256) f.template operator()<64, 4, false>();
  else if (chunks <= 512) f.template operator()<64, 8, false>();
  else if (chunks <= 1024) f.template operator()<256, 4, false>();
  else if (chunks <= 2048) f.template operator()<256, 8, false>();
  else if (chunks <= 3072) f.template operator()<256, 12, false>();
  else if (chunks <= 4096) f.template operator()<256, 16, false>();
  else if (chunks <= 8192) f.template operator()<512, 16, false>();
  else if constexpr (T::kPer == 8) f.template operator()<512, 12, true>();
  else if (chunks <= 16384) f.template operator()<1024, 16, false>();
  else f.template operator()<1024, 12, true>();
}

}  // namespace
}  // namespace acdc

using namespace acdc;

extern "C" size_t acdc_logprob_workspace_size(int64_t rows, int32_t classes, int32_t dtype) {
  return sizes_ok(rows, classes, dtype) ? logprob_bytes(rows, classes, dtype) : 0;
}

extern "C" int acdc_logprob_forward(const void* logits, int32_t dtype, int64_t stride, const void* targets,
                                    int32_t target_bits, int64_t rows, int32_t classes, float* logp, float* entropy,
                                    float* saved, void* workspace, size_t workspace_bytes, acdc_stream_t stream) {
  int rc;
  if (!logits_ok(logits, dtype, stride, targets, target_bits, rows, classes, &rc)) return rc;
  if (rows == 0) return ACDC_OK;
  if (!floats_ok({logp}, {entropy}) || !aligned_to(saved, 16) || !aligned_to(workspace, 16)) return ACDC_ERR_INVALID_ARG;
  if (workspace == nullptr || workspace_bytes < logprob_bytes(rows, classes, dtype)) return ACDC_ERR_WORKSPACE;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  const Logits l{logits, dtype, stride, targets, target_bits, rows, classes};
  const RowOut out{logp, entropy, reinterpret_cast<float4*>(saved), nullptr, nullptr};
  return launch_values(l, out, static_cast<float4*>(workspace), s);
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
  const Logits l{logits, dtype, stride, targets, target_bits, rows, classes};
  return launch_grad(l, reinterpret_cast<const float4*>(saved), grad_logp, grad_entropy, scale, 1.f, grad_logits,
                     grad_stride, reinterpret_cast<hipStream_t>(stream));
}

extern "C" size_t acdc_policy_workspace_size(int64_t rows, int32_t classes, int32_t dtype) {
  return sizes_ok(rows, classes, dtype) ? layout(rows, classes, dtype, 0).total : 0;
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
  const Workspace w = layout(rows, classes, dtype, 0);
  if (w.total > 0 && (workspace == nullptr || workspace_bytes < w.total)) return ACDC_ERR_WORKSPACE;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  char* ws = static_cast<char*>(workspace);
  const Logits l{logits, dtype, stride, targets, target_bits, rows, classes};
  const PolicyArgs a{targets, target_bits, logp_old, logp_ref, advantages, weights, rows, p};
  double* sums = reinterpret_cast<double*>(ws + w.sums);
  float* partial = reinterpret_cast<float*>(ws + w.partial);
  float4* parts = reinterpret_cast<float4*>(ws + w.parts);
  const int groups = rows > 0 ? int((rows + weight_group(rows) - 1) / weight_group(rows)) : 0;
  auto sum_weights = [&] {
    if (p.mean != 0) hipLaunchKernelGGL(k_weight_sums, dim3(unsigned(groups)), dim3(kThreads), 0, s, a, sums);
  };
  auto sum_stats = [&](unsigned blocks) {
    hipLaunchKernelGGL(k_total<kStats>, dim3(1), dim3(128 * kStats), 0, s, partial, int(blocks), 1.f, stats);
  };

  // Enough rows to fill the card, or rows of a wave each: one pass.
  const int split = split_of(rows, classes, dtype);
  if (rows > 0 && grad_logits != nullptr && split == 1) {
    with_type(dtype, [&]<class T>() {
      with_row_shape<T>(classes / T::kPer, [&]<int THREADS, int NC, bool LONG>() {
        const RowOut out{logp, nullptr, reinterpret_cast<float4*>(saved), row_grads,
                         row_grads != nullptr ? row_grads + rows : nullptr};
        auto go = [&](auto kernel, unsigned blocks, int wg, float* to) {
          hipLaunchKernelGGL(kernel, dim3(blocks), dim3(wg), 0, s, a, static_cast<const typename T::Elem*>(logits),
                             (long long)stride, classes, rows * blocks > kOwnWeights ? sums : nullptr, groups, static_cast<typename T::Elem*>(grad_logits),
                             (long long)grad_stride, out, to);
        };
        auto blocks_of = [&](int per) { return unsigned(std::min<int64_t>((rows + per - 1) / per, kMaxPartials)); };
        // one workgroup's rows: a launch instead of three
        auto tiles = [&](auto one, int most, auto many, int each) {
          if (rows <= most) {
            go(one, 1, 1024, stats);
          } else {
            const unsigned blocks = blocks_of(each);
            if (rows * blocks > kOwnWeights) sum_weights();
            go(many, blocks, 512, partial);
            sum_stats(blocks);
          }
        };
        if constexpr (THREADS == 16) {
          tiles(k_policy_short<T, 16, NC>, 64, k_policy_short<T, 8, NC>, 32);
        } else if constexpr (THREADS == 64 && NC <= 4) {
          constexpr int RPW = 4 / NC;
          tiles(k_policy_tile<T, 16, RPW, NC>, 16 * RPW, k_policy_tile<T, 8, RPW, NC>, 8 * RPW);
        } else {
          constexpr int WG = THREADS < kThreads ? kThreads : THREADS;
          const unsigned blocks = blocks_of(WG / THREADS);
          if (rows * blocks > kOwnWeights) sum_weights();
          if (double(rows) * double(stride) * sizeof(typename T::Elem) >= kKeepBytes)
            go(k_policy_fused<T, WG, THREADS, NC, LONG, true>, blocks, WG, partial);
          else
            go(k_policy_fused<T, WG, THREADS, NC, LONG, false>, blocks, WG, partial);
          sum_stats(blocks);
        }
      });
    });
    return done();
  }

  float4* stat = saved != nullptr ? reinterpret_cast<float4*>(saved) : reinterpret_cast<float4*>(ws + w.stat);
  float* grads = row_grads != nullptr ? row_grads : reinterpret_cast<float*>(ws + w.grads);
  if (rows > 0) {
    rc = launch_stats(l, split, RowOut{nullptr, nullptr, stat, nullptr, nullptr}, parts, s);
    if (rc != ACDC_OK) return rc;
  }
  const RowOut out{logp, nullptr, split > 1 ? stat : nullptr, grads, grads + rows};
  with_type(dtype, [&]<class T>() {
    auto go = [&](unsigned blocks, float* to) {
      hipLaunchKernelGGL(k_policy_rows<T>, dim3(blocks), dim3(kWide), 0, s, a, static_cast<const typename T::Elem*>(logits),
                         (long long)stride, classes, parts, split, sums, groups, stat, out, to);
    };
    if (rows <= kWide) {
      go(1, stats);
    } else {
      const unsigned blocks = unsigned(std::min<int64_t>((rows + kWide - 1) / kWide, kMaxPartials / 8));
      sum_weights();
      go(blocks, partial);
      sum_stats(blocks);
    }
  });
  rc = done();
  if (rc != ACDC_OK || rows == 0 || grad_logits == nullptr) return rc;
  return launch_grad(l, stat, grads, grads + rows, nullptr, p.grad_scale, grad_logits, grad_stride, s);
}

extern "C" size_t acdc_preference_workspace_size(int64_t rows, int32_t classes, int32_t dtype, int64_t pairs) {
  if (!sizes_ok(rows, classes, dtype) || pairs < 0 || pairs > 0x3fffffff) return 0;
  return layout(rows, classes, dtype, pairs).total;
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
  const Workspace w = layout(rows, classes, dtype, pairs);
  if (w.total > 0 && (workspace == nullptr || workspace_bytes < w.total)) return ACDC_ERR_WORKSPACE;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  char* ws = static_cast<char*>(workspace);
  float4* stat = saved != nullptr ? reinterpret_cast<float4*>(saved) : reinterpret_cast<float4*>(ws + w.stat);
  float* grads = row_grads != nullptr ? row_grads : reinterpret_cast<float*>(ws + w.grads);
  float* partial = reinterpret_cast<float*>(ws + w.partial);
  const Logits l{logits, dtype, stride, targets, target_bits, rows, classes};
  if (rows > 0) {
    // with g and h of 0 for every row; the pairs then give their rows a g
    rc = launch_values(l, RowOut{logp, nullptr, stat, grads, grads + rows}, reinterpret_cast<float4*>(ws + w.parts), s);
    if (rc != ACDC_OK) return rc;
  }
  // one workgroup, a wave for each pair, saves the launch that adds the stats
  const PairArgs a{targets, offsets, target_bits, offset_bits, logp_ref, rows, pairs, p.beta, p.label_smoothing};
  if (pairs <= kWide / 64) {
    hipLaunchKernelGGL((k_pairs<kWide, 64>), dim3(1), dim3(kWide), 0, s, a, stat, grads, stats);
  } else {
    const unsigned blocks = unsigned(std::min<int64_t>(pairs, kMaxPartials));
    hipLaunchKernelGGL((k_pairs<kThreads, kThreads>), dim3(blocks), dim3(kThreads), 0, s, a, stat, grads, partial);
    hipLaunchKernelGGL(k_total<kPairStats>, dim3(1), dim3(128 * kPairStats), 0, s, partial, int(blocks), float(1.0 / double(pairs)),
                       stats);
  }
  rc = done();
  if (rc != ACDC_OK || rows == 0 || grad_logits == nullptr) return rc;
  return launch_grad(l, stat, grads, grads + rows, nullptr, p.grad_scale, grad_logits, grad_stride, s);
}
