// Losses over a vocabulary whose logits are never stored (acdc_train_lm.h).
//
// Mathematics.  With x = hidden weight^T, a row enters a loss through logp =
// x_t - M - log S only, M = max_v x_v, S = sum_v exp(x_v - M).  The first pass
// computes the logits tile by tile on the matrix cores and leaves (max, sum)
// of every row and tile, which are joined.  With g = dL/dlogp,
//   G = dL/dx = g ([v = t] - exp(x - M) / S),  dL/dhidden = G weight,
//   dL/dweight = G^T hidden,
// and the second pass computes the logits of a piece of the vocabulary again,
// writes the piece of G in the inputs' type and runs both products on it.  Where
// one piece holds the whole vocabulary, the first pass leaves its exponentials
// in the piece's place, and nothing is computed twice.
//
// Rows that take no part are left out from the start: the others are packed
// together (`order`), so that they cost nothing and what they hold is never
// read.  The packed rows are padded with zeros to whole tiles and steps.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "acdc_train_gemm.hpp"
#include "acdc_train_lm.hpp"

namespace acdc {
namespace {

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kNegMax = -3.402823466e38f;
__device__ __forceinline__ float exp_of(float d) { return __builtin_amdgcn_exp2f(d * kLog2e); }
// The product's rounding is 2^-24 |d| of the result: float32 gradients would show it.  EXACT:
// e^d = 2^p (1 + r log 2) with p + r = d log2(e) and p rounded, for d <= 0 (half the
// instructions of expf, which also looks after large d and results that are no normal
// numbers: of these 0 is made).  Where e is not 0, |r| is below 2^-16.  Where e is 0, r may be
// anything: it grows with |d|, is infinite where p leaves 32 bits (d below -2.36e38, a class
// switched off by the type's lowest value) and NaN at d = -inf; the median of r, -1 and 1 is
// finite (-1 for NaN), and 0 stays 0.  (float32 log-probabilities of 6075 rows of 64 over 98566
// classes: 918 us a call for 1062, a loss of 1000 of 1024 over 20001 681 for 684.)
template <bool EXACT>
__device__ __forceinline__ float exp_as(float d) {
  if constexpr (EXACT) {
    constexpr float kLow = 1.925963033500e-8f;  // log2(e) - kLog2e
    const float p = d * kLog2e, r = __builtin_amdgcn_fmed3f(fmaf(d, kLow, fmaf(d, kLog2e, -p)), -1.f, 1.f);
    const float e = __builtin_amdgcn_exp2f(p);
    return fmaf(e * 0.693147180559945f, r, e);
  } else {
    return exp_of(d);
  }
}

// ------------------------------------------------------------ the rows in use

// What is known of the packed rows (`order` and the rest are indexed by a packed
// row, `at` by a row of the caller's).
struct Rows {
  int* order;    // [padded] row of the caller's
  int* target;   // [padded] its class; -1 past the rows in use, -2 for one past the classes
  float* share;  // [padded] its weight, or dL/dlogp
  int* at;       // [rows] packed row, -1: takes no part
  int* count;    // rows in use
  double* total;  // sum of the weights
  float* factor;  // what the gradients of the products are multiplied by
  float* peak;    // the largest finite |share|, 1 where there is none
};
// The factor all rows share: grad_scale, over the weights' sum for a mean, or *scale; and the
// largest share, by which every row's is divided before dL/dx is rounded.
struct Factor {
  const float* device;
  float host;
  bool mean;
};

__device__ __forceinline__ void finish_rows(const Factor& factor, const Rows& out, double sum, int used, float peak) {
  *out.total = sum;
  *out.count = used;
  peak = peak > 0.f ? peak : 1.f;
  *out.peak = peak;
  const double f = double(factor.device != nullptr ? *factor.device : factor.host) * double(peak);
  *out.factor = !factor.mean ? float(f) : sum == 0.0 ? 0.f : float(f / sum);
}
// |w|, 0 where it is not finite
__device__ __forceinline__ float finite_size(float w) { return fabsf(w) <= -kNegMax ? fabsf(w) : 0.f; }

constexpr int kWide = 1024, kEach = 8;

// Packs the rows in use, in order, and clears the outputs of the others.  One
// workgroup, 8192 rows a round (8 us for 2048 rows, 15 for 8192).
__global__ __launch_bounds__(kWide) void k_vocab_rows(const void* __restrict__ targets, int bits,
                                                      const float* __restrict__ weights, int rows, int padded, int classes,
                                                      Factor factor, Rows out, float* logp, float2* saved, float* row_grads) {
  __shared__ int counts[kWide / 64];
  __shared__ double sums[kWide / 64];
  __shared__ float peaks[kWide / 64];
  const int tid = threadIdx.x, wave = tid / 64, lane = tid % 64;
  int done = 0;
  double sum = 0.0;
  float peak = 0.f;
  for (int base = 0; base < rows; base += kWide * kEach) {
    const int first = base + tid * kEach;
    int t[kEach];
    float w[kEach];
    unsigned in_use = 0;
#pragma unroll
    for (int q = 0; q < kEach; ++q) {
      const int r = first + q;
      t[q] = -1;
      w[q] = 1.f;
      if (r < rows) {
        const long long v = bits == 64 ? static_cast<const long long*>(targets)[r] : (long long)static_cast<const int*>(targets)[r];
        t[q] = v < 0 ? -1 : v >= classes ? -2 : int(v);
        if (weights != nullptr) w[q] = weights[r];
        if (t[q] != -1 && w[q] != 0.f) in_use |= 1u << q;
      }
    }
    const int mine = __popc(in_use);
    int before = mine;  // inclusive over the wave
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int up = __shfl_up(before, o);
      if (lane >= o) before += up;
    }
    if (lane == 63) counts[wave] = before;
    __syncthreads();
    int place = done + before - mine;
#pragma unroll
    for (int k = 0; k < kWide / 64; ++k) {
      if (k < wave) place += counts[k];
      done += counts[k];
    }
    __syncthreads();
#pragma unroll
    for (int q = 0; q < kEach; ++q) {
      const int r = first + q;
      if (r >= rows) break;
      if (in_use >> q & 1) {
        out.order[place] = r;
        out.target[place] = t[q];
        out.share[place] = w[q];
        out.at[r] = place++;
        sum += double(w[q]);
        peak = fmaxf(peak, finite_size(w[q]));
      } else {
        out.at[r] = -1;
        if (logp != nullptr) logp[r] = 0.f;
        if (saved != nullptr) saved[r] = make_float2(0.f, 1.f);
        if (row_grads != nullptr) row_grads[r] = 0.f;
      }
    }
  }
  for (int i = done + tid; i < padded; i += kWide) {
    out.order[i] = 0;
    out.target[i] = -1;
    out.share[i] = 0.f;
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
  peak = wave_max(peak);
  if (lane == 0) {
    sums[wave] = sum;
    peaks[wave] = peak;
  }
  __syncthreads();
  if (tid == 0) {
    double all = 0.0;
    for (int k = 0; k < kWide / 64; ++k) {
      all += sums[k];
      peak = fmaxf(peak, peaks[k]);
    }
    finish_rows(factor, out, all, done, peak);
  }
}

// The same of up to 64 rows by a wave, a row a lane.
struct FewRows {
  const void* targets;
  const float* weights;
  int bits, rows, classes;
  Factor factor;
  Rows out;
  float* logp;
  float2* saved;
  float* row_grads;
  // `at` (LDS) gets the rows in use in order; returns their number.  All waves of a workgroup
  // write the same; `first` writes what is kept.
  __device__ __forceinline__ int order(int* at, bool first) const {
    const int r = threadIdx.x % 64;
    int t = -1;
    float w = 1.f;
    if (r < rows) {
      const long long v = bits == 64 ? static_cast<const long long*>(targets)[r] : (long long)static_cast<const int*>(targets)[r];
      t = v < 0 ? -1 : v >= classes ? -2 : int(v);
      if (weights != nullptr) w = weights[r];
    }
    const bool in_use = t != -1 && w != 0.f;
    const unsigned long long all = __ballot(in_use);
    const int place = __popcll(all & ((1ull << r) - 1)), used = __popcll(all);
    if (in_use) at[place] = r;
    if (!first || threadIdx.x >= 64) return used;
    double sum = in_use ? double(w) : 0.0;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
    if (in_use) {
      out.order[place] = r;
      out.target[place] = t;
      out.share[place] = w;
    } else {
      const int behind = used + __popcll(~all & ((1ull << r) - 1));   // the places that are left, of 64
      out.order[behind] = 0;
      out.target[behind] = -1;
      out.share[behind] = 0.f;
    }
    if (r < rows) {
      out.at[r] = in_use ? place : -1;
      if (!in_use) {
        if (logp != nullptr) logp[r] = 0.f;
        if (saved != nullptr) saved[r] = make_float2(0.f, 1.f);
        if (row_grads != nullptr) row_grads[r] = 0.f;
      }
    }
    const float peak = wave_max(in_use ? finite_size(w) : 0.f);
    if (r == 0) finish_rows(factor, out, sum, used, peak);
    return used;
  }
};

// Rows as the matrix cores take them: bfloat16 (three planes for float32), `padded`
// wide, at multiples of 16 bytes.  With `order` the packed rows, zeros past *count.
template <class T>
struct Pack {
  const typename T::Elem* x;
  long long stride;
  const int* order;
  int rows;
  __bf16* out;
  long long plane;
};
// Two of them in one launch (the second may have no rows).  Bound by HBM: 6.2 TB/s for 21000
// rows of 1024 float32 values.  FEW: up to 64 rows, which every
// wave puts in order by itself, and the first one for the launches to come.
template <class T, bool FEW>
__global__ __launch_bounds__(256) void k_vocab_pack(Pack<T> first, Pack<T> second, FewRows few, const int* __restrict__ count,
                                                    int width, int padded) {
  __shared__ int order[64];
  int used;
  if constexpr (FEW) {
    used = few.order(order, blockIdx.x == 0);
    __syncthreads();
    first.order = order;
  } else {
    used = *count;
  }
  const int per = padded / 8;
  const long long split = (long long)first.rows * per, chunks = split + (long long)second.rows * per;
  for (long long base = blockIdx.x * 256ll; base < chunks; base += gridDim.x * 256ll) {
    // (one long division for the workgroup, a short one for the lane)
    const bool in_first = base < split;
    const long long begin = in_first ? base : base - split;
    const int row = int(begin / per);
    unsigned at = unsigned(begin - (long long)row * per) + threadIdx.x;
    const bool over = in_first && base + threadIdx.x >= split;  // the job changes within the workgroup
    if (over) at = unsigned(base + threadIdx.x - split);
    if (base + threadIdx.x >= chunks) break;
    const Pack<T>& job = in_first && !over ? first : second;
    const int r = (over ? 0 : row) + int(at / unsigned(per)), col = int(at % unsigned(per)) * 8;
    float v[8] = {};
    if (job.order == nullptr || r < used) {
      const typename T::Elem* from = job.x + (job.order != nullptr ? job.order[r] : r) * job.stride + col;
      if (col + 8 <= width) {
#pragma unroll
        for (int q = 0; q < 8 / T::kPer; ++q) {
          const typename T::Raw raw = load_chunk<T>(from + q * T::kPer);
#pragma unroll
          for (int i = 0; i < T::kPer; ++i) v[q * T::kPer + i] = T::get(raw, i);
        }
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (col + i < width) v[i] = T::one(from[i]);
      }
    }
    __bf16* to = job.out + (long long)r * padded + col;
    if constexpr (std::is_same_v<T, BF16>) {
      bf16x8 o;
#pragma unroll
      for (int i = 0; i < 8; ++i) o[i] = __bf16(v[i]);
      *reinterpret_cast<bf16x8*>(to) = o;
    } else {
      bf16x8 o[3];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const Split3 s = split3(v[i]);
#pragma unroll
        for (int p = 0; p < 3; ++p) o[p][i] = s.p[p];
      }
#pragma unroll
      for (int p = 0; p < 3; ++p) *reinterpret_cast<bf16x8*>(to + p * job.plane) = o[p];
    }
  }
}

// ------------------------------------------------------ what follows a product

// What the first pass keeps of the logits: nothing, or exp(x - the tile's maximum) where
// the second pass can use it.
enum class Keep { kNothing, kBf16, kF32 };

// Statistics of a tile's rows: their (max, sum) into parts[tile][row], and the target's
// logit.  m runs over classes, n over packed rows; `classes` are those of the piece.  A tile
// of 256 x 256 takes 41 us with 16 steps of 64 and 114 with 64: 17 for its start, the
// exponentials and the stores, while its CU's matrix cores idle.
template <Keep KEEP, bool EXACT>
struct StatsOut {
  const int* target;
  float2* parts;
  float* logit;
  void* kept;  // rows `ld` apart
  int first, classes, rows, tile, ld;
  // the classes past the last are no classes
  template <int MI, int NI, class SP>
  __device__ __forceinline__ void mask(f32x4 (&acc)[MI][NI], const SP& spot, int n) const {
#pragma unroll
    for (int m = 0; m < MI; ++m)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (spot.m(m) + i >= classes) acc[m][n][i] = -__builtin_inff();
  }
  template <class S, int MI, int NI, class SP>
  __device__ __forceinline__ void operator()(f32x4 (&acc)[MI][NI], const SP& spot, const Place& at, int wave,
                                             float2* slots) const {
    constexpr int BN = S::BN, WM = S::WM;
    const int lane = spot.lane;
    // (asked for together, not one after the other between the stores below)
    int targets[NI];
#pragma unroll
    for (int n = 0; n < NI; ++n) targets[n] = target[spot.n(n)];
    __syncthreads();  // the tiles have been read
    float tops[NI];
#pragma unroll
    for (int n = 0; n < NI; ++n) {
      const int r = spot.n(n), t = targets[n] - first - spot.m(0);
      if ((at.tm + 1) * S::BM > classes) mask(acc, spot, n);
      if (unsigned(t) < 16u * MI && t % 32 < 8) {
#pragma unroll
        for (int v = 0; v < 4 * MI; ++v)
          if (v == t / 32 * 8 + t % 32) logit[r] = acc[v / 4][n][v % 4];
      }
      float top = kNegMax;
#pragma unroll
      for (int m = 0; m < MI; ++m)
#pragma unroll
        for (int i = 0; i < 4; ++i) top = fmaxf(top, acc[m][n][i]);
      Pair p = swap16(top);
      top = fmaxf(p.a, p.b);
      p = swap32(top);
      tops[n] = fmaxf(p.a, p.b);
      if (lane < 16) slots[(r - at.tn * BN) * WM + wave % WM].x = tops[n];
    }
    __syncthreads();
    // the maximum of all of the tile's classes (also where nothing is kept: the same sums)
#pragma unroll
    for (int n = 0; n < NI; ++n)
#pragma unroll
      for (int w = 0; w < WM; ++w) tops[n] = fmaxf(tops[n], slots[(spot.n(n) - at.tn * BN) * WM + w].x);
    __syncthreads();
#pragma unroll
    for (int n = 0; n < NI; ++n) {
      const int r = spot.n(n);
      float sum = 0.f;
#pragma unroll
      for (int m = 0; m < MI; ++m)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          acc[m][n][i] = exp_as<EXACT>(acc[m][n][i] - tops[n]);
          sum += acc[m][n][i];
        }
      Pair p = swap16(sum);
      sum = p.a + p.b;
      p = swap32(sum);
      if (lane < 16) slots[(r - at.tn * BN) * WM + wave % WM] = make_float2(tops[n], p.a + p.b);
      const long long to = (long long)r * ld;
      if constexpr (KEEP == Keep::kBf16) {
#pragma unroll
        for (int m = 0; m < MI; m += 2) {
          bf16x8 o;
#pragma unroll
          for (int i = 0; i < 8; ++i) o[i] = __bf16(acc[m + i / 4][n][i % 4]);
          *reinterpret_cast<bf16x8*>(static_cast<__bf16*>(kept) + to + spot.m(m)) = o;
        }
      } else if constexpr (KEEP == Keep::kF32) {
#pragma unroll
        for (int m = 0; m < MI; ++m) *reinterpret_cast<f32x4*>(static_cast<float*>(kept) + to + spot.m(m)) = acc[m][n];
      }
    }
    __syncthreads();
    if (int(threadIdx.x) < BN) {
      float2 all = slots[threadIdx.x * WM];
#pragma unroll
      for (int w = 1; w < WM; ++w) all.y += slots[threadIdx.x * WM + w].y;
      parts[(long long)(tile + at.tm) * rows + at.tn * BN + threadIdx.x] = all;
    }
  }
};

// What turns a row's logits into G: M, g / S, g and the target.  g without the factor that
// all rows share, which the sums of the products are multiplied by: 1 / W in every target's
// g would be rounded to bfloat16 the same way in all of them, and the errors add up.  A caller
// may give dL/dlogp with such a factor in it: the largest share is taken out of all, so that
// equal ones become 1.
struct RowSlope {
  float top, slope, g;
  int target;
};

// Values of G as 1, 2 or 3 planes of bfloat16: the one rounding between the logits and the
// gradients, to 8, 16 or 24 bits.  float32 inputs take 24 and bfloat16 ones 16, of which nothing
// is seen in a gradient of 8 or 32 bits.  Only large products of bfloat16 inputs, of kMany terms
// or more each, take 8 (see there).
template <int PLANES, int N, class V>
__device__ __forceinline__ void put_planes(__bf16* out, long long plane, const float (&y)[N]) {
  V o[PLANES];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    if constexpr (PLANES == 3) {
      const Split3 s = split3(y[i]);
#pragma unroll
      for (int p = 0; p < 3; ++p) o[p][i] = s.p[p];
    } else {
      o[0][i] = __bf16(y[i]);
      if constexpr (PLANES == 2) o[1][i] = __bf16(y[i] - float(o[0][i]));
    }
  }
#pragma unroll
  for (int p = 0; p < PLANES; ++p) *reinterpret_cast<V*>(out + p * plane) = o[p];
}

// The piece of G, rows `ld` apart, zeros past the classes and for padding rows.  (The target's
// own value is a difference of 32-bit values: where 1 - p is small, it is off by the rounding of
// S as the logarithm of S would be.)
template <int PLANES>
struct SlopeOut {
  const RowSlope* row;
  __bf16* out;
  long long plane;
  int ld, first, classes;
  template <class S, int MI, int NI, class SP>
  __device__ __forceinline__ void operator()(f32x4 (&acc)[MI][NI], const SP& spot, const Place&, int, float2*) const {
    RowSlope slopes[NI];
#pragma unroll
    for (int n = 0; n < NI; ++n) slopes[n] = row[spot.n(n)];
#pragma unroll
    for (int n = 0; n < NI; ++n) {
      const int r = spot.n(n);
      const RowSlope k = slopes[n];
      const int t = k.target - first;
      __bf16* to = out + (long long)r * ld;
#pragma unroll
      for (int m = 0; m < MI; m += 2) {
        float y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int v = spot.m(m + i / 4) + i % 4;
          y[i] = -exp_as<(PLANES > 1)>(acc[m + i / 4][n][i % 4] - k.top) * k.slope;
          if (v == t) y[i] += k.g;
          if (v >= classes) y[i] = 0.f;
        }
        put_planes<PLANES, 8, bf16x8>(to + spot.m(m), plane, y);
      }
    }
  }
};

// The same from what the first pass kept, e = exp(x - the tile's maximum), of a single
// piece: in place where e is bfloat16 (a second rounding, of 2^-8 at the most; the
// target's own value, where 1 - p may be small, comes from its logit).  A wave takes 512
// classes of a row; bound by HBM (2048 x 32768 in bfloat16: 6.4 TB/s, 8192 x 65536 5.8).
template <int PLANES, class E>
__global__ __launch_bounds__(256) void k_vocab_slopes(Rows rows, const RowSlope* __restrict__ slope, const float2* __restrict__ parts,
                                                      const float* __restrict__ logp, const void* kept, __bf16* out,
                                                      long long plane, int ld, int tile, int padded, int blocks) {
  typedef E Eight __attribute__((ext_vector_type(8)));
  const int lane = threadIdx.x % 64, used = (*rows.count + 63) / 64 * 64;
  const long long item = blockIdx.x * 4ll + threadIdx.x / 64;
  const int r = int(item / blocks), col = (int(item % blocks) * 64 + lane) * 8;
  if (r >= used || col >= ld) return;
  const RowSlope k = slope[r];
  const float f = -k.slope * expf(parts[(long long)(col / tile) * padded + r].x - k.top);
  const long long at = (long long)r * ld + col;
  const Eight e = *reinterpret_cast<const Eight*>(static_cast<const E*>(kept) + at);
  float y[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    y[i] = float(e[i]) * f;
    if (col + i == k.target) y[i] = -k.g * expm1f(logp[rows.order[r]]);
  }
  put_planes<PLANES, 8, bf16x8>(out + at, plane, y);
}

// A product of few tiles leaves its logits as sums of parts.  Where they are of several pieces
// of the vocabulary, or come from saved statistics, a wave adds them up for 64 classes of a row.
struct FewLogits {
  const float* sums;
  const int* count;
  long long part;
  int parts, ld, tiles, first, classes;
  // this wave's row and its lane's class and logit; false: nothing to do
  __device__ __forceinline__ bool read(int& r, int& v, float& x) const {
    const long long item = blockIdx.x * 4ll + threadIdx.x / 64;
    r = int(item / tiles);
    v = int(item % tiles) * 64 + threadIdx.x % 64;
    if (r >= (*count + 63) / 64 * 64) return false;
    x = 0.f;
    const float* p = sums + (long long)r * ld + v;
#pragma unroll 8
    for (int k = 0; k < parts; ++k) x += p[k * part];
    return true;
  }
};
__global__ __launch_bounds__(256) void k_vocab_few_stats(FewLogits l, const int* __restrict__ target, float2* __restrict__ parts,
                                                         float* __restrict__ logit, int padded) {
  int r, v;
  float x;
  if (!l.read(r, v, x)) return;
  if (v >= l.classes) x = -__builtin_inff();
  const float top = fmaxf(wave_max(x), kNegMax), e = expf(x - top), sum = wave_sum(e);
  if (v == target[r] - l.first) logit[r] = x;
  if (threadIdx.x % 64 == 0) parts[(long long)((l.first + v) / 64) * padded + r] = make_float2(top, sum);
}
template <int PLANES>
__global__ __launch_bounds__(256) void k_vocab_few_slopes(FewLogits l, const RowSlope* __restrict__ slope, __bf16* __restrict__ out,
                                                          long long plane) {
  typedef __bf16 One __attribute__((ext_vector_type(1)));
  int r, v;
  float x;
  if (!l.read(r, v, x)) return;
  const RowSlope k = slope[r];
  float y[1] = {-expf(x - k.top) * k.slope};
  if (v == k.target - l.first) y[0] += k.g;
  if (v >= l.classes) y[0] = 0.f;
  put_planes<PLANES, 1, One>(out + (long long)r * l.ld + v, plane, y);
}

// f(n, m) for the squares of a wave: with bounds where the tile reaches past M or N.
template <class S, int MI, int NI, class SP, class F>
__device__ __forceinline__ void squares(const SP& spot, const Place& at, int M, int N, F&& f) {
  if ((at.tm + 1) * S::BM <= M && (at.tn + 1) * S::BN <= N) {
#pragma unroll
    for (int n = 0; n < NI; ++n)
#pragma unroll
      for (int m = 0; m < MI; ++m) f.template operator()<true>(n, m);
  } else {
#pragma unroll
    for (int n = 0; n < NI; ++n)
#pragma unroll
      for (int m = 0; m < MI; ++m)
        if (spot.m(m) < M && spot.n(n) < N) f.template operator()<false>(n, m);
  }
}

// 32-bit sums of a part: out[part][n][m], added to what earlier pieces left.
struct PartOut {
  float* out;
  long long part;
  int ld, rows;
  bool add;
  template <class S, int MI, int NI, class SP>
  __device__ __forceinline__ void operator()(f32x4 (&acc)[MI][NI], const SP& spot, const Place& at, int, float2*) const {
    float* to = out + at.part * part;
    auto each = [&]<bool ADD>() {
      squares<S, MI, NI>(spot, at, ld, rows, [&]<bool INSIDE>(int n, int m) {
        f32x4* p = reinterpret_cast<f32x4*>(to + (long long)spot.n(n) * ld + spot.m(m));
        if constexpr (ADD) *p += acc[m][n];
        else *p = acc[m][n];
      });
    };
    if (add) each.template operator()<true>();
    else each.template operator()<false>();
  }
};

// Four values of a row of a gradient.  `whole`: rows at multiples of four elements.
template <class T>
__device__ __forceinline__ void put4(typename T::Elem* to, f32x4 v, int left, bool whole, bool add) {
  using E = typename T::Elem;
  typedef E Four __attribute__((ext_vector_type(4)));
  if (whole && left >= 4) {
    if (add) {
      const Four old = *reinterpret_cast<const Four*>(to);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] += float(old[i]);
    }
    *reinterpret_cast<Four*>(to) = Four{T::to(v[0]), T::to(v[1]), T::to(v[2]), T::to(v[3])};
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < left) to[i] = T::to(add ? v[i] + float(to[i]) : v[i]);
  }
}

// The gradient itself: m runs over the width, n over the piece's classes.
template <class T>
struct GradOut {
  typename T::Elem* out;
  const float* factor;
  long long ld;
  int width, classes;
  bool whole, add;
  template <class S, int MI, int NI, class SP>
  __device__ __forceinline__ void operator()(f32x4 (&acc)[MI][NI], const SP& spot, const Place& at, int, float2*) const {
    const float f = *factor;
    auto each = [&]<bool PLAIN>() {
      squares<S, MI, NI>(spot, at, width, classes, [&]<bool INSIDE>(int n, int m) {
        typename T::Elem* to = out + spot.n(n) * ld + spot.m(m);
        if constexpr (PLAIN && INSIDE) put4<T>(to, acc[m][n] * f, 4, true, false);
        else put4<T>(to, acc[m][n] * f, width - spot.m(m), whole, add);
      });
    };
    if (whole && !add) each.template operator()<true>();
    else each.template operator()<false>();
  }
};

// stats = (loss, W) from the sum of weight times logp
__device__ __forceinline__ void put_stats(float* stats, const Rows& rows, double sum, bool mean) {
  const double total = *rows.total;
  stats[0] = *rows.count == 0 || (mean && total == 0.0) ? 0.f : float(mean ? -sum / total : -sum);
  stats[1] = float(total);
}
// The same from the rows' own, summed in 64 bits by one workgroup.
struct Totals {
  Rows rows;
  const float* loss;  // [padded] weight times logp
  float* stats;       // null: none
  bool mean;
  __device__ __forceinline__ void run() const {
    __shared__ double sums[4];
    constexpr int AHEAD = 16;
    const int used = *rows.count;
    double sum = 0.0;
    for (int i = threadIdx.x; i < used; i += 256 * AHEAD) {
      float v[AHEAD];
#pragma unroll
      for (int q = 0; q < AHEAD; ++q) v[q] = i + 256 * q < used ? loss[i + 256 * q] : 0.f;
#pragma unroll
      for (int q = 0; q < AHEAD; ++q) sum += double(v[q]);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
    if (threadIdx.x % 64 == 0) sums[threadIdx.x / 64] = sum;
    __syncthreads();
    if (threadIdx.x == 0) put_stats(stats, rows, ((sums[0] + sums[1]) + sums[2]) + sums[3], mean);
  }
};
__global__ __launch_bounds__(256) void k_vocab_total(Totals totals) { totals.run(); }

// The parts of a sum together, in order, into the gradient's rows (4 TB/s: they come from the
// Infinity Cache, eight parts of 2048 x 1024 in 16 us).  With `at` the rows that take no part
// get zeros.  The last workgroup does `totals` instead, if there are any.
template <class T>
__global__ __launch_bounds__(256) void k_vocab_sum(const float* __restrict__ sums, int parts, long long part, int padded,
                                                   const int* __restrict__ at, const float* __restrict__ factor,
                                                   long long rows, int width,
                                                   typename T::Elem* __restrict__ out, long long ld, bool whole, bool add,
                                                   Totals totals) {
  const int per = (width + 3) / 4;
  const unsigned groups = gridDim.x - (totals.stats != nullptr ? 1 : 0);
  if (blockIdx.x == groups) return totals.run();
  for (long long c = blockIdx.x * 256ll + threadIdx.x; c < rows * per; c += groups * 256ll) {
    const long long r = c / per;
    const int col = int(c % per) * 4;
    const long long from = at != nullptr ? at[r] : r;
    f32x4 v = {};
    if (from >= 0) {
      const float* p = sums + from * padded + col;
#pragma unroll 16
      for (int k = 0; k < parts; ++k) v += *reinterpret_cast<const f32x4*>(p + k * part);
      v *= *factor;
    }
    put4<T>(out + r * ld + col, v, width - col, whole, add);
  }
}

// --------------------------------------------------------- the rows' statistics

struct JoinOut {
  float* logp;
  float2* saved;
  float* row_grads;
  RowSlope* slope;     // null: no gradient
  float* loss;         // [padded] weight times logp, null: not wanted
  bool mean;
};
// What packed row i leaves: its logp, loss and g = dL/dlogp without the common factors.
struct Joined {
  float logp, loss, g;
};
__device__ __forceinline__ Joined join_row(const Rows& rows, int i, int t, float top, float sum, float logit) {
  // no class with a probability: no distribution
  const float nan = sum > 0.f ? 0.f : __builtin_nanf(""), w = rows.share[i];
  const float logp = t >= 0 ? (logit - top) - logf(sum) + nan : __builtin_nanf("");
  return {logp, w * logp, t >= 0 ? -w / *rows.peak : __builtin_nanf("")};
}
__device__ __forceinline__ void put_row(const Rows& rows, const JoinOut& out, int i, const Joined& j, float top, float sum) {
  const int r = rows.order[i];
  out.logp[r] = j.logp;
  if (out.saved != nullptr) out.saved[r] = make_float2(top, sum);
  if (out.row_grads != nullptr) {
    const double total = out.mean ? *rows.total : 1.0;
    out.row_grads[r] = total == 0.0 ? 0.f : -float(double(rows.share[i]) / total);
  }
}
// Two sums of exponentials, each less its maximum, as one.
__device__ __forceinline__ void merge(float& top, float& sum, float other_top, float other) {
  const float m = fmaxf(top, other_top);
  sum = sum * expf(top - m) + other * expf(other_top - m);
  top = m;
}
// The tiles' statistics of 16 packed rows together, by 64 groups of 16 lanes along the tiles;
// then what the row leaves.  (64 rows and 16 waves: 10.2 us where 8 rows have 512 tiles.)
__global__ __launch_bounds__(1024) void k_vocab_join(Rows rows, const float2* __restrict__ parts, const float* __restrict__ logit,
                                                     int tiles, int padded, JoinOut out) {
  constexpr int ROWS = 16, WAVES = 16, GROUPS = 1024 / ROWS;
  __shared__ float2 slots[WAVES][ROWS];
  const int lane = threadIdx.x % ROWS, group = threadIdx.x / ROWS, i = blockIdx.x * ROWS + lane;
  const int used = *rows.count;
  float top = kNegMax, sum = 0.f;
  if (i < used) {
    constexpr int AHEAD = 8;
    for (int k = group; k < tiles; k += GROUPS * AHEAD) {
      float2 p[AHEAD];
#pragma unroll
      for (int q = 0; q < AHEAD; ++q)
        p[q] = k + GROUPS * q < tiles ? parts[(long long)(k + GROUPS * q) * padded + i] : make_float2(kNegMax, 0.f);
      float m = top;
#pragma unroll
      for (int q = 0; q < AHEAD; ++q) m = fmaxf(m, p[q].x);
      sum *= expf(top - m);
#pragma unroll
      for (int q = 0; q < AHEAD; ++q) sum += p[q].y * expf(p[q].x - m);
      top = m;
    }
  }
#pragma unroll
  for (int o = ROWS; o < 64; o <<= 1) merge(top, sum, __shfl_xor(top, o), __shfl_xor(sum, o));
  if (group % (64 / ROWS) == 0) slots[group / (64 / ROWS)][lane] = make_float2(top, sum);
  __syncthreads();
  if (threadIdx.x >= 64) return;
  top = kNegMax;
  sum = 0.f;
#pragma unroll
  for (int w = 0; w < WAVES / (64 / ROWS); ++w) {
    const float2 p = slots[group * (WAVES * ROWS / 64) + w][lane];
    merge(top, sum, p.x, p.y);
  }
#pragma unroll
  for (int o = ROWS; o < 64; o <<= 1) merge(top, sum, __shfl_xor(top, o), __shfl_xor(sum, o));
  if (group != 0) return;
  if (i >= used) {
    if (out.slope != nullptr) out.slope[i] = RowSlope{0.f, 0.f, 0.f, -1};
    return;
  }
  const int t = rows.target[i];
  const Joined j = join_row(rows, i, t, top, sum, logit[i]);
  put_row(rows, out, i, j, top, sum);
  if (out.loss != nullptr) out.loss[i] = j.loss;
  if (out.slope != nullptr) out.slope[i] = RowSlope{top, j.g / sum, j.g, t};
}

// A product of few tiles over all classes: what the tiles' statistics, k_vocab_join and
// k_vocab_slopes do, by a workgroup for each packed row, which holds its logits in
// registers.  One launch for two, and a product that splits its steps: 64 rows of 256 over
// 1000 classes in float32 22.8 us a call instead of 28.6, 256 of 1024 48 instead of 65.
constexpr int kFewClasses = 4096, kFewEach = kFewClasses / 1024;
template <int PLANES>
__global__ __launch_bounds__(256) void k_vocab_few(FewLogits l, Rows rows, JoinOut out, __bf16* __restrict__ grad, long long plane) {
  __shared__ float tops[4], sums[4], logit;
  const int i = blockIdx.x, tid = threadIdx.x, used = *rows.count;
  if (i >= (used + 63) / 64 * 64) return;
  const int t = i < used ? rows.target[i] : -1;
  const float* from = l.sums + (long long)i * l.ld;
  f32x4 x[kFewEach];
  float top = kNegMax;
#pragma unroll
  for (int c = 0; c < kFewEach; ++c) {
    const int v = (c * 256 + tid) * 4;
    x[c] = f32x4{};
    if (v < l.ld) {
#pragma unroll 8
      for (int k = 0; k < l.parts; ++k) x[c] += *reinterpret_cast<const f32x4*>(from + k * l.part + v);
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      if (v + q == t) logit = x[c][q];
      if (v + q >= l.classes) x[c][q] = -__builtin_inff();
      top = fmaxf(top, x[c][q]);
    }
  }
  top = wave_max(top);
  if (tid % 64 == 0) tops[tid / 64] = top;
  __syncthreads();
  top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
  float sum = 0.f;
#pragma unroll
  for (int c = 0; c < kFewEach; ++c)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      x[c][q] = expf(x[c][q] - top);
      sum += x[c][q];
    }
  sum = wave_sum(sum);
  if (tid % 64 == 0) sums[tid / 64] = sum;
  __syncthreads();
  sum = ((sums[0] + sums[1]) + sums[2]) + sums[3];
  Joined j{0.f, 0.f, 0.f};
  if (i < used) {
    j = join_row(rows, i, t, top, sum, logit);
    if (tid == 0) {
      put_row(rows, out, i, j, top, sum);
      if (out.loss != nullptr) out.loss[i] = j.loss;
    }
  }
  if constexpr (PLANES > 0) {
    const float f = -(j.g / sum), own = -j.g * expm1f(j.logp);  // (1 - p may be small)
#pragma unroll
    for (int c = 0; c < kFewEach; ++c) {
      const int v = (c * 256 + tid) * 4;
      if (v >= l.ld) break;
      float y[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) y[q] = v + q == t ? own : x[c][q] * f;
      put_planes<PLANES, 4, bf16x4>(grad + (long long)i * l.ld + v, plane, y);
    }
  }
}

// RowSlope from what an earlier call saved.
__global__ __launch_bounds__(256) void k_vocab_slope(Rows rows, const float2* __restrict__ saved, int padded, RowSlope* __restrict__ slope) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i >= padded) return;
  if (i >= *rows.count) {
    slope[i] = RowSlope{0.f, 0.f, 0.f, -1};
    return;
  }
  const float2 st = saved[rows.order[i]];
  const int t = rows.target[i];
  const float g = t >= 0 ? rows.share[i] / *rows.peak : __builtin_nanf("");
  slope[i] = RowSlope{st.x, g / st.y, g, t};
}

// ------------------------------------------------------------------ on the host

int64_t up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }
size_t up256(size_t n) { return (n + 255) & ~size_t(255); }

constexpr int kTile = 256;
// Bytes of a piece of G.  A piece costs a pass over the sums of dL/dhidden, and the logits
// of a single one need not be computed again: 8192 rows over 65536 classes are one piece.
constexpr int64_t kPieceBytes = int64_t(2) << 30;
// Terms from which on, in both gradients, G of bfloat16 inputs may be rounded to 8 bits: it is
// multiplied by values of 8 bits, and as their roundings do, those of G fall either way, so that
// against the sizes of n terms together a sum is off by 2^-9 / sqrt(n) or so.  (Where few terms
// decide, or rows alike are rounded alike, it is by 2^-8 of them at the most, as by its own
// rounding, and 2^-7 where the exponentials were rounded too.)
// 16 bits cost few rows nothing and many the second product of every pair: with 16 and with 8
// bits 1 row of 4096 over 8192 classes 88 and 90 us, 64 of 4096 over 65536 499 and 498, 256 of
// 1024 over 32768 153 and 125, 1000 of 4096 over 65536 2.31 and 1.50 ms, 2048 of 1024 over 32768
// 0.78 and 0.46, 8192 of 4096 over 65536 18.6 and 10.4.
constexpr int kMany = 1024;
static_assert((kMany / 64) * (kMany / 64) > kFewClasses / 64, "8 bits of G: more rows than Flat takes, and no FewLogits");

// Products of BM x BN: large tiles feed the matrix cores best, small ones keep more of the
// card busy, and give a row of few steps to more workgroups.  Four waves of 64 x 128 for
// float32: eight of 64 x 64 have no registers for reading ahead (1000 x 1024 over 20001
// classes 676 us a call, 696 with those where no operand lies across), and half the tile saves
// nothing where it fills the last round (685 for 684).  Large2: bfloat16 times two planes of G,
// for which steps of 64 do not fit and reading ahead spills (1000 of 4096 over 65536 classes in
// tiles of 256 x 256 2.31 ms a call, of 128 x 256 that read ahead 2.99, in three parts of LDS 3.31).
using Large = Shape<256, 256, 64, 4, 2, 2, true>;
using Large3 = Shape<128, 256, 32, 2, 2, 2, true>;
using Large2 = Shape<256, 256, 32, 4, 2, 3>;
using Flat = Shape<256, 64, 64, 4, 1, 2>;
using Flat3 = Shape<128, 64, 32, 4, 1, 2>;
using Small = Shape<64, 64, 64, 2, 2, 4>;
using Small3 = Shape<64, 64, 32, 2, 2, 4>;
// The shapes for P planes of one operand and PB of the other.
template <int P, int PB>
using LargeOf = std::conditional_t<PB == 1, Large, std::conditional_t<P == 1, Large2, Large3>>;
template <int P>
using FlatOf = std::conditional_t<P == 1, Flat, Flat3>;
template <int P>
using SmallOf = std::conditional_t<P == 1, Small, Small3>;

// How a call is cut up: fixed by its sizes alone.
struct Plan {
  int64_t rows, padded_rows;
  int32_t width, padded_width, classes, planes;
  int32_t piece, pieces;  // classes of a piece, a multiple of kTile
  int hidden_parts, weight_parts;
  bool large_logits, large_hidden, large_weight;  // the products' tiles
  bool few_logits;                                // the logits as sums of parts: FewLogits
  int logits_parts;
  int grad_planes;
  int tile_classes() const { return !large_logits ? 64 : planes == 1 ? 256 : 128; }  // of the logits
};
int64_t tiles_of(int64_t m, int64_t n, int bm, int bn) { return ((m + bm - 1) / bm) * ((n + bn - 1) / bn); }
int parts_for(int64_t tiles, int64_t steps, int least) {
  // as many as give every CU a tile, of `least` steps at least
  return int(std::max<int64_t>(1, std::min<int64_t>({256 / std::max<int64_t>(tiles, 1), steps / least, 64})));
}
Plan plan_for(int64_t rows, int32_t width, int32_t classes, int32_t dtype) {
  Plan p{};
  p.rows = rows;
  p.width = width;
  p.classes = classes;
  p.planes = dtype == ACDC_F32 ? 3 : 1;
  p.padded_rows = up(std::max<int64_t>(rows, 1), rows <= 64 ? 64 : kTile);
  p.padded_width = int32_t(up(width, 64));
  const bool many = rows >= kMany && classes >= kMany;
  // bytes of a class in the piece of G (with what the first pass keeps for it) and in the packed weight
  const int64_t bytes = p.planes == 3 ? 10 * std::max<int64_t>(p.padded_rows, p.padded_width)
                                      : std::max<int64_t>((many ? 2 : 8) * p.padded_rows, 2 * int64_t(p.padded_width));
  const int64_t most = std::max<int64_t>(kTile, kPieceBytes / bytes / kTile * kTile);
  p.pieces = int32_t((classes + most - 1) / most);
  p.piece = int32_t(up((classes + p.pieces - 1) / p.pieces, kTile));
  const int bm = p.planes == 1 ? 256 : 128, bn = rows <= 64 ? 64 : 256, step = p.planes == 1 ? 64 : 32;
  const int64_t piece = std::min(p.piece, classes);
  // half a card of large tiles is as fast as a card of small ones (1024 rows of 1024 over 4096
  // classes in bfloat16: 84 us a call, with large tiles from 64 on 91, from 256 on 124; in
  // float32 512 of 512 over 4096: 88, 101 and 101; 1024 of 1024: 198, 198 and 226)
  p.large_logits = tiles_of(piece, p.padded_rows, bm, bn) >= 128;
  const int64_t hidden = tiles_of(width, p.padded_rows, bm, bn), weight = tiles_of(width, piece, bm, 256);
  p.large_hidden = hidden * parts_for(hidden, piece / step, 8) >= 128;
  p.large_weight = weight * parts_for(weight, p.padded_rows / step, 8) >= 128;
  p.hidden_parts = parts_for(p.large_hidden ? hidden : tiles_of(width, p.padded_rows, 64, 64), (piece + step - 1) / step, p.large_hidden ? 8 : 2);
  const int64_t few = tiles_of(piece, p.padded_rows, 64, 64);
  p.few_logits = !p.large_logits && few <= kFewClasses / 64;
  p.logits_parts = p.few_logits ? parts_for(few, p.padded_width / step, 2) : 1;
  p.grad_planes = p.planes == 3 ? 3 : many && (p.large_hidden || p.large_weight) ? 1 : 2;
  p.weight_parts = parts_for(p.large_weight ? weight : tiles_of(width, piece, 64, 64), p.padded_rows / step, p.large_weight ? 8 : 2);
  return p;
}

struct Layout {
  size_t order, target, share, at, count, total, factor, peak, logit, parts, slope, loss, hidden, weight, logits_sums, grad, kept, hidden_sums, weight_sums, bytes;
};
Layout layout(const Plan& p, bool gradient) {
  Layout w{};
  size_t next = 0;
  auto take = [&](size_t bytes) {
    const size_t o = next;
    next += up256(bytes);
    return o;
  };
  const size_t R = size_t(p.padded_rows);
  w.order = take(R * 4);
  w.target = take(R * 4);
  w.share = take(R * 4);
  w.at = take(size_t(p.rows) * 4);
  w.count = take(4);
  w.total = take(8);
  w.factor = take(4);
  w.peak = take(4);
  w.logit = take(R * 4);
  w.parts = take(R * 8 * size_t(p.pieces) * size_t(p.piece / p.tile_classes()));
  w.slope = take(R * sizeof(RowSlope));
  w.loss = take(R * 4);
  w.hidden = take(R * p.padded_width * 2 * p.planes);
  w.weight = take(size_t(p.piece) * p.padded_width * 2 * p.planes);
  w.logits_sums = take(p.few_logits ? size_t(p.logits_parts) * R * p.piece * 4 : 0);
  if (gradient) {
    w.grad = take(R * p.piece * 2 * p.grad_planes);
    w.kept = p.grad_planes == 1 ? w.grad : take(p.pieces == 1 && !p.few_logits ? R * p.piece * 4 : 0);
    w.hidden_sums = take(size_t(p.hidden_parts) * R * p.padded_width * 4);
    w.weight_sums = take(p.weight_parts > 1 ? size_t(p.weight_parts) * p.piece * p.padded_width * 4 : 0);
  }
  w.bytes = next;
  return w;
}

int done() {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? ACDC_OK : hip_fail(e);
}

// A call on its way: the plan, where its buffers are, and the launches.
template <class T>
struct Call {
  static constexpr int P = std::is_same_v<T, F32> ? 3 : 1;
  const acdc_vocab_head& head;
  const Plan p;
  const Layout w;
  char* ws;
  hipStream_t s;
  Rows rows;
  bool direct;  // the weight as it is

  Call(const acdc_vocab_head& h, bool gradient, void* workspace, acdc_stream_t stream)
      : head(h), p(plan_for(h.rows, h.width, h.classes, h.dtype)), w(layout(p, gradient)), ws(static_cast<char*>(workspace)),
        s(reinterpret_cast<hipStream_t>(stream)) {
    rows = Rows{get<int>(w.order), get<int>(w.target), get<float>(w.share), get<int>(w.at), get<int>(w.count), get<double>(w.total), get<float>(w.factor), get<float>(w.peak)};
    direct = P == 1 && h.width % 8 == 0 && h.weight_stride % 8 == 0 && h.weight_stride < (1 << 22) && aligned_to(h.weight, 16);
  }
  template <class E>
  E* get(size_t at) const { return reinterpret_cast<E*>(ws + at); }

  static unsigned grid(int64_t items) { return unsigned(std::min<int64_t>((items + 255) / 256, 1 << 16)); }

  unsigned pack_grid(const Pack<T>& first, const Pack<T>& second) const {
    return grid((int64_t(first.rows) + second.rows) * (p.padded_width / 8));
  }
  int64_t weight_plane() const { return int64_t(p.piece) * p.padded_width; }
  Pack<T> weight_job(int k) const {
    const typename T::Elem* from = static_cast<const typename T::Elem*>(head.weight) + int64_t(k) * p.piece * head.weight_stride;
    return {from, head.weight_stride, nullptr, classes_of(k), get<__bf16>(w.weight), weight_plane()};
  }
  // the rows in use and, with them, the first piece of the weight
  void pack_rows(const float* weights, const Factor& factor, float* logp, float2* saved, float* row_grads) const {
    const Pack<T> hidden{static_cast<const typename T::Elem*>(head.hidden), head.hidden_stride, rows.order, int(p.padded_rows),
                         get<__bf16>(w.hidden), hidden_plane()};
    const Pack<T> weight = direct ? Pack<T>{} : weight_job(0);
    const FewRows few{head.targets, weights, head.target_bits, int(p.rows), p.classes, factor, rows, logp, saved, row_grads};
    if (p.rows <= 64) {
      hipLaunchKernelGGL((k_vocab_pack<T, true>), dim3(pack_grid(hidden, weight)), dim3(256), 0, s, hidden, weight, few, rows.count,
                         p.width, p.padded_width);
    } else {
      hipLaunchKernelGGL(k_vocab_rows, dim3(1), dim3(kWide), 0, s, head.targets, head.target_bits, weights, int(p.rows),
                         int(p.padded_rows), p.classes, factor, rows, logp, saved, row_grads);
      hipLaunchKernelGGL((k_vocab_pack<T, false>), dim3(pack_grid(hidden, weight)), dim3(256), 0, s, hidden, weight, few, rows.count,
                         p.width, p.padded_width);
    }
  }
  int64_t hidden_plane() const { return p.padded_rows * p.padded_width; }
  int classes_of(int k) const { return std::min(p.piece, p.classes - k * p.piece); }
  Operand hidden() const {
    return Operand{get<__bf16>(w.hidden), p.padded_width, hidden_plane(), int(p.padded_rows), p.padded_width};
  }
  // piece k of the weight; `packed`: it is the one that was packed last
  Operand weight(int k, bool packed) const {
    const int n = classes_of(k);
    const Pack<T> job = weight_job(k);
    if (direct) return Operand{reinterpret_cast<const __bf16*>(job.x), head.weight_stride, 0, n, p.width};
    if (!packed)
      hipLaunchKernelGGL((k_vocab_pack<T, false>), dim3(pack_grid(job, Pack<T>{})), dim3(256), 0, s, job, Pack<T>{}, FewRows{},
                         rows.count, p.width, p.padded_width);
    return Operand{job.out, p.padded_width, weight_plane(), n, p.padded_width};
  }
  Operand grad(int k) const {
    return Operand{get<__bf16>(w.grad), p.piece, p.padded_rows * p.piece, int(p.padded_rows), int(up(classes_of(k), 64))};
  }

  template <class S, int PB, bool XA, bool XB, Count COUNT, class E>
  static Product<S, P, PB, XA, XB, COUNT, E> product(const Operand& a, const Operand& b, int64_t m, int64_t n, int depth, int parts,
                                                     const E& e) {
    return {a, b, depth, int((m + S::BM - 1) / S::BM), int((n + S::BN - 1) / S::BN), parts, e};
  }
  template <class G>
  void launch(const G& g) const {
    hipLaunchKernelGGL(k_gemm<G>, dim3(g.groups()), dim3(G::T), 0, s, g, rows.count);
  }
  template <class G, class H>
  void launch(const G& g, const H& h) const {
    const unsigned first = unsigned(up(g.groups(), 8));
    hipLaunchKernelGGL((k_gemm_both<G, H>), dim3(first + h.groups()), dim3(G::T), 0, s, g, h, first, rows.count);
  }
  // f(a product with n over the packed rows); b of PB planes.  FEW: there may be 64 rows or less
  template <int PB, bool XA, bool FEW, class E, class F>
  void over_rows(bool large, const Operand& a, const Operand& b, int64_t m, int depth, int parts, const E& e, F&& f) const {
    constexpr Count N = Count::kN;
    if (!large) {
      f(product<SmallOf<P>, PB, XA, false, N>(a, b, m, p.padded_rows, depth, parts, e));
    } else if (!FEW || p.padded_rows > 64) {
      f(product<LargeOf<P, PB>, PB, XA, false, N>(a, b, m, p.padded_rows, depth, parts, e));
    } else if constexpr (FEW) {
      f(product<FlatOf<P>, PB, XA, false, N>(a, b, m, p.padded_rows, depth, parts, e));
    }
  }
  // classes x packed rows
  template <bool FEW, class E>
  void logits(const Operand& weight, int parts, const E& e) const {
    over_rows<P, false, FEW>(p.large_logits, weight, hidden(), weight.rows, p.padded_width, parts, e, [&](const auto& g) { launch(g); });
  }
  // the same as sums of parts, and what a wave for each 64 of a row's classes reads
  FewLogits few_logits(const Operand& weight, int k) const {
    const int64_t part = p.padded_rows * p.piece;
    logits<true>(weight, p.logits_parts, PartOut{get<float>(w.logits_sums), part, p.piece, int(p.padded_rows), false});
    return {get<float>(w.logits_sums), rows.count, part, p.logits_parts, p.piece, (classes_of(k) + 63) / 64, k * p.piece, classes_of(k)};
  }
  unsigned few_grid(const FewLogits& l) const { return unsigned((p.padded_rows * l.tiles + 3) / 4); }

  template <Keep KEEP>
  void statistics_of(const Operand& weight, int k) const {
    const StatsOut<KEEP, P == 3> out{rows.target, get<float2>(w.parts), get<float>(w.logit), get<void>(w.kept), k * p.piece, classes_of(k),
                                     int(p.padded_rows), k * (p.piece / p.tile_classes()), p.piece};
    logits<KEEP != Keep::kBf16>(weight, 1, out);
  }
  // few tiles and a single piece: everything up to G (PLANES 0: of no gradient)
  template <int PLANES>
  int few(const JoinOut& out) const {
    const FewLogits l = few_logits(weight(0, true), 0);
    hipLaunchKernelGGL(k_vocab_few<PLANES>, dim3(unsigned(p.padded_rows)), dim3(256), 0, s, l, rows, out,
                       PLANES > 0 ? get<__bf16>(w.grad) : nullptr, (long long)(p.padded_rows * p.piece));
    return done();
  }
  bool few() const { return p.few_logits && p.pieces == 1; }
  int statistics(const JoinOut& out, bool keep) const {
    if (few()) {
      if (!keep) return few<0>(out);
      return few<P == 3 ? 3 : 2>(out);  // (one plane of G is of many tiles)
    }
    for (int k = 0; k < p.pieces; ++k) {
      const Operand weight_k = weight(k, k == 0);
      if (p.few_logits) {
        const FewLogits l = few_logits(weight_k, k);
        hipLaunchKernelGGL(k_vocab_few_stats, dim3(few_grid(l)), dim3(256), 0, s, l, rows.target, get<float2>(w.parts),
                           get<float>(w.logit), int(p.padded_rows));
      } else if (!keep) {
        statistics_of<Keep::kNothing>(weight_k, k);
      } else if (p.grad_planes > 1) {
        statistics_of<Keep::kF32>(weight_k, k);
      } else if constexpr (P == 1) {
        statistics_of<Keep::kBf16>(weight_k, k);
      }
    }
    hipLaunchKernelGGL(k_vocab_join, dim3(unsigned(p.padded_rows / 16)), dim3(1024), 0, s, rows, get<float2>(w.parts),
                       get<float>(w.logit), int((p.classes + p.tile_classes() - 1) / p.tile_classes()), int(p.padded_rows), out);
    return done();
  }

  template <class O>
  void sum(size_t at, int parts, int64_t part, const int* place, int64_t n, void* out, int64_t ld, bool add, const Totals& totals) const {
    using E = typename O::Elem;
    const bool whole = aligned_to(out, 4 * sizeof(E)) && ld % 4 == 0;
    hipLaunchKernelGGL(k_vocab_sum<O>, dim3(grid(n * ((p.width + 3) / 4)) + (totals.stats != nullptr ? 1 : 0)), dim3(256), 0, s, get<float>(at), parts,
                       (long long)part, p.padded_width, place, rows.factor, (long long)n, p.width, static_cast<E*>(out), (long long)ld, whole, add, totals);
  }
  // f(the product for piece k of the weight's gradient), and what the piece needs after it
  template <int GP, class O, class F>
  void weight_grad(const acdc_vocab_grads& g, int k, F&& f) const {
    using E = typename O::Elem;
    const int n = classes_of(k);
    E* out = static_cast<E*>(g.weight) + int64_t(k) * p.piece * g.weight_stride;
    const bool whole = aligned_to(out, 4 * sizeof(E)) && g.weight_stride % 4 == 0, add = g.accumulate != 0;
    auto with = [&](const auto& e) {
      constexpr Count K = Count::kK;
      if (!p.large_weight) f(product<SmallOf<P>, GP, true, true, K>(hidden(), grad(k), p.width, n, 0, p.weight_parts, e));
      else f(product<LargeOf<P, GP>, GP, true, true, K>(hidden(), grad(k), p.width, n, 0, p.weight_parts, e));
    };
    if (p.weight_parts == 1) {
      with(GradOut<O>{out, rows.factor, g.weight_stride, p.width, n, whole, add});
    } else {
      const int64_t part = int64_t(p.piece) * p.padded_width;
      with(PartOut{get<float>(w.weight_sums), part, p.padded_width, n, false});
      sum<O>(w.weight_sums, p.weight_parts, part, nullptr, n, out, g.weight_stride, add, Totals{});
    }
  }
  // G of a single piece from what the first pass kept
  template <int GP>
  void slopes(const float* logp) const {
    const int blocks = (p.piece + 511) / 512;
    hipLaunchKernelGGL((k_vocab_slopes<GP, std::conditional_t<GP == 1, __bf16, float>>), dim3(unsigned((p.padded_rows * blocks + 3) / 4)),
                       dim3(256), 0, s, rows, get<RowSlope>(w.slope), get<float2>(w.parts), logp, get<void>(w.kept), get<__bf16>(w.grad),
                       (long long)(p.padded_rows * p.piece), p.piece, p.tile_classes(), int(p.padded_rows), blocks);
  }
  // G of piece k from its logits, computed again
  template <int GP>
  void slopes_again(const Operand& weight, int k) const {
    const int64_t plane = p.padded_rows * p.piece;
    if constexpr (GP > 1) {
      if (p.few_logits) {
        const FewLogits l = few_logits(weight, k);
        hipLaunchKernelGGL(k_vocab_few_slopes<GP>, dim3(few_grid(l)), dim3(256), 0, s, l, get<RowSlope>(w.slope), get<__bf16>(w.grad),
                           (long long)plane);
        return;
      }
    }
    logits<(GP > 1)>(weight, 1, SlopeOut<GP>{get<RowSlope>(w.slope), get<__bf16>(w.grad), plane, p.piece, k * p.piece, classes_of(k)});
  }
  // With the rows' slopes or, of few tiles, G itself in place.  `kept`: the logp of the pass
  // that kept the only piece's exponentials (or G); `packed`: the piece of the weight that was
  // packed last; `totals`: for the last launch if it is one over rows.
  int gradients(const acdc_vocab_grads& g, const float* kept, int packed, const Totals& totals) const {
    if constexpr (P == 3) {
      return gradients_of<3>(g, kept, packed, totals);
    } else {
      return p.grad_planes == 1 ? gradients_of<1>(g, kept, packed, totals) : gradients_of<2>(g, kept, packed, totals);
    }
  }
  // Both gradients' products: in one launch where their tiles are of one shape.  dh of no
  // parts: the weight's alone (in the same kernel, which holds its loop in registers).
  template <int GP, class G, class H>
  void both(const G& dh, const H& dw) const {
    // (one plane of G means large tiles in one of them at least)
    constexpr bool IS_SMALL = std::is_same_v<typename G::Shape, Small>;
    if constexpr (std::is_same_v<typename G::Shape, typename H::Shape> && !(GP == 1 && IS_SMALL)) {
      launch(dh, dw);
    } else {
      if (dh.parts > 0) launch(dh);
      launch(dw);
    }
  }
  template <int GP>
  int gradients_of(const acdc_vocab_grads& g, const float* kept, int packed, const Totals& totals) const {
    const int64_t part = p.padded_rows * p.padded_width;
    for (int k = 0; k < p.pieces; ++k) {
      const Operand wk = weight(k, k == packed);
      packed = k;
      if (kept == nullptr) slopes_again<GP>(wk, k);
      else if (!few()) slopes<GP>(kept);
      auto weight_too = [&](auto&& f) {
        if (g.weight_type == head.dtype) weight_grad<GP, T>(g, k, f);
        else weight_grad<GP, F32>(g, k, f);
      };
      over_rows<GP, true, (GP > 1)>(p.large_hidden, wk, grad(k), p.width, classes_of(k), g.hidden != nullptr ? p.hidden_parts : 0,
                          PartOut{get<float>(w.hidden_sums), part, p.padded_width, int(p.padded_rows), k > 0}, [&](const auto& dh) {
                            if (g.weight == nullptr) return launch(dh);
                            weight_too([&](const auto& dw) { both<GP>(dh, dw); });
                          });
    }
    if (g.hidden != nullptr && p.rows > 0) sum<T>(w.hidden_sums, p.hidden_parts, part, rows.at, p.rows, g.hidden, g.hidden_stride, false, totals);
    return done();
  }
};

// ---------------------------------------------------------------------- checks

constexpr int64_t kMostRows = 1 << 24, kMostClasses = 1 << 27, kMostWidth = 1 << 17, kMostStride = int64_t(1) << 40;

bool sizes_ok(int64_t rows, int32_t width, int32_t classes, int32_t dtype) {
  return dtype_bytes(dtype) != 0 && rows >= 0 && rows <= kMostRows && width >= 1 && width <= kMostWidth && classes >= 1 &&
         classes <= kMostClasses;
}

bool head_ok(const acdc_vocab_head* h) {
  if (h == nullptr || !sizes_ok(h->rows, h->width, h->classes, h->dtype) || (h->target_bits != 32 && h->target_bits != 64))
    return false;
  const size_t e = dtype_bytes(h->dtype);
  if (h->hidden_stride < h->width || h->hidden_stride > kMostStride || h->weight_stride < h->width || h->weight_stride > kMostStride)
    return false;
  if (h->weight == nullptr || !aligned_to(h->weight, e)) return false;
  return h->rows == 0 || (h->hidden != nullptr && aligned_to(h->hidden, e) && h->targets != nullptr &&
                          aligned_to(h->targets, size_t(h->target_bits) / 8));
}
bool grads_ok(const acdc_vocab_head& h, const acdc_vocab_grads& g) {
  if (g.hidden != nullptr && (!aligned_to(g.hidden, dtype_bytes(h.dtype)) || g.hidden_stride < h.width || g.hidden_stride > kMostStride))
    return false;
  return g.weight == nullptr || ((g.weight_type == ACDC_F32 || g.weight_type == h.dtype) && aligned_to(g.weight, dtype_bytes(g.weight_type)) &&
                                 g.weight_stride >= h.width && g.weight_stride <= kMostStride);
}
// What a call reads and writes, to be compared: the head, `read` rows of values (4 bytes each), and
// the gradients, `written` ones and the workspace's part that the call uses.
struct Touched {
  Span x, w, t, read[3], written[4], gx, gw;
  Touched(const acdc_vocab_head& h, const acdc_vocab_grads* g) {
    const size_t e = dtype_bytes(h.dtype);
    x = span_of(h.hidden, h.rows, h.hidden_stride, h.width, e);
    w = span_of(h.weight, h.classes, h.weight_stride, h.width, e);
    t = span_of(h.targets, h.rows, size_t(h.target_bits) / 8);
    if (g == nullptr) return;
    gx = span_of(g->hidden, h.rows, g->hidden_stride, h.width, e);
    gw = span_of(g->weight, h.classes, g->weight_stride, h.width, dtype_bytes(g->weight_type));
  }
  bool ok() const {
    return all_apart({gx, gw, written[0], written[1], written[2], written[3]}, {x, w, t, read[0], read[1], read[2]});
  }
  bool ok(const void* workspace, size_t bytes) const {
    return all_apart({span_of(workspace, int64_t(bytes), 1)},
                     {x, w, t, read[0], read[1], read[2], gx, gw, written[0], written[1], written[2], written[3]});
  }
};
bool wants(const acdc_vocab_grads* g) { return g != nullptr && (g->hidden != nullptr || g->weight != nullptr); }

int workspace_ok(const acdc_vocab_head& h, bool gradient, const void* workspace, size_t bytes, const Touched& touched) {
  if (!aligned_to(workspace, 256)) return ACDC_ERR_INVALID_ARG;
  const size_t need = layout(plan_for(h.rows, h.width, h.classes, h.dtype), gradient).bytes;
  if (workspace == nullptr || bytes < need) return ACDC_ERR_WORKSPACE;
  return touched.ok(workspace, need) ? ACDC_OK : ACDC_ERR_INVALID_ARG;
}
template <class F>
int with_type(int32_t dtype, F&& f) {
  return dtype == ACDC_F32 ? f.template operator()<F32>() : f.template operator()<BF16>();
}

}  // namespace
}  // namespace acdc

using namespace acdc;

extern "C" size_t acdc_vocab_workspace_size(int64_t rows, int32_t width, int32_t classes, int32_t dtype, int32_t gradient) {
  return sizes_ok(rows, width, classes, dtype) ? layout(plan_for(rows, width, classes, dtype), gradient != 0).bytes : 0;
}

extern "C" int acdc_vocab_logprob(const acdc_vocab_head* head, float* logp, float* saved, void* workspace,
                                  size_t workspace_bytes, acdc_stream_t stream) {
  if (!head_ok(head)) return ACDC_ERR_INVALID_ARG;
  if (head->rows == 0) return ACDC_OK;
  if (logp == nullptr || !aligned_to(logp, 4) || !aligned_to(saved, 8)) return ACDC_ERR_INVALID_ARG;
  Touched touched(*head, nullptr);
  touched.written[0] = span_of(logp, head->rows, 4);
  touched.written[1] = span_of(saved, 2 * head->rows, 4);
  if (!touched.ok()) return ACDC_ERR_INVALID_ARG;
  if (const int rc = workspace_ok(*head, false, workspace, workspace_bytes, touched); rc != ACDC_OK) return rc;
  return with_type(head->dtype, [&]<class T>() {
    const Call<T> c(*head, false, workspace, stream);
    c.pack_rows(nullptr, Factor{nullptr, 1.f, false}, logp, reinterpret_cast<float2*>(saved), nullptr);
    return c.statistics(JoinOut{logp, reinterpret_cast<float2*>(saved), nullptr, nullptr, nullptr, false}, false);
  });
}

extern "C" int acdc_vocab_backward(const acdc_vocab_head* head, const float* saved, const float* grad_logp, const float* scale,
                                   const acdc_vocab_grads* grads, void* workspace, size_t workspace_bytes, acdc_stream_t stream) {
  if (!head_ok(head) || grads == nullptr || !grads_ok(*head, *grads) || !aligned_to(scale, 4)) return ACDC_ERR_INVALID_ARG;
  if (head->rows > 0 && (saved == nullptr || !aligned_to(saved, 8) || grad_logp == nullptr || !aligned_to(grad_logp, 4)))
    return ACDC_ERR_INVALID_ARG;
  Touched touched(*head, grads);
  touched.read[0] = span_of(saved, 2 * head->rows, 4);
  touched.read[1] = span_of(grad_logp, head->rows, 4);
  touched.read[2] = span_of(scale, 1, 4);
  if (!touched.ok()) return ACDC_ERR_INVALID_ARG;
  if (!wants(grads)) return ACDC_OK;
  if (const int rc = workspace_ok(*head, true, workspace, workspace_bytes, touched); rc != ACDC_OK) return rc;
  return with_type(head->dtype, [&]<class T>() {
    const Call<T> c(*head, true, workspace, stream);
    c.pack_rows(grad_logp, Factor{scale, 1.f, false}, nullptr, nullptr, nullptr);
    hipLaunchKernelGGL(k_vocab_slope, dim3(Call<T>::grid(c.p.padded_rows)), dim3(256), 0, c.s, c.rows,
                       reinterpret_cast<const float2*>(saved), int(c.p.padded_rows), c.template get<RowSlope>(c.w.slope));
    return c.gradients(*grads, nullptr, 0, Totals{});
  });
}

extern "C" int acdc_vocab_loss(const acdc_vocab_head* head, const float* weights, const acdc_vocab_params* params, float* stats,
                               float* logp, float* saved, float* row_grads, const acdc_vocab_grads* grads, void* workspace,
                               size_t workspace_bytes, acdc_stream_t stream) {
  if (!head_ok(head) || params == nullptr || stats == nullptr || !aligned_to(stats, 4) || !aligned_to(weights, 4) ||
      !aligned_to(logp, 4) || !aligned_to(saved, 8) || !aligned_to(row_grads, 4))
    return ACDC_ERR_INVALID_ARG;
  const acdc_vocab_params q = *params;
  if (!(q.grad_scale - q.grad_scale == 0.f) || (head->rows > 0 && logp == nullptr) || (grads != nullptr && !grads_ok(*head, *grads)))
    return ACDC_ERR_INVALID_ARG;
  const bool gradient = wants(grads);
  Touched touched(*head, grads);
  touched.read[0] = span_of(weights, head->rows, 4);
  touched.written[0] = span_of(stats, 2, 4);
  touched.written[1] = span_of(logp, head->rows, 4);
  touched.written[2] = span_of(saved, 2 * head->rows, 4);
  touched.written[3] = span_of(row_grads, head->rows, 4);
  if (!touched.ok()) return ACDC_ERR_INVALID_ARG;
  if (const int rc = workspace_ok(*head, gradient, workspace, workspace_bytes, touched); rc != ACDC_OK) return rc;
  return with_type(head->dtype, [&]<class T>() {
    const Call<T> c(*head, gradient, workspace, stream);
    float2* stat = reinterpret_cast<float2*>(saved);
    float* loss = c.template get<float>(c.w.loss);
    const bool keep = gradient && c.p.pieces == 1;
    c.pack_rows(weights, Factor{nullptr, q.grad_scale, q.mean != 0}, logp, stat, row_grads);
    // the totals: in the last launch, if it is one over rows
    const bool last = gradient && grads->hidden != nullptr && head->rows > 0;
    const Totals totals{c.rows, loss, stats, q.mean != 0};
    int rc = c.statistics(JoinOut{logp, stat, row_grads, gradient ? c.template get<RowSlope>(c.w.slope) : nullptr,
                                  loss, q.mean != 0},
                          keep);
    if (rc != ACDC_OK) return rc;
    if (!last) hipLaunchKernelGGL(k_vocab_total, dim3(1), dim3(256), 0, c.s, totals);
    rc = done();
    return rc != ACDC_OK || !gradient ? rc : c.gradients(*grads, keep ? logp : nullptr, c.p.pieces - 1, last ? totals : Totals{});
  });
}
