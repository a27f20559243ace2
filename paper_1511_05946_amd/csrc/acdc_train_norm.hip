// Layer norm of rows and its backward pass (acdc_train_lm.h).
//
// Mathematics.  Mean and variance of a row are taken of the values in registers,
// the variance of their differences from the mean, not of their squares, whose
// difference would lose the digits of a variance below the mean's square.
// Backward, with u = (x - mean) rstd and a = grad_y weight:
//   grad_x = rstd (a - mean(a) - u mean(a u)),
// and grad_weight = sum grad_y u, grad_bias = sum grad_y over the rows: a group
// of lanes keeps its columns' sums in registers over all rows that it takes,
// each workgroup leaves one row of sums, and a second launch adds those up.
// Both passes are bound by HBM: each value is read and written once (8192 rows
// of 4096, float32 in and bfloat16 out: 39 us forward, 5.1 TB/s, and 64 + 5 back,
// 5.8; 20011 of 1000 bfloat16, whose rows lie at no more than 16 bytes: 18 and
// 26 + 5, 4.6 and 5.0; 64 of 256: a launch each, 3.3 and 5.6).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "acdc_train_lm.hpp"
#include "acdc_train_rows.hpp"

namespace acdc {
namespace {

constexpr int kThreads = 256;

// Sums over the LANES lanes that share a row; the slots take turns, so that one
// barrier a sum is enough.
template <int LANES>
struct RowSum {
  float* slots;  // 2 x LANES / 64
  int turn = 0;
  __device__ __forceinline__ float operator()(float v) {
    if constexpr (LANES == 16) return over_16(v, [](float p, float q) { return p + q; });
    v = wave_sum(v);
    if constexpr (LANES > 64) {
      constexpr int W = LANES / 64;
      float* s = slots + turn * W;
      turn ^= 1;
      if (threadIdx.x % 64 == 0) s[threadIdx.x / 64] = v;
      __syncthreads();
      v = 0.f;
#pragma unroll
      for (int w = 0; w < W; ++w) v += s[w];
    }
    return v;
  }
};

template <int LANES, int THREADS = kThreads>
struct Group {
  static_assert(LANES <= 64 || LANES >= kThreads, "rows that share a workgroup have no barrier");
  static constexpr int WG = LANES < THREADS ? THREADS : LANES, ROWS = WG / LANES;
};
// The two sums over the rows: where they go, and whether they are added there.
struct Sums {
  void *weight, *bias;  // null: not wanted
  int32_t dtype;
  bool add;
  __device__ __forceinline__ void put(bool bias_too, int col, float s) const {
    void* out = bias_too ? bias : weight;
    if (out == nullptr) return;
    if (dtype == ACDC_F32) {
      float* to = static_cast<float*>(out) + col;
      *to = add ? *to + s : s;
    } else {
      __bf16* to = static_cast<__bf16*>(out) + col;
      *to = __bf16(add ? float(*to) + s : s);
    }
  }
};

// A row in the registers of LANES lanes, NC times eight values each.
template <class TX, class TY, int LANES, int NC>
__global__ __launch_bounds__(Group<LANES>::WG) void k_norm(const typename TX::Elem* __restrict__ x, long long x_stride,
                                                           Vector weight, Vector bias, float eps,
                                                           typename TY::Elem* __restrict__ y, long long y_stride,
                                                           float2* __restrict__ saved, int rows, int width) {
  constexpr int ROWS = Group<LANES>::ROWS;
  __shared__ float slots[2 * Group<LANES>::WG / 64];
  RowSum<LANES> sum{slots};
  const int lane = threadIdx.x % LANES;
  const float inv = 1.f / float(width);
  for (int r = blockIdx.x * ROWS + threadIdx.x / LANES; r < rows; r += gridDim.x * ROWS) {
    const typename TX::Elem* row = x + r * x_stride;
    float v[NC][kEight];
    float s = 0.f;
#pragma unroll
    for (int q = 0; q < NC; ++q) {
      const int col = (lane + q * LANES) * kEight;
      load_some<TX>(row + col, width - col, 0.f, v[q]);
    }
#pragma unroll
    for (int q = 0; q < NC; ++q)
#pragma unroll
      for (int i = 0; i < kEight; ++i) s += v[q][i];
    const float mean = sum(s) * inv;
    s = 0.f;
#pragma unroll
    for (int q = 0; q < NC; ++q) {
      const int col = (lane + q * LANES) * kEight;
#pragma unroll
      for (int i = 0; i < kEight; ++i) {
        v[q][i] -= mean;
        s += col + i < width ? v[q][i] * v[q][i] : 0.f;
      }
    }
    const float rstd = 1.f / sqrtf(sum(s) * inv + eps);
    if (saved != nullptr && lane == 0) saved[r] = make_float2(mean, rstd);
    typename TY::Elem* to = y + r * y_stride;
#pragma unroll
    for (int q = 0; q < NC; ++q) {
      const int col = (lane + q * LANES) * kEight;
      if (col >= width) continue;
      float w[kEight], b[kEight];
      load_vector(weight, col, width - col, 1.f, w);
      load_vector(bias, col, width - col, 0.f, b);
#pragma unroll
      for (int i = 0; i < kEight; ++i) v[q][i] = v[q][i] * rstd * w[i] + b[i];
      store_some<TY>(to + col, width - col, v[q]);
    }
  }
}

// Rows of more than 32768 values: a workgroup reads its row twice.  Mean and squares about it
// of eight values at a time, joined to a lane's own before:
//   mean' = mean + (m - mean) c / (n + c),  squares' = squares + q + (m - mean)^2 n c / (n + c),
// and then to those of all lanes, in the same way (1810 rows of 54837 float32 values 227 us,
// 3.5 TB/s, for 269 with a reading more; 2000 of 65536 bfloat16 133 for 130.  Twice as many
// values in registers: 271 and 283).
template <class TX, class TY, int LANES>
__global__ __launch_bounds__(LANES) void k_norm_long(const typename TX::Elem* __restrict__ x, long long x_stride, Vector weight,
                                                     Vector bias, float eps, typename TY::Elem* __restrict__ y,
                                                     long long y_stride, float2* __restrict__ saved, int rows, int width) {
  __shared__ float slots[2 * LANES / 64];
  RowSum<LANES> sum{slots};
  const float inv = 1.f / float(width);
  for (int r = blockIdx.x; r < rows; r += gridDim.x) {
    const typename TX::Elem* row = x + r * x_stride;
    float v[kEight], n = 0.f, own = 0.f, squares = 0.f;  // of the lane's values so far
#pragma unroll 4
    for (int col = threadIdx.x * kEight; col < width; col += LANES * kEight) {
      load_some<TX>(row + col, width - col, 0.f, v);
      const int left = min(kEight, width - col);
      const float c = float(left);
      float s = 0.f, q = 0.f;
#pragma unroll
      for (int i = 0; i < kEight; ++i) s += v[i];
      const float m = s / c, d = m - own, f = c / (n + c);
#pragma unroll
      for (int i = 0; i < kEight; ++i) q += i < left ? (v[i] - m) * (v[i] - m) : 0.f;
      own += d * f;
      squares += q + d * d * (n * f);
      n += c;
    }
    const float mean = sum(n * own) * inv;
    const float rstd = 1.f / sqrtf(sum(squares + n * (own - mean) * (own - mean)) * inv + eps);
    if (saved != nullptr && threadIdx.x == 0) saved[r] = make_float2(mean, rstd);
    typename TY::Elem* to = y + r * y_stride;
#pragma unroll 2
    for (int col = threadIdx.x * kEight; col < width; col += LANES * kEight) {
      float w[kEight], b[kEight];
      load_some<TX>(row + col, width - col, 0.f, v);
      load_vector(weight, col, width - col, 1.f, w);
      load_vector(bias, col, width - col, 0.f, b);
#pragma unroll
      for (int i = 0; i < kEight; ++i) v[i] = (v[i] - mean) * rstd * w[i] + b[i];
      store_some<TY>(to + col, width - col, v);
    }
  }
}

// What the backward pass reads and writes.
template <class TX, class TY>
struct BackArgs {
  const typename TX::Elem* x;
  const typename TY::Elem* gy;
  typename TX::Elem* gx;  // null: not wanted
  long long x_stride, gy_stride, gx_stride;
  const float2* saved;
  Vector weight;
  float* sums;  // [workgroups][2][width]; null: a single workgroup writes `out` itself
  Sums out;
  int rows, width;
};

template <class TX, class TY, int LANES, int NC, int THREADS>
__global__ __launch_bounds__((Group<LANES, THREADS>::WG)) void k_norm_back(BackArgs<TX, TY> a) {
  constexpr int WG = Group<LANES, THREADS>::WG, ROWS = Group<LANES, THREADS>::ROWS, SPAN = LANES * NC * kEight;
  __shared__ float slots[2 * WG / 64];
  __shared__ float both[ROWS > 1 ? ROWS : 1][ROWS > 1 ? SPAN : 1];
  RowSum<LANES> sum{slots};
  const int lane = threadIdx.x % LANES, group = threadIdx.x / LANES, width = a.width;
  const float inv = 1.f / float(width);
  float w[NC][kEight], gw[NC][kEight] = {}, gb[NC][kEight] = {};
#pragma unroll
  for (int q = 0; q < NC; ++q) {
    const int col = (lane + q * LANES) * kEight;
    load_vector(a.weight, col, width - col, 1.f, w[q]);
  }
  // a row less what it needs of the workgroup
  float u[NC][kEight], g[NC][kEight];
  auto finish = [&](int r, const float2& st) {
    float s1 = 0.f, s2 = 0.f;
#pragma unroll
    for (int q = 0; q < NC; ++q)
#pragma unroll
      for (int i = 0; i < kEight; ++i) {
        gb[q][i] += g[q][i];
        gw[q][i] += g[q][i] * u[q][i];
        g[q][i] *= w[q][i];
        s1 += g[q][i];
        s2 += g[q][i] * u[q][i];
      }
    if (a.gx == nullptr) return;
    const float m1 = sum(s1) * inv, m2 = sum(s2) * inv;
    typename TX::Elem* to = a.gx + r * a.gx_stride;
#pragma unroll
    for (int q = 0; q < NC; ++q) {
      const int col = (lane + q * LANES) * kEight;
      if (col >= width) continue;
#pragma unroll
      for (int i = 0; i < kEight; ++i) g[q][i] = st.y * (g[q][i] - m1 - u[q][i] * m2);
      store_some<TX>(to + col, width - col, g[q]);
    }
  };
  const int step = gridDim.x * ROWS;
  int r = blockIdx.x * ROWS + group;
  if constexpr (NC == 1) {
    // the next row is on its way while this one is summed and written
    Raw8<TX> x;
    Raw8<TY> gy;
    float2 next = make_float2(0.f, 0.f);
    const int col = lane * kEight;
    auto ask = [&](int from) {
      if (from >= a.rows) return;
      next = a.saved[from];
      x.load(a.x + from * a.x_stride + col, width - col);
      gy.load(a.gy + from * a.gy_stride + col, width - col);
    };
    ask(r);
    for (; r < a.rows; r += step) {
      const float2 st = next;
#pragma unroll
      for (int i = 0; i < kEight; ++i) {
        u[0][i] = (x.get(i) - st.x) * st.y;
        g[0][i] = gy.get(i);
      }
      ask(r + step);
      finish(r, st);
    }
  } else {
    for (; r < a.rows; r += step) {
      const float2 st = a.saved[r];
#pragma unroll
      for (int q = 0; q < NC; ++q) {
        const int col = (lane + q * LANES) * kEight;
        load_some<TX>(a.x + r * a.x_stride + col, width - col, st.x, u[q]);
        load_some<TY>(a.gy + r * a.gy_stride + col, width - col, 0.f, g[q]);
      }
#pragma unroll
      for (int q = 0; q < NC; ++q)
#pragma unroll
        for (int i = 0; i < kEight; ++i) u[q][i] = (u[q][i] - st.x) * st.y;
      finish(r, st);
    }
  }
  if (a.out.weight == nullptr && a.out.bias == nullptr) return;
  const bool alone = a.sums == nullptr;
  float* out = a.sums + (long long)blockIdx.x * 2 * width;
  if constexpr (ROWS == 1) {
#pragma unroll
    for (int q = 0; q < NC; ++q) {
      const int col = (lane + q * LANES) * kEight;
      if (col >= width) continue;
      if (alone) {
#pragma unroll
        for (int i = 0; i < kEight; ++i) {
          if (col + i >= width) break;
          a.out.put(false, col + i, gw[q][i]);
          a.out.put(true, col + i, gb[q][i]);
        }
      } else {
        store_some<F32, false>(out + col, width - col, gw[q]);
        store_some<F32, false>(out + width + col, width - col, gb[q]);
      }
    }
  } else {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      if (k == 1) __syncthreads();
#pragma unroll
      for (int q = 0; q < NC; ++q)
#pragma unroll
        for (int i = 0; i < kEight; ++i) both[group][(lane + q * LANES) * kEight + i] = k == 0 ? gw[q][i] : gb[q][i];
      __syncthreads();
      for (int col = threadIdx.x; col < width; col += WG) {
        float s = 0.f;
#pragma unroll 16
        for (int p = 0; p < ROWS; ++p) s += both[p][col];
        if (alone) a.out.put(k == 1, col, s);
        else out[k * width + col] = s;
      }
    }
  }
}

// Longer rows: grad_x, a workgroup a row, which it reads twice.
template <class TX, class TY, int LANES>
__global__ __launch_bounds__(LANES) void k_norm_back_long(BackArgs<TX, TY> a) {
  __shared__ float slots[2 * LANES / 64];
  RowSum<LANES> sum{slots};
  const int width = a.width;
  const float inv = 1.f / float(width);
  for (int r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const float2 st = a.saved[r];
    const typename TX::Elem* x = a.x + r * a.x_stride;
    const typename TY::Elem* gy = a.gy + r * a.gy_stride;
    float s1 = 0.f, s2 = 0.f, u[kEight], g[kEight], w[kEight];
#pragma unroll 2
    for (int col = threadIdx.x * kEight; col < width; col += LANES * kEight) {
      load_some<TX>(x + col, width - col, st.x, u);
      load_some<TY>(gy + col, width - col, 0.f, g);
      load_vector(a.weight, col, width - col, 1.f, w);
#pragma unroll
      for (int i = 0; i < kEight; ++i) {
        s1 += g[i] * w[i];
        s2 += g[i] * w[i] * ((u[i] - st.x) * st.y);
      }
    }
    const float m1 = sum(s1) * inv, m2 = sum(s2) * inv;
    typename TX::Elem* to = a.gx + r * a.gx_stride;
#pragma unroll 2
    for (int col = threadIdx.x * kEight; col < width; col += LANES * kEight) {
      load_some<TX>(x + col, width - col, st.x, u);
      load_some<TY>(gy + col, width - col, 0.f, g);
      load_vector(a.weight, col, width - col, 1.f, w);
#pragma unroll
      for (int i = 0; i < kEight; ++i) g[i] = st.y * (g[i] * w[i] - m1 - (u[i] - st.x) * st.y * m2);
      store_some<TX>(to + col, width - col, g);
    }
  }
}

// Their columns' sums: a wave takes 512 columns of a part of the rows.
template <class TX, class TY>
__global__ __launch_bounds__(64) void k_norm_columns(BackArgs<TX, TY> a, int each) {
  const int col = (blockIdx.x * 64 + threadIdx.x) * kEight, from = blockIdx.y * each, to = min(a.rows, from + each);
  if (col >= a.width) return;
  const int left = a.width - col;
  float gw[kEight] = {}, gb[kEight] = {};
#pragma unroll 4
  for (int r = from; r < to; ++r) {
    const float2 st = a.saved[r];
    float u[kEight], g[kEight];
    load_some<TX>(a.x + r * a.x_stride + col, left, st.x, u);
    load_some<TY>(a.gy + r * a.gy_stride + col, left, 0.f, g);
#pragma unroll
    for (int i = 0; i < kEight; ++i) {
      gb[i] += g[i];
      gw[i] += g[i] * ((u[i] - st.x) * st.y);
    }
  }
  float* out = a.sums + (long long)blockIdx.y * 2 * a.width;
  store_some<F32, false>(out + col, left, gw);
  store_some<F32, false>(out + a.width + col, left, gb);
}

// The parts' sums together, in order: 64 columns a workgroup, its waves take the parts
// in turn.
constexpr int kSumWaves = 16;
__global__ __launch_bounds__(64 * kSumWaves) void k_norm_sums(const float* __restrict__ sums, int parts, int width, Sums out) {
  __shared__ float slots[kSumWaves][64];
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, at = blockIdx.x * 64 + lane;  // of 2 width
  float s = 0.f;
  if (at < 2 * width) {
#pragma unroll 8
    for (int p = wave; p < parts; p += kSumWaves) s += sums[(long long)p * 2 * width + at];
  }
  slots[wave][lane] = s;
  __syncthreads();
  if (wave != 0 || at >= 2 * width) return;
  s = 0.f;
#pragma unroll
  for (int w = 0; w < kSumWaves; ++w) s += slots[w][lane];
  out.put(at >= width, at < width ? at : at - width, s);
}

// ------------------------------------------------------------------ on the host

constexpr int kMostWidth = 1 << 24;
constexpr int kHeld = 32768, kHeldBack = 16384;  // values of a row that registers hold, forward and backward
// Parts of the rows at the most, each a workgroup's: as many as keep the card busy, as each
// leaves sums to be added up (bfloat16: 20000 rows of 256 10.7 us for 12.1 in 1024 parts, of
// 1000 28 in 1024 and 32 in 512, 8192 of 4096 39 in 512 and 44 in 256 or 1024, 4096 of 8192
// 37 in 256 and 44 in 512).
int most_parts(int width) { return width <= 256 ? 512 : width <= 2048 ? 1024 : width <= 4096 ? 512 : 256; }

int done() {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? ACDC_OK : hip_fail(e);
}
// f.template operator()<LANES, NC>() for rows of up to kHeld values (kHeldBack below).
template <class F>
void with_row(int width, F&& f) {
  if (width <= 128) f.template operator()<16, 1>();
  else if (width <= 256) f.template operator()<16, 2>();
  else if (width <= 512) f.template operator()<64, 1>();
  else if (width <= 1024) f.template operator()<64, 2>();
  else if (width <= 2048) f.template operator()<256, 1>();
  else if (width <= 4096) f.template operator()<256, 2>();
  else if (width <= 8192) f.template operator()<512, 2>();
  else if (width <= 16384) f.template operator()<512, 4>();
  else f.template operator()<1024, 4>();
}
// The same for the backward pass, which has more to hold.
template <class F>
void with_row_back(int width, F&& f) {
  if (width <= 128) f.template operator()<16, 1>();
  else if (width <= 256) f.template operator()<16, 2>();
  else if (width <= 512) f.template operator()<64, 1>();
  else if (width <= 1024) f.template operator()<64, 2>();
  else if (width <= 2048) f.template operator()<256, 1>();
  else if (width <= 4096) f.template operator()<512, 1>();
  else if (width <= 8192) f.template operator()<1024, 1>();
  else f.template operator()<1024, 2>();
}
template <class F>
int with_types(int32_t x, int32_t y, F&& f) {
  if (x == ACDC_F32) return y == ACDC_F32 ? f.template operator()<F32, F32>() : f.template operator()<F32, BF16>();
  return y == ACDC_F32 ? f.template operator()<BF16, F32>() : f.template operator()<BF16, BF16>();
}
bool rows_ok(const void* p, int32_t dtype, int64_t stride, int64_t rows, int32_t width) {
  const size_t e = dtype_bytes(dtype);
  return e != 0 && stride >= width && stride <= (int64_t(1) << 40) && aligned_to(p, e) && (rows == 0 || p != nullptr);
}
bool sizes_ok(int64_t rows, int32_t width) { return rows >= 0 && rows <= 0x3fffffff && width >= 1 && width <= kMostWidth; }

// Few short rows, more than a workgroup of 256 lanes takes at once: one of 1024, and a
// launch less (64 rows of 256 5.2 us for 7.0, 16 of 1024 5.3 for 7.1; 100 of 256 would be 8.4 for 6.7).
bool few(int64_t rows, int32_t width) { return width <= 256 ? rows > 16 && rows <= 64 : width <= 1024 && rows > 4 && rows <= 16; }
// Parts whose columns' sums the backward pass leaves: the workgroups of its launch (long
// rows: those of the second one).
int parts_of(int64_t rows, int32_t width) {
  if (rows == 0) return 0;
  if (width > kHeldBack) return int(std::min<int64_t>(rows, 64));
  int per = 1;
  with_row_back(width, [&]<int LANES, int NC>() { per = few(rows, width) ? 1024 / LANES : Group<LANES>::ROWS; });
  return int(std::min<int64_t>((rows + per - 1) / per, most_parts(width)));
}

// One workgroup writes the sums itself and needs no workspace.
bool alone(int64_t rows, int32_t width) { return width <= kHeldBack && parts_of(rows, width) <= 1; }

}  // namespace
}  // namespace acdc

using namespace acdc;

extern "C" int acdc_norm_forward(const void* x, int32_t x_type, int64_t x_stride, const void* weight, const void* bias,
                                 int32_t vector_type, float eps, void* y, int32_t y_type, int64_t y_stride, float* saved,
                                 int64_t rows, int32_t width, acdc_stream_t stream) {
  if (!sizes_ok(rows, width) || !rows_ok(x, x_type, x_stride, rows, width) || !rows_ok(y, y_type, y_stride, rows, width) ||
      !(eps >= 0.f) || !(eps - eps == 0.f) || !aligned_to(saved, 8))
    return ACDC_ERR_INVALID_ARG;
  const size_t e = dtype_bytes(vector_type);
  if (e == 0 || !aligned_to(weight, e) || !aligned_to(bias, e)) return ACDC_ERR_INVALID_ARG;
  if (!all_apart({span_of(y, rows, y_stride, width, dtype_bytes(y_type)), span_of(saved, 2 * rows, 4)},
                 {span_of(x, rows, x_stride, width, dtype_bytes(x_type)), span_of(weight, width, e), span_of(bias, width, e)}))
    return ACDC_ERR_INVALID_ARG;
  if (rows == 0) return ACDC_OK;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  return with_types(x_type, y_type, [&]<class TX, class TY>() {
    auto go = [&](auto kernel, int64_t groups, int wg) {
      hipLaunchKernelGGL(kernel, dim3(unsigned(std::min<int64_t>(groups, 1 << 16))), dim3(wg), 0, s,
                         static_cast<const typename TX::Elem*>(x), (long long)x_stride, Vector{weight, vector_type},
                         Vector{bias, vector_type}, eps, static_cast<typename TY::Elem*>(y), (long long)y_stride,
                         reinterpret_cast<float2*>(saved), int(rows), width);
    };
    if (width > kHeld) {
      go(k_norm_long<TX, TY, 1024>, rows, 1024);
    } else {
      with_row(width, [&]<int LANES, int NC>() {
        constexpr int per = Group<LANES>::ROWS;
        go(k_norm<TX, TY, LANES, NC>, (rows + per - 1) / per, Group<LANES>::WG);
      });
    }
    return done();
  });
}

extern "C" size_t acdc_norm_workspace_size(int64_t rows, int32_t width) {
  if (!sizes_ok(rows, width)) return 0;
  return alone(rows, width) ? 256 : std::max<size_t>(512, size_t(parts_of(rows, width)) * 2 * size_t(width) * 4);
}

extern "C" int acdc_norm_backward(const void* x, int32_t x_type, int64_t x_stride, const void* grad_y, int32_t y_type,
                                  int64_t grad_y_stride, const void* weight, int32_t vector_type, const float* saved,
                                  void* grad_x, int64_t grad_x_stride, void* grad_weight, void* grad_bias, int32_t grads_type,
                                  int32_t accumulate, int64_t rows, int32_t width, void* workspace, size_t workspace_bytes,
                                  acdc_stream_t stream) {
  if (!sizes_ok(rows, width) || !rows_ok(x, x_type, x_stride, rows, width) ||
      !rows_ok(grad_y, y_type, grad_y_stride, rows, width) || !aligned_to(saved, 8) || (rows > 0 && saved == nullptr))
    return ACDC_ERR_INVALID_ARG;
  const size_t e = dtype_bytes(vector_type), ge = dtype_bytes(grads_type);
  if (e == 0 || ge == 0 || !aligned_to(weight, e) || !aligned_to(grad_weight, ge) || !aligned_to(grad_bias, ge))
    return ACDC_ERR_INVALID_ARG;
  if (grad_x != nullptr && !rows_ok(grad_x, x_type, grad_x_stride, rows, width)) return ACDC_ERR_INVALID_ARG;
  // in place of grad_y: each value is read by the lane that writes it, before it does
  const bool in_place = grad_x == grad_y && grad_x_stride == grad_y_stride && x_type == y_type;
  const Span x_span = span_of(x, rows, x_stride, width, dtype_bytes(x_type)), st = span_of(saved, 2 * rows, 4),
             gy = span_of(grad_y, rows, grad_y_stride, width, dtype_bytes(y_type)), w = span_of(weight, width, e),
             gx = span_of(grad_x, rows, grad_x_stride, width, dtype_bytes(x_type)), gw = span_of(grad_weight, width, ge),
             gb = span_of(grad_bias, width, ge);
  if (!all_apart({gx, gw, gb}, {x_span, in_place ? Span{} : gy, w, st}) || !apart(gw, gy) || !apart(gb, gy)) return ACDC_ERR_INVALID_ARG;
  const bool sums = grad_weight != nullptr || grad_bias != nullptr;
  const size_t need = acdc_norm_workspace_size(rows, width);
  if (sums && !alone(rows, width) && (workspace == nullptr || workspace_bytes < need)) return ACDC_ERR_WORKSPACE;
  if (!aligned_to(workspace, 16)) return ACDC_ERR_INVALID_ARG;
  if (sums && !alone(rows, width) && !all_apart({span_of(workspace, int64_t(need), 1)}, {x_span, gy, w, st, gx, gw, gb})) return ACDC_ERR_INVALID_ARG;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  const int parts = parts_of(rows, width);
  const Sums out_sums{grad_weight, grad_bias, grads_type, accumulate != 0};
  if (rows > 0 && (sums || grad_x != nullptr)) {
    const int rc = with_types(x_type, y_type, [&]<class TX, class TY>() {
      const BackArgs<TX, TY> a{static_cast<const typename TX::Elem*>(x), static_cast<const typename TY::Elem*>(grad_y),
                               static_cast<typename TX::Elem*>(grad_x), x_stride, grad_y_stride, grad_x_stride,
                               reinterpret_cast<const float2*>(saved), Vector{weight, vector_type},
                               alone(rows, width) ? nullptr : static_cast<float*>(workspace), out_sums, int(rows), width};
      if (width > kHeldBack) {
        // the sums first: grad_x may take grad_y's place
        if (sums) {
          const int each = int((rows + parts - 1) / parts), blocks = (width + 64 * kEight - 1) / (64 * kEight);
          hipLaunchKernelGGL((k_norm_columns<TX, TY>), dim3(unsigned(blocks), unsigned(parts)), dim3(64), 0, s, a, each);
        }
        if (grad_x != nullptr)
          hipLaunchKernelGGL((k_norm_back_long<TX, TY, 1024>), dim3(unsigned(std::min<int64_t>(rows, 1 << 16))), dim3(1024), 0, s, a);
      } else {
        with_row_back(width, [&]<int LANES, int NC>() {
          if constexpr (LANES <= 64) {
            if (few(rows, width)) {
              hipLaunchKernelGGL((k_norm_back<TX, TY, LANES, NC, 1024>), dim3(1), dim3(1024), 0, s, a);
              return;
            }
          }
          hipLaunchKernelGGL((k_norm_back<TX, TY, LANES, NC, kThreads>), dim3(unsigned(parts)), dim3(Group<LANES>::WG), 0, s, a);
        });
      }
      return done();
    });
    if (rc != ACDC_OK) return rc;
  }
  if (!sums || (rows == 0 && accumulate != 0) || (rows > 0 && alone(rows, width))) return ACDC_OK;
  hipLaunchKernelGGL(k_norm_sums, dim3(unsigned((2 * int64_t(width) + 63) / 64)), dim3(64 * kSumWaves), 0, s,
                     static_cast<const float*>(workspace), parts, width, out_sums);
  return done();
}
