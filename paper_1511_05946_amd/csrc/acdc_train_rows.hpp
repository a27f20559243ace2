// Rows of float32 or bfloat16 values as eight at a time, for the operators that
// read one type and write another.
#pragma once

#include "acdc_train.hpp"

namespace acdc {

constexpr int kEight = 8;

template <class T>
__device__ __forceinline__ void load8(const typename T::Elem* p, float (&v)[kEight]) {
#pragma unroll
  for (int q = 0; q < kEight / T::kPer; ++q) {
    const typename T::Raw raw = load_chunk<T>(p + q * T::kPer);
#pragma unroll
    for (int i = 0; i < T::kPer; ++i) v[q * T::kPer + i] = T::get(raw, i);
  }
}
// The first `left` of them (all where there are more); the others are `fill`.
template <class T>
__device__ __forceinline__ void load_some(const typename T::Elem* p, int left, float fill, float (&v)[kEight]) {
  if (left >= kEight) {
    load8<T>(p, v);
  } else {
#pragma unroll
    for (int i = 0; i < kEight; ++i) v[i] = i < left ? T::one(p[i]) : fill;
  }
}
template <class T, bool NT = true>
__device__ __forceinline__ void store_some(typename T::Elem* p, int left, const float (&v)[kEight]) {
  if (left >= kEight) {
#pragma unroll
    for (int q = 0; q < kEight / T::kPer; ++q) {
      typename T::Raw* to = reinterpret_cast<typename T::Raw*>(p + q * T::kPer);
      if constexpr (NT) __builtin_nontemporal_store(T::pack(v + q * T::kPer), to);
      else *to = T::pack(v + q * T::kPer);
    }
  } else {
#pragma unroll
    for (int i = 0; i < kEight; ++i)
      if (i < left) p[i] = T::to(v[i]);
  }
}

// Eight as they lie in memory (those behind `left` are 0), to be asked for ahead.
template <class T>
struct Raw8 {
  typename T::Raw raw[kEight / T::kPer];
  __device__ __forceinline__ void load(const typename T::Elem* p, int left) {
    if (left >= kEight) {
#pragma unroll
      for (int q = 0; q < kEight / T::kPer; ++q) raw[q] = load_chunk<T>(p + q * T::kPer);
    } else {
      float v[kEight];
#pragma unroll
      for (int i = 0; i < kEight; ++i) v[i] = i < left ? T::one(p[i]) : 0.f;
#pragma unroll
      for (int q = 0; q < kEight / T::kPer; ++q) raw[q] = T::pack(v + q * T::kPer);
    }
  }
  __device__ __forceinline__ float get(int i) const { return T::get(raw[i / T::kPer], i % T::kPer); }
};

// The same in 512 columns from `col` on, for the lanes of a wave: eight columns a lane
// that follow one another or, with APART, four and 256 columns on four more.  32 bytes a
// lane would be two instructions that each touch half of every line.
template <class T>
__device__ __forceinline__ void load4(const typename T::Elem* p, int left, float fill, float* v) {
  if (left >= 4) {
    if constexpr (T::kPer == 4) {
      const typename T::Raw raw = load_chunk<T>(p);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = T::get(raw, i);
    } else {
      typedef unsigned Half __attribute__((ext_vector_type(2), aligned(2)));
      const Half raw = *reinterpret_cast<const Half*>(p);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(i % 2 ? raw[i / 2] & 0xffff0000u : raw[i / 2] << 16);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = i < left ? T::one(p[i]) : fill;
  }
}
template <class T, bool NT>
__device__ __forceinline__ void store4(typename T::Elem* p, int left, const float* v) {
  if (left >= 4) {
    if constexpr (T::kPer == 4) {
      typename T::Raw* to = reinterpret_cast<typename T::Raw*>(p);
      if constexpr (NT) __builtin_nontemporal_store(T::pack(v), to);
      else *to = T::pack(v);
    } else {
      typedef unsigned Half __attribute__((ext_vector_type(2), aligned(2)));
      const Half raw = {T::pack2(v[0], v[1]), T::pack2(v[2], v[3])};
      Half* to = reinterpret_cast<Half*>(p);
      if constexpr (NT) __builtin_nontemporal_store(raw, to);
      else *to = raw;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < left) p[i] = T::to(v[i]);
  }
}
template <bool APART>
struct Columns {
  int first, width;  // of the lane's
  __device__ __forceinline__ Columns(int col, int lane, int w) : first(col + lane * (APART ? 4 : kEight)), width(w) {}
  __device__ __forceinline__ bool any() const { return first < width; }
  template <class T>
  __device__ __forceinline__ void load(const typename T::Elem* row, float (&v)[kEight]) const {
    if constexpr (APART) {
      load4<T>(row + first, width - first, 0.f, v);
      load4<T>(row + first + 256, width - first - 256, 0.f, v + 4);
    } else {
      load_some<T>(row + first, width - first, 0.f, v);
    }
  }
  template <class T, bool NT = true>
  __device__ __forceinline__ void store(typename T::Elem* row, const float (&v)[kEight]) const {
    if constexpr (APART) {
      store4<T, NT>(row + first, width - first, v);
      store4<T, NT>(row + first + 256, width - first - 256, v + 4);
    } else {
      store_some<T, NT>(row + first, width - first, v);
    }
  }
};
template <class A, class B>
constexpr bool kApart = A::kPer == 4 || B::kPer == 4;

// A vector whose type a launch knows only when it runs (weights, their gradients).
struct Vector {
  const void* p;  // null: not there
  int32_t dtype;
};
__device__ __forceinline__ void load_vector(const Vector& w, int at, int left, float fill, float (&v)[kEight]) {
  if (w.p == nullptr) {
#pragma unroll
    for (int i = 0; i < kEight; ++i) v[i] = fill;
  } else if (w.dtype == ACDC_F32) {
    load_some<F32>(static_cast<const float*>(w.p) + at, left, 0.f, v);
  } else {
    load_some<BF16>(static_cast<const __bf16*>(w.p) + at, left, 0.f, v);
  }
}

}  // namespace acdc
