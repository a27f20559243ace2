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
