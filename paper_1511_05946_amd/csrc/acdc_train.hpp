// What the kernels of the training operators share: element types in memory,
// sums over a wave and a workgroup, host-side checks.
#pragma once

#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

#include "acdc_status.hpp"
#include "acdc_train.h"

namespace acdc {

// ------------------------------------------------------------ element types
// A chunk is 16 bytes of a row.  Rows start at any element (odd widths,
// slices of wider rows): the hardware reads and writes 16 bytes at any
// element's alignment, and the aligned(...) types say so to the compiler.
struct F32 {
  using Elem = float;
  static constexpr int kPer = 4;  // values of a chunk
  typedef float Raw __attribute__((ext_vector_type(4), aligned(4)));
  __device__ __forceinline__ static float get(const Raw& r, int i) { return r[i]; }
  __device__ __forceinline__ static float one(Elem e) { return e; }
  __device__ __forceinline__ static Raw pack(const float* v) { return Raw{v[0], v[1], v[2], v[3]}; }
  __device__ __forceinline__ static Elem to(float v) { return v; }
};
struct BF16 {
  using Elem = __bf16;
  static constexpr int kPer = 8;
  typedef unsigned Raw __attribute__((ext_vector_type(4), aligned(2)));
  __device__ __forceinline__ static float get(const Raw& r, int i) {
    return __uint_as_float(i % 2 ? r[i / 2] & 0xffff0000u : r[i / 2] << 16);
  }
  __device__ __forceinline__ static float one(Elem e) { return float(e); }
  // round to nearest, ties to even: the only rounding of a value on its way out
  __device__ __forceinline__ static unsigned pack2(float a, float b) {
    typedef __bf16 Two __attribute__((ext_vector_type(2)));
    const Two t = {__bf16(a), __bf16(b)};
    return __builtin_bit_cast(unsigned, t);
  }
  __device__ __forceinline__ static Raw pack(const float* v) {
    return Raw{pack2(v[0], v[1]), pack2(v[2], v[3]), pack2(v[4], v[5]), pack2(v[6], v[7])};
  }
  __device__ __forceinline__ static Elem to(float v) { return __bf16(v); }
};
template <class T>
__device__ __forceinline__ typename T::Raw load_chunk(const typename T::Elem* p) {
  return *reinterpret_cast<const typename T::Raw*>(p);
}
template <class T>
__device__ __forceinline__ void store_chunk(typename T::Elem* p, const typename T::Raw& r) {
  *reinterpret_cast<typename T::Raw*>(p) = r;
}

// ------------------------------------------------------------- host checks
inline bool aligned_to(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
inline size_t dtype_bytes(int32_t dtype) { return dtype == ACDC_F32 ? 4 : dtype == ACDC_BF16 ? 2 : 0; }

}  // namespace acdc
