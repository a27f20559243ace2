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
// Loads and stores of data that passes through the card once (NT) carry the
// hint that the caches need not keep it: what they hold of other data stays,
// and a write goes out without its line being brought in.
template <bool NT, class V>
__device__ __forceinline__ V load_as(const V* p) {
  if constexpr (NT) return __builtin_nontemporal_load(p);
  else return *p;
}
template <bool NT, class V>
__device__ __forceinline__ void store_as(V* p, const V& v) {
  if constexpr (NT) __builtin_nontemporal_store(v, p);
  else *p = v;
}
template <class T>
__device__ __forceinline__ typename T::Raw load_chunk(const typename T::Elem* p) {
  return *reinterpret_cast<const typename T::Raw*>(p);
}
template <class T>
__device__ __forceinline__ void store_chunk(typename T::Elem* p, const typename T::Raw& r) {
  store_as<true>(reinterpret_cast<typename T::Raw*>(p), r);
}
// The same at a lane's byte offset from an address that the whole wave shares:
// the address stays in scalar registers, and a thread keeps one offset.
template <class T, bool NT = false>
__device__ __forceinline__ typename T::Raw load_chunk_at(const typename T::Elem* p, unsigned fixed, unsigned lane) {
  return load_as<NT>(reinterpret_cast<const typename T::Raw*>((reinterpret_cast<const char*>(p) + fixed) + lane));
}
template <class T>
__device__ __forceinline__ void store_chunk_at(typename T::Elem* p, unsigned fixed, unsigned lane,
                                               const typename T::Raw& r) {
  store_as<true>(reinterpret_cast<typename T::Raw*>((reinterpret_cast<char*>(p) + fixed) + lane), r);
}
// A value that all lanes of the wave hold, moved to a scalar register.
__device__ __forceinline__ float uniform(float v) {
  return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(v)));
}
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// -------------------------------------------------- over the lanes of a wave
// Every lane gets the result: within 16 lanes by DPP (a neighbour's register
// read as an operand), then across them by the lane swaps of gfx950.  A
// shuffle through LDS would take its latency six times over.
template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
  return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), CTRL, 0xf, 0xf, true));
}
struct Pair {
  float a, b;
};
__device__ __forceinline__ Pair swap16(float v) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return {__uint_as_float(r[0]), __uint_as_float(r[1])};
}
__device__ __forceinline__ Pair swap32(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return {__uint_as_float(r[0]), __uint_as_float(r[1])};
}
template <class F>
__device__ __forceinline__ float over_16(float v, F&& f) {
  v = f(v, dpp<0xB1>(v));     // quad_perm 1,0,3,2
  v = f(v, dpp<0x4E>(v));     // quad_perm 2,3,0,1
  v = f(v, dpp<0x141>(v));    // row_half_mirror
  return f(v, dpp<0x140>(v));  // row_mirror
}
template <class F>
__device__ __forceinline__ float over_wave(float v, F&& f) {
  v = over_16(v, f);
  Pair p = swap16(v);
  v = f(p.a, p.b);
  p = swap32(v);
  return f(p.a, p.b);
}
__device__ __forceinline__ float wave_max(float v) {
  return over_wave(v, [](float a, float b) { return fmaxf(a, b); });
}
__device__ __forceinline__ float wave_sum(float v) {
  return over_wave(v, [](float a, float b) { return a + b; });
}

// What a wave's lanes wrote to LDS before it, all of its lanes may read after it.
// (The lanes run together, but without it the compiler may order one lane's load
// before another's store: to a single thread they are different addresses.)
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// ------------------------------------------------------------- host checks
inline bool aligned_to(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
inline size_t dtype_bytes(int32_t dtype) { return dtype == ACDC_F32 ? 4 : dtype == ACDC_BF16 ? 2 : 0; }

}  // namespace acdc
