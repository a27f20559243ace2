// Matrix product on the matrix cores for the vocabulary's losses:
//   C[m][n] = sum_k A(m, k) B(n, k),  bfloat16 operands, 32-bit sums.
//
// An operand lies in memory with k along its rows ("along"), or with k across
// them ("across": row k holds the values of all m), so that the three products
// of the loss read hidden, weight and the logits' gradient as they are, and
// nothing is transposed on the way.
//
// A workgroup of 4 or 8 waves computes BM x BN of C; steps of 64 k go through
// two halves of LDS.  While the waves compute on one half, the other one is
// filled by loads that write LDS themselves (16 bytes a lane), so that a step
// needs one barrier and no registers in between.  LDS words are permuted by
// the row (Along::swizzle, Across::swizzle): 8 lanes that read 16 bytes each
// touch all banks once, and so do the transposing reads of "across" tiles.
//
// float32 values x = x0 + x1 + x2 are three planes of bfloat16 (8 of 24 bits
// each, exact): the product runs over the six pairs of planes that matter,
// smallest first; what is left out is below 2^-26 of a product.
#pragma once

#include <type_traits>

#include "acdc_train.hpp"

namespace acdc {

using bf16x4 = __bf16 __attribute__((ext_vector_type(4)));
using bf16x8 = __bf16 __attribute__((ext_vector_type(8)));
using f32x4 = float __attribute__((ext_vector_type(4)));
using s16x4 = short __attribute__((ext_vector_type(4)));

#define ACDC_LDS __attribute__((address_space(3)))
#define ACDC_GLOBAL __attribute__((address_space(1)))

constexpr int kStepK = 64;  // k of a step

// x as three bfloat16 whose sum is x.  A value that is not finite stays in the
// first plane; one that would round to infinity is cut instead.
struct Split3 {
  __bf16 p[3];
};
__device__ __forceinline__ Split3 split3(float x) {
  Split3 s;
  s.p[0] = __bf16(x);
  float r = float(s.p[0]);
  if (r - r != 0.f && x - x == 0.f) {
    s.p[0] = __builtin_bit_cast(__bf16, (unsigned short)(__float_as_uint(x) >> 16));
    r = float(s.p[0]);
  }
  const float d = x - r, low = d == d ? d : 0.f;  // inf - inf
  s.p[1] = __bf16(low);
  s.p[2] = __bf16(low - float(s.p[1]));
  return s;
}

// The pairs of planes in order, four bits each.
template <int PLANES>
struct Pairs;
template <>
struct Pairs<1> {
  static constexpr int N = 1;
  static constexpr unsigned A = 0, B = 0;
};
template <>
struct Pairs<3> {
  static constexpr int N = 6;
  static constexpr unsigned A = 0x010210, B = 0x001012;  // 0,1,2,0,1,0 and 2,1,0,1,0,0
};

// rows x cols values in memory, `ld` apart, both >= 1, cols a multiple of 8 and
// rows at multiples of 16 bytes.  A tile may reach past either: it then reads the
// last row or the last 8 columns again, so that every address is inside.
struct Operand {
  const __bf16* p;
  int64_t ld;      // 1024 ld bytes fit in 32 bits
  int64_t plane;   // elements from plane to plane
  int rows, cols;
};

// The tile of X values (m or n) by 64 k of an operand with k along its rows:
// 128 bytes of LDS a value, 8 chunks of 16 bytes.
template <int X, int THREADS, int SPREAD>
struct Along {
  static constexpr int N = X * 8 / THREADS;
  const char* base;
  unsigned off[N];
  int64_t plane;
  int cols, tid;
  // The rows that 8 lanes read at once are 0 .. 7 (SPREAD 0), or 0 .. 3 and four more
  // SPREAD rows on: eight different values for either.
  __device__ __forceinline__ static int swizzle(int row) {
    return SPREAD == 0 ? row & 7 : (row & 3) | (row / (SPREAD > 0 ? SPREAD : 1) & 1) << 2;
  }
  __device__ __forceinline__ void init(const Operand& o, int x0, int t) {
    base = reinterpret_cast<const char*>(o.p + int64_t(x0) * o.ld);
    plane = o.plane * 2;
    cols = o.cols;
    tid = t;
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int c = t + j * THREADS, row = c >> 3;
      off[j] = unsigned(min(row, o.rows - 1 - x0)) * unsigned(o.ld * 2) + unsigned(((c & 7) ^ swizzle(row)) << 4);
    }
  }
  __device__ __forceinline__ void load(char ACDC_LDS* lds, int p, int k, int wave) const {
    const char* at = base + p * plane + int64_t(k) * (kStepK * 2);
    if ((k + 1) * kStepK <= cols) {
#pragma unroll
      for (int j = 0; j < N; ++j) put(lds, at + off[j], j, wave);
    } else {
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const int c = tid + j * THREADS, row = c >> 3, col = ((c & 7) ^ swizzle(row)) * 8;
        put(lds, at + off[j] - (col - min(col, cols - 8 - k * kStepK)) * 2, j, wave);
      }
    }
  }
  __device__ __forceinline__ static void put(char ACDC_LDS* lds, const char* from, int j, int wave) {
    __builtin_amdgcn_global_load_lds((const ACDC_GLOBAL void*)from, (ACDC_LDS void*)(lds + (j * THREADS + wave * 64) * 16),
                                     16, 0, 0);
  }
  // 8 k (of `half`, 32 k) of value `row`, for lane's quarter
  __device__ __forceinline__ static bf16x8 read(const char ACDC_LDS* tile, int row, int half, int lane) {
    return *(const bf16x8 ACDC_LDS*)(tile + row * 128 + ((half * 4 + (lane >> 4)) ^ swizzle(row)) * 16);
  }
};

// The same of an operand with k across its rows: 64 rows of X values.
template <int X, int THREADS>
struct Across {
  static constexpr int N = X * 8 / THREADS, CHUNKS = X / 8;
  const char* base;
  unsigned off[N];
  int64_t plane, step;
  unsigned ld2;
  int rows, tid;
  // A transposing read takes 16 values of the rows k .. k + 3 and k + 8 .. k + 11 at once
  // per half wave: eight times 32 bytes, at eight different places of 256 bytes.
  __device__ __forceinline__ static int swizzle(int k) { return ((k & 3) | (k >> 3 & 1) << 2) << 1; }
  __device__ __forceinline__ void init(const Operand& o, int x0, int t) {
    base = reinterpret_cast<const char*>(o.p + x0);
    plane = o.plane * 2;
    ld2 = unsigned(o.ld * 2);
    step = o.ld * (2 * kStepK);
    rows = o.rows;
    tid = t;
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int c = t + j * THREADS, k = c / CHUNKS, x = ((c % CHUNKS) ^ swizzle(k)) * 8;
      off[j] = unsigned(k) * ld2 + unsigned(min(x, o.cols - 8 - x0) * 2);
    }
  }
  __device__ __forceinline__ void load(char ACDC_LDS* lds, int p, int k, int wave) const {
    const char* at = base + p * plane + k * step;
    if ((k + 1) * kStepK <= rows) {
#pragma unroll
      for (int j = 0; j < N; ++j) Along<X, THREADS, 0>::put(lds, at + off[j], j, wave);
    } else {
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const int row = (tid + j * THREADS) / CHUNKS;
        const int past = row - min(row, rows - 1 - k * kStepK);
        Along<X, THREADS, 0>::put(lds, at + off[j] - int64_t(past) * ld2, j, wave);
      }
    }
  }
  // 8 k of the values x .. x + 15, lane & 15 of them: two reads that transpose 4 x 16 values
  // within 16 lanes (lane i reads 4 values of row i / 4 and gets 4 rows of value i)
  __device__ __forceinline__ static bf16x8 read(const char ACDC_LDS* tile, int x, int half, int lane) {
    const int i = lane & 15, at = x + (i & 3) * 4;
    union {
      bf16x8 v;
      s16x4 h[2];
    } u;
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      const int k = half * 32 + (lane >> 4) * 8 + (i >> 2) + q * 4;
      const char ACDC_LDS* a = tile + k * (X * 2) + ((at >> 3) ^ swizzle(k)) * 16 + (at & 7) * 2;
      u.h[q] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 ACDC_LDS*)a);
    }
    return u.v;
  }
};

// What one workgroup computes: tile (tm, tn) of mt x nt, part `part` of the steps.
// The tiles of one XCD (workgroups go round the eight of them) lie together, in groups
// of 8 n-tiles that run along m, so that its L2 holds what they share.
struct Place {
  int tm, tn, part;
};
__device__ __forceinline__ Place place_of(unsigned id, int mt, int nt) {
  const unsigned tiles = unsigned(mt) * unsigned(nt);
  Place p;
  p.part = int(id / tiles);
  id %= tiles;
  const unsigned per = tiles / 8, rest = tiles % 8, xcd = id % 8;
  id = xcd * per + min(xcd, rest) + id / 8;
  constexpr unsigned GROUP = 8;
  const unsigned g = id / (GROUP * mt), first = g * GROUP, wide = min(GROUP, nt - first);
  const unsigned in = id - g * GROUP * mt;
  p.tn = int(first + in % wide);
  p.tm = int(in / wide);
  return p;
}

// Where a lane's results stand: of MI x NI squares of 16 x 16, acc[mi][ni][i] is
// m = m(mi) + i, n = n(ni).  With A along, the rows of a wave's tile are dealt to the
// squares so that a lane's 4 MI values of m follow one another.
template <int MI, int NI, bool RUN>
struct Spot {
  int m0, n0, lane;
  __device__ __forceinline__ int m(int mi) const {
    return RUN ? m0 + (lane >> 4) * (4 * MI) + mi * 4 : m0 + mi * 16 + (lane >> 4) * 4;
  }
  __device__ __forceinline__ int n(int ni) const { return n0 + ni * 16 + (lane & 15); }
};

// Steps: of the pairs of planes, each over `ksteps` steps of k; `parts` workgroups share
// a tile's.  *count (may be null): rows in use; with COUNT_N the n-tiles past them end at
// once, otherwise (COUNT_K) they bound k.
enum class Count { kNone, kN, kK };

template <int BM, int BN, int WM, int WN, int PLANES, bool ACROSS_A, bool ACROSS_B, Count COUNT, class Epilogue>
__global__ __launch_bounds__(WM* WN * 64) void k_gemm(Operand A, Operand B, int ksteps, int mt, int nt, int parts,
                                                      const int* __restrict__ count, Epilogue epilogue) {
  constexpr int T = WM * WN * 64, MI = BM / WM / 16, NI = BN / WN / 16, HALF = (BM + BN) * 128;
  using StageA = std::conditional_t<ACROSS_A, Across<BM, T>, Along<BM, T, 4 * MI>>;
  using StageB = std::conditional_t<ACROSS_B, Across<BN, T>, Along<BN, T, 0>>;
  __shared__ __attribute__((aligned(1024))) char lds[2 * HALF];  // (the epilogue exchanges values there too)
  const int tid = threadIdx.x, wave = uniform(tid >> 6), lane = tid & 63;
  const Place at = place_of(blockIdx.x, mt, nt);
  if constexpr (COUNT == Count::kN) {
    if (at.tn * BN >= *count) return;
  }
  if constexpr (COUNT == Count::kK) ksteps = (*count + kStepK - 1) / kStepK;
  // this part's steps: from .. to of all pairs
  const int total = Pairs<PLANES>::N * ksteps, per = (total + parts - 1) / parts;
  const int from = min(total, at.part * per), to = min(total, from + per);
  StageA a;
  StageB b;
  a.init(A, at.tm * BM, tid);
  b.init(B, at.tn * BN, tid);
  char ACDC_LDS* const base = (char ACDC_LDS*)lds;
  int pair = PLANES == 1 ? 0 : from / max(ksteps, 1), k = PLANES == 1 ? from : from - pair * ksteps;
  auto fetch = [&](char ACDC_LDS* half) {
    a.load(half, (Pairs<PLANES>::A >> (4 * pair)) & 15, k, wave);
    b.load(half + BM * 128, (Pairs<PLANES>::B >> (4 * pair)) & 15, k, wave);
    if (++k == ksteps && PLANES > 1) {
      k = 0;
      ++pair;
    }
  };
  f32x4 acc[MI][NI] = {};
  const int wm = wave % WM, wn = wave / WM;
  if (from < to) fetch(base);
  for (int s = from; s < to; ++s) {
    const char ACDC_LDS* tile = base + ((s - from) & 1) * HALF;
    // this wave's loads are there, then everyone's; and everyone has read the other half
    __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0)
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
    if (s + 1 < to) fetch(base + ((s + 1 - from) & 1) * HALF);
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      bf16x8 bv[NI];
#pragma unroll
      for (int n = 0; n < NI; ++n) {
        const int x = wn * (BN / WN) + n * 16;
        bv[n] = StageB::read(tile + BM * 128, ACROSS_B ? x : x + (lane & 15), half, lane);
      }
#pragma unroll
      for (int m = 0; m < MI; ++m) {
        const int x = wm * (BM / WM), j = lane & 15;
        const bf16x8 av = StageA::read(tile, ACROSS_A ? x + m * 16 : x + (j >> 2) * (4 * MI) + m * 4 + (j & 3), half, lane);
#pragma unroll
        for (int n = 0; n < NI; ++n) acc[m][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(av, bv[n], acc[m][n], 0, 0, 0);
      }
    }
  }
  const Spot<MI, NI, !ACROSS_A> spot{at.tm * BM + wm * (BM / WM), at.tn * BN + wn * (BN / WN), lane};
  epilogue.template operator()<BM, BN, WM, WN, MI, NI>(acc, spot, at, wave, reinterpret_cast<float2*>(lds));
}

}  // namespace acdc
