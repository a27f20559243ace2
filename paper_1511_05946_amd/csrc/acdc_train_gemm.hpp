// Matrix product on the matrix cores for the vocabulary's losses:
//   C[m][n] = sum_k A(m, k) B(n, k),  bfloat16 operands, 32-bit sums.
//
// An operand lies in memory with k along its rows ("along"), or with k across
// them ("across": row k holds the values of all m), so that the three products
// of the loss read hidden, weight and the logits' gradient as they are, and
// nothing is transposed on the way.
//
// A workgroup computes BM x BN of C; steps of BK k go through STAGES parts of
// LDS.  While the waves compute on one of them, the others are filled by loads
// that write LDS themselves (16 bytes a lane), so that a step needs one barrier
// and no registers in between.  LDS words are permuted by the row
// (Along::swizzle, Across::swizzle): 8 lanes that read 16 bytes each touch all
// banks once, and so do the transposing reads of "across" tiles.
//
// 7373 rows of 4096 over 65536 classes in tiles of 256 x 256, steps of 64, eight waves:
// 1.42 PFLOP/s in the main loop with both operands along, 1.32 as a launch of
// the two products of the gradients.  The loop is bound by its loads into LDS that
// miss L2 (with both operands along, before: 1.21 PFLOP/s, 1.47 where all of them hit,
// 1.61 with no load into LDS, 1.95 with the matrix instructions alone).  Slower:
// steps of 32 in four or five parts of LDS (0.98, 1.11), tiles of 128 x 256 of which a CU has
// two (9.65 ms a call became 11.8), four waves of 128 x 128 each (registers
// run out), squares of 32 x 32 (1.86 for 2.10 alone).
//
// float32 values x = x0 + x1 + x2 are three planes of bfloat16 (8 of 24 bits
// each, exact): a step multiplies the six pairs of planes that matter,
// smallest first; what is left out is below 2^-26 of a product.  Of bfloat16 times
// two planes both pairs are multiplied (1000 rows of 4096 over 65536 classes: the
// gradients' products 1.75 ms, 1.23 PFLOP/s).
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

// rows x cols values in memory, `ld` apart, both >= 1, cols a multiple of 8 and
// rows at multiples of 16 bytes.  A tile may reach past either: it then reads the
// last row or the last 8 columns again, so that every address is inside.
struct Operand {
  const __bf16* p;
  int64_t ld;      // the rows that a tile reads at once span less than 4 GB
  int64_t plane;   // elements from plane to plane
  int rows, cols;
};

// The tile of X values (m or n) by BK k of an operand with k along its rows: BK / 8 chunks
// of 16 bytes a value.
template <int X, int BK, int THREADS, bool DEALT>
struct Along {
  static constexpr int CHUNKS = BK / 8, N = X * CHUNKS / THREADS, BYTES = X * BK * 2;
  const char* base;
  unsigned off[N];
  int64_t plane;
  int cols, tid;
  // The rows that 8 lanes read at once are 0 .. 7 or, dealt as in Spot, 0 .. 3 and 8 .. 11;
  // they are to touch eight different 16-byte columns of 128 bytes.
  __device__ __forceinline__ static int swizzle(int row) {
    const int far = DEALT ? row >> 3 & 1 : row >> 2 & 1;
    return CHUNKS == 8 ? (row & 3) | far << 2 : (row >> 1 & 1) | far << 1;
  }
  __device__ __forceinline__ void init(const Operand& o, int x0, int t) {
    base = reinterpret_cast<const char*>(o.p + int64_t(x0) * o.ld);
    plane = o.plane * 2;
    cols = o.cols;
    tid = t;
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int c = t + j * THREADS, row = c / CHUNKS;
      off[j] = unsigned(min(row, o.rows - 1 - x0)) * unsigned(o.ld * 2) + unsigned(((c % CHUNKS) ^ swizzle(row)) << 4);
    }
  }
  // step k of plane p; FULL: it ends inside the operand
  template <bool FULL>
  __device__ __forceinline__ void load(char ACDC_LDS* lds, int p, int k, int wave) const {
    const char* at = base + p * plane + int64_t(k) * (BK * 2);
    if (FULL || (k + 1) * BK <= cols) {
#pragma unroll
      for (int j = 0; j < N; ++j) put(lds, at, off[j], j, wave);
    } else {
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const int c = tid + j * THREADS, row = c / CHUNKS, col = ((c % CHUNKS) ^ swizzle(row)) * 8;
        put(lds, at + off[j] - (col - min(col, cols - 8 - k * BK)) * 2, j, wave);
      }
    }
  }
  // chunk j of the thread's, from a uniform address and an offset of its own.  (The offset
  // stays 32 bits wide: its extension, if it were taken out of the loop, would need two
  // registers and an addition a load.)
  __device__ __forceinline__ static void put(char ACDC_LDS* lds, const char* from, unsigned off, int j, int wave) {
    asm("" : "+v"(off));
    put(lds, from + off, j, wave);
  }
  __device__ __forceinline__ static void put(char ACDC_LDS* lds, const char* from, int j, int wave) {
    __builtin_amdgcn_global_load_lds((const ACDC_GLOBAL void*)from, (ACDC_LDS void*)(lds + (j * THREADS + wave * 64) * 16),
                                     16, 0, 0);
  }
  // Where a lane's 8 k of a part (32 k) of the first square begin: those of the others are a
  // fixed number of bytes on.
  struct Reader {
    unsigned at[BK / 32];
    __device__ __forceinline__ void init(int x, int lane) {
      const int j = lane & 15, row = DEALT ? x + (j >> 2) * 8 + (j & 3) : x + j;
#pragma unroll
      for (int part = 0; part < BK / 32; ++part) at[part] = row * (BK * 2) + ((part * 4 + (lane >> 4)) ^ swizzle(row)) * 16;
    }
    __device__ __forceinline__ bf16x8 read(const char ACDC_LDS* tile, int square, int part) const {
      return *(const bf16x8 ACDC_LDS*)(tile + at[part] + (DEALT ? square / 2 * 32 + square % 2 * 4 : square * 16) * (BK * 2));
    }
  };
};

// The same of an operand with k across its rows: BK rows of X values.
template <int X, int BK, int THREADS>
struct Across {
  static constexpr int CHUNKS = X / 8, N = BK * CHUNKS / THREADS, BYTES = X * BK * 2;
  // Chunk j of a thread's is j EVERY rows on; 16 rows on the permutation is the same, so
  // that KEPT offsets are enough.
  static constexpr int EVERY = THREADS / CHUNKS, KEPT = EVERY < 16 ? 16 / EVERY : 1;
  static_assert(N % KEPT == 0);
  const char* base;
  unsigned off[KEPT];
  int64_t plane, step;
  unsigned ld2;
  int rows, tid;
  // A transposing read takes 16 values of the rows k .. k + 3 and k + 8 .. k + 11 at once
  // per half wave: eight times 32 bytes, at eight different places of 256 bytes (of which
  // rows of 64 values fill half, so that k's lowest bit already tells two of them apart).
  __device__ __forceinline__ static int swizzle(int k) {
    return CHUNKS == 8 ? ((k >> 1 & 1) | (k >> 3 & 1) << 1) << 1 : ((k & 3) | (k >> 3 & 1) << 2) << 1;
  }
  __device__ __forceinline__ void init(const Operand& o, int x0, int t) {
    base = reinterpret_cast<const char*>(o.p + x0);
    plane = o.plane * 2;
    ld2 = unsigned(o.ld * 2);
    step = o.ld * (2 * BK);
    rows = o.rows;
    tid = t;
#pragma unroll
    for (int j = 0; j < KEPT; ++j) {
      const int k = t / CHUNKS + j * EVERY, x = ((t % CHUNKS) ^ swizzle(k)) * 8;
      off[j] = unsigned(k) * ld2 + unsigned(min(x, o.cols - 8 - x0) * 2);
    }
  }
  // step k of plane p; FULL: it ends inside the operand
  template <bool FULL>
  __device__ __forceinline__ void load(char ACDC_LDS* lds, int p, int k, int wave) const {
    const char* at = base + p * plane + k * step;
    if (FULL || (k + 1) * BK <= rows) {
#pragma unroll
      for (int j = 0; j < N; ++j) Along<X, BK, THREADS, false>::put(lds, at + int64_t(j / KEPT * KEPT * EVERY) * ld2, off[j % KEPT], j, wave);
    } else {
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const int row = tid / CHUNKS + j * EVERY;
        const int past = row - min(row, rows - 1 - k * BK);
        Along<X, BK, THREADS, false>::put(lds, at + off[j % KEPT] + int64_t(j / KEPT * KEPT * EVERY - past) * ld2, j, wave);
      }
    }
  }
  // 8 k of 16 values, lane & 15 of them: two reads that transpose 4 x 16 values within 16
  // lanes (lane i reads 4 values of row i / 4 and gets 4 rows of value i)
  struct Reader {
    unsigned at;
    __device__ __forceinline__ void init(int x, int lane) {
      const int i = lane & 15, k = (lane >> 4) * 8 + (i >> 2), from = x + (i & 3) * 4;
      at = k * (X * 2) + ((from >> 3) ^ swizzle(k)) * 16 + (from & 7) * 2;
    }
    __device__ __forceinline__ bf16x8 read(const char ACDC_LDS* tile, int square, int part) const {
      union {
        bf16x8 v;
        s16x4 h[2];
      } u;
      // 16 values on are 32 bytes, under the permutation (x is a multiple of all squares' values)
      const char ACDC_LDS* from = tile + (at ^ (square * 32));
#pragma unroll
      for (int q = 0; q < 2; ++q)
        u.h[q] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 ACDC_LDS*)(from + (part * 32 + q * 4) * (X * 2)));
      return u.v;
    }
  };
};

// What one workgroup computes: tile (tm, tn) of mt x nt, part `part` of the steps.
// What one XCD computes (workgroups go round the eight of them) lies together: a part, whose
// tiles read the same steps of both operands (2048 rows of G over 32768 classes times a weight
// of 1024, 32 tiles in 8 parts: 250 MB from HBM, for 740 with an eighth of the tiles of every
// part), and of a part groups of 4 n-tiles that run along m: 32 CUs ask for 12 different tiles a
// step (65536 x 7424 x 4096: 1.22 PFLOP/s; groups of 2 1.13, of 8 1.20, of 16 1.13).
struct Place {
  int tm, tn, part;
};
__device__ __forceinline__ Place place_of(unsigned id, int mt, int nt, int parts) {
  const unsigned tiles = unsigned(mt) * unsigned(nt), all = tiles * unsigned(parts);
  const unsigned per = all / 8, rest = all % 8, xcd = id % 8;
  id = xcd * per + min(xcd, rest) + id / 8;
  Place p;
  p.part = int(id / tiles);
  id %= tiles;
  constexpr unsigned GROUP = 4;
  const unsigned g = id / (GROUP * mt), first = g * GROUP, wide = min(GROUP, nt - first);
  const unsigned in = id - g * GROUP * mt;
  p.tn = int(first + in % wide);
  p.tm = int(in / wide);
  return p;
}

// Where a lane's results stand: of MI x NI squares of 16 x 16, acc[mi][ni][i] is
// m = m(mi) + i, n = n(ni).  With A along, the rows of a wave's tile are dealt to pairs of
// squares so that a lane has eight values of m that follow one another, and four lanes 32
// (64 bytes of bfloat16).
template <int MI, int NI, bool DEALT>
struct Spot {
  int m0, n0, lane;
  __device__ __forceinline__ int m(int mi) const {
    return DEALT ? m0 + mi / 2 * 32 + (lane >> 4) * 8 + mi % 2 * 4 : m0 + mi * 16 + (lane >> 4) * 4;
  }
  __device__ __forceinline__ int n(int ni) const { return n0 + ni * 16 + (lane & 15); }
};

// How rows in use bound a product: kN: the n-tiles past *count end at once; kK: they are
// the k.
enum class Count { kN = 1, kK };

// The shape of a workgroup: BM x BN of C by WM x WN waves, steps of BK, of which STAGES
// are in LDS at a time.
template <int BM_, int BN_, int BK_, int WM_, int WN_, int STAGES_, bool AHEAD_ = false>
struct Shape {
  static constexpr int BM = BM_, BN = BN_, BK = BK_, WM = WM_, WN = WN_, STAGES = STAGES_, THREADS = WM * WN * 64;
  static constexpr int MI = BM / WM / 16, NI = BN / WN / 16;
  static constexpr bool AHEAD = AHEAD_;
};

// Waits until at most N of this wave's loads are on their way.
template <int N>
__device__ __forceinline__ void wait_loads() {
  static_assert(N >= 0 && N < 64);
  __builtin_amdgcn_s_waitcnt(0x0f70 | (N & 15) | (N >> 4) << 14);
}

// The parts of LDS, each an object of its own: only so does the compiler see that a transposing
// read of one of them need not wait for the loads on their way into another (7373 rows of 4096
// over 65536 classes 10.34 ms a call with one object, 9.50 so; float32 1000 of 1024 over 20001
// 772 and 698 us).
struct Stages {
  char ACDC_LDS* at[4];
};
// STAGE bytes for each of STAGES of them.
#define ACDC_STAGES(name, STAGE, STAGES)                                                     \
  __shared__ __attribute__((aligned(1024))) char name##_0[STAGE], name##_1[STAGE],           \
      name##_2[STAGES > 2 ? STAGE : 16], name##_3[STAGES > 3 ? STAGE : 16];                  \
  const Stages name{{(char ACDC_LDS*)name##_0, (char ACDC_LDS*)name##_1, (char ACDC_LDS*)name##_2, \
                     (char ACDC_LDS*)name##_3}}

// A product and what follows it: mt x nt tiles, whose steps `parts` workgroups share each.
template <class S, int PA, int PB, bool ACROSS_A, bool ACROSS_B, Count COUNT, class Epilogue>
struct Product {
  using Shape = S;
  static constexpr int T = S::THREADS, BM = S::BM, BN = S::BN, BK = S::BK, MI = S::MI, NI = S::NI, STAGES = S::STAGES;
  using StageA = std::conditional_t<ACROSS_A, Across<BM, BK, T>, Along<BM, BK, T, true>>;
  using StageB = std::conditional_t<ACROSS_B, Across<BN, BK, T>, Along<BN, BK, T, false>>;
  static constexpr int STAGE = PA * StageA::BYTES + PB * StageB::BYTES, LOADS = PA * StageA::N + PB * StageB::N;
  static_assert(STAGES * STAGE <= 160 * 1024);
  Operand A, B;
  int depth, mt, nt, parts;
  Epilogue epilogue;
  unsigned groups() const { return unsigned(int64_t(mt) * nt * parts); }
  __device__ __forceinline__ void run(unsigned id, const Stages& lds, const int* __restrict__ count) const;
};

// Workgroup `id` of the product's.  *count: the rows in use.
template <class S, int PA, int PB, bool ACROSS_A, bool ACROSS_B, Count COUNT, class Epilogue>
__device__ __forceinline__ void Product<S, PA, PB, ACROSS_A, ACROSS_B, COUNT, Epilogue>::run(unsigned id, const Stages& lds,
                                                                                             const int* __restrict__ count) const {
  constexpr int MOST = PA > PB ? PA : PB;
  const int tid = threadIdx.x, wave = uniform(tid >> 6), lane = tid & 63;
  const Place at = place_of(id, mt, nt, parts);
  int depth = this->depth;
  if constexpr (COUNT == Count::kN) {
    if (at.tn * BN >= *count) return;
  }
  if constexpr (COUNT == Count::kK) depth = *count;
  // this part's steps: from .. to
  const int total = (depth + BK - 1) / BK, per = (total + parts - 1) / parts;
  const int from = min(total, at.part * per), to = min(total, from + per);
  StageA a;
  StageB b;
  a.init(A, at.tm * BM, tid);
  b.init(B, at.tn * BN, tid);
  auto fetch = [&]<bool FULL>(int slot, int k) {
    char ACDC_LDS* stage = lds.at[slot];
#pragma unroll
    for (int p = 0; p < PA; ++p) a.template load<FULL>(stage + p * StageA::BYTES, p, k, wave);
#pragma unroll
    for (int p = 0; p < PB; ++p) b.template load<FULL>(stage + PA * StageA::BYTES + p * StageB::BYTES, p, k, wave);
  };
  f32x4 acc[MI][NI] = {};
  const int wm = wave % S::WM, wn = wave / S::WM;
  typename StageA::Reader ra;
  typename StageB::Reader rb;
  ra.init(wm * (BM / S::WM), lane);
  rb.init(wn * (BN / S::WN), lane);
  // one part (32 k) of a step as the matrix cores take it
  struct Part {
    bf16x8 a[PA][MI], b[PB][NI];
  };
  auto read = [&](int slot, int part, Part& f) {
    const char ACDC_LDS* stage = lds.at[slot];
#pragma unroll
    for (int p = 0; p < PB; ++p)
#pragma unroll
      for (int n = 0; n < NI; ++n) f.b[p][n] = rb.read(stage + PA * StageA::BYTES + p * StageB::BYTES, n, part);
#pragma unroll
    for (int p = 0; p < PA; ++p)
#pragma unroll
      for (int m = 0; m < MI; ++m) f.a[p][m] = ra.read(stage + p * StageA::BYTES, m, part);
  };
  auto multiply = [&](const Part& f) {
#pragma unroll
    for (int m = 0; m < MI; ++m)
      // the pairs of planes that matter, smallest first
#pragma unroll
      for (int both = MOST - 1; both >= 0; --both)
#pragma unroll
        for (int p = 0; p <= both && p < PA; ++p)
#pragma unroll
          for (int n = 0; n < NI && both - p < PB; ++n)
            acc[m][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f.a[p][m], f.b[both - p][n], acc[m][n], 0, 0, 0);
  };
  // this wave's loads but `left` of them are there, then everyone's; and everyone has read
  // what it asked of LDS
  auto meet = [&] {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
  };
  // step s has arrived
  auto arrive = [&](int s) {
    if (STAGES > 2 && s + STAGES - 2 < to) wait_loads<LOADS * (STAGES - 2)>();
    else wait_loads<0>();
    meet();
  };
  constexpr int READS = PA * (ACROSS_A ? 2 : 1) * MI + PB * (ACROSS_B ? 2 : 1) * NI;
  constexpr int PAIRS = PA == PB ? PA * (PA + 1) / 2 : MOST;  // of planes
  static_assert(PA == PB || PA == 1);
#pragma unroll
  for (int q = 0; q < STAGES - 1; ++q)
    if (from + q < to) fetch.template operator()<false>(q, from + q);
  // (step s is in part (s - from) % STAGES of LDS, a constant wherever one is used)
  if constexpr (S::AHEAD && BK == 32) {
    // The registers of one step are read while the matrix cores work on the other's.
    static_assert(STAGES == 2);
    constexpr int PER = PAIRS * MI * NI / READS;
    Part even, odd;
    int s = from;
    if (from < to) {
      if (from + 1 < to) {
        fetch.template operator()<false>(1, from + 1);
        wait_loads<LOADS>();
      } else {
        wait_loads<0>();
      }
      meet();
      read(0, 0, even);
    }
    // step s is in `now`, and step s + 2 takes its place in LDS
    auto step = [&]<bool FULL, int SLOT>(const Part& now, Part& then) {
      wait_loads<0>();
      meet();
      read(SLOT ^ 1, 0, then);  // (nothing, after the last step)
      if constexpr (FULL) {
        fetch.template operator()<true>(SLOT, s + 2);
      } else {
        if (s + 2 < to) fetch.template operator()<false>(SLOT, s + 2);
      }
      multiply(now);
      if constexpr (FULL) {
#pragma unroll
        for (int i = 0; i < READS; ++i) {
          __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
          if (i < LOADS) __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);
          __builtin_amdgcn_sched_group_barrier(0x008, PER, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      ++s;
    };
    // (the last step of all may end outside the operand)
    while (s + 4 < to) {
      step.template operator()<true, 0>(even, odd);
      step.template operator()<true, 1>(odd, even);
    }
#pragma nounroll
    while (s < to) {
      step.template operator()<false, 0>(even, odd);
      if (s < to) step.template operator()<false, 1>(odd, even);
    }
  } else if constexpr (S::AHEAD) {
    // The registers of one part are read while the matrix cores work on the other's.
    static_assert(BK == 64 && STAGES == 2 && MOST == 1);
    constexpr int PER = MI * NI / READS;
    Part first, second;
    int s = from;
    if (from < to) {
      arrive(from);
      read(0, 0, first);
      if (from + 1 < to) fetch.template operator()<false>(1, from + 1);
    }
    // (the last step of all may end outside the operand)
    auto step = [&]<int SLOT>() {
      read(SLOT, 1, second);
      multiply(first);
#pragma unroll
      for (int i = 0; i < READS; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x008, PER, 0);
      }
      __builtin_amdgcn_sched_barrier(0);
      wait_loads<0>();
      meet();
      read(SLOT ^ 1, 0, first);
      fetch.template operator()<true>(SLOT, s + 2);
      multiply(second);
#pragma unroll
      for (int i = 0; i < READS; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        if (i < LOADS) __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x008, PER, 0);
      }
      __builtin_amdgcn_sched_barrier(0);
      ++s;
    };
    auto last = [&]<int SLOT>() {
      read(SLOT, 1, second);
      multiply(first);
      wait_loads<0>();
      meet();
      read(SLOT ^ 1, 0, first);  // (nothing, after the last step)
      if (s + 2 < to) fetch.template operator()<false>(SLOT, s + 2);
      multiply(second);
      ++s;
    };
    while (s + 4 < to) {
      step.template operator()<0>();
      step.template operator()<1>();
    }
#pragma nounroll
    while (s < to) {
      last.template operator()<0>();
      if (s < to) last.template operator()<1>();
    }
  } else {
    for (int s = from; s < to; s += STAGES) {
#pragma unroll
      for (int q = 0; q < STAGES; ++q) {
        if (s + q >= to) break;
        arrive(s + q);
        if (s + q + STAGES - 1 < to) fetch.template operator()<false>((q + STAGES - 1) % STAGES, s + q + STAGES - 1);
#pragma unroll
        for (int part = 0; part < BK / 32; ++part) {
          Part f;
          read(q, part, f);
          multiply(f);
        }
      }
    }
  }
  const Spot<MI, NI, !ACROSS_A> spot{at.tm * BM + wm * (BM / S::WM), at.tn * BN + wn * (BN / S::WN), lane};
  epilogue.template operator()<S>(acc, spot, at, wave, (float2*)(char*)lds.at[0]);
}

// (the epilogue exchanges values in the LDS of the tiles)
template <class P>
__global__ __launch_bounds__(P::T) void k_gemm(P product, const int* __restrict__ count) {
  ACDC_STAGES(lds, P::STAGE, P::STAGES);
  product.run(blockIdx.x, lds, count);
}

// Two products in one launch, the second from workgroup `first` on (a multiple of 8: the
// XCDs): its tiles fill the CUs that the first one's last round leaves idle, and small
// products cost one launch (64 rows of 256 over 1000 classes: 32.1 us a call in two, 28.8 so;
// 1000 of 1024 over 20001: 786 and 772).
template <class P, class Q>
__global__ __launch_bounds__(P::T) void k_gemm_both(P p, Q q, unsigned first, const int* __restrict__ count) {
  static_assert(P::T == Q::T && P::STAGE == Q::STAGE && P::STAGES == Q::STAGES);
  ACDC_STAGES(lds, P::STAGE, P::STAGES);
  if (blockIdx.x >= first) q.run(blockIdx.x - first, lds, count);
  else if (blockIdx.x < unsigned(p.mt * p.nt * p.parts)) p.run(blockIdx.x, lds, count);
}

}  // namespace acdc
