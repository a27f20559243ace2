// Rows of a weight looked up by tokens, and the weight's gradient
// (acdc_train_lm.h).
//
// The gradient of a class is the sum of the gradients of its rows.  The rows
// are sorted by token (a stable radix sort), so that those of a class follow
// one another, in their order; then pieces of 16 to 64 sorted rows are summed
// class by class.  A class that begins and ends within a piece is written at
// once; of one that goes on, each piece leaves a partial sum, and a second
// launch adds those up in order.  No sum depends on the order in which
// anything runs.  Bound by HBM: each gradient row is read once, each row of
// the weight's gradient written once (8192 rows of 4096 over 65536 classes in
// bfloat16: zeros over 537 MB while one workgroup sorts, 98 us, 5.5 TB/s; sums
// 32 us, 4.8; 131072 of 257 over 1000: sort 15 us in three launches, sums 33,
// 4.4 TB/s, the longest classes' partial sums 14).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "acdc_train_lm.hpp"
#include "acdc_train_rows.hpp"

namespace acdc {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kSpan = 64 * kEight;  // columns that a wave takes at a time

// `classes` for a row that takes no part: sorted behind all others.
__device__ __forceinline__ int key_of(const void* tokens, int bits, long long r, int classes) {
  const long long t = bits == 64 ? static_cast<const long long*>(tokens)[r] : (long long)static_cast<const int*>(tokens)[r];
  return t < 0 || t >= classes ? classes : int(t);
}

// ----------------------------------------------------------------- the lookup

// A wave takes one of `split` parts of ROWS rows, whose tokens and values it asks for
// together.  Bound by the rows written: 131072 of 257 float32 values 4.9 TB/s.
template <class TW, class TO, int ROWS>
__global__ __launch_bounds__(kThreads) void k_embed(const void* __restrict__ tokens, int bits,
                                                    const typename TW::Elem* __restrict__ weight, long long weight_stride,
                                                    float scale, typename TO::Elem* __restrict__ out, long long out_stride,
                                                    int rows, int width, int classes, int split) {
  const int lane = threadIdx.x % 64;
  const unsigned items = (unsigned(rows) + ROWS - 1) / ROWS * unsigned(split);
  for (unsigned item = blockIdx.x * kWaves + uniform(int(threadIdx.x / 64)); item < items; item += gridDim.x * kWaves) {
    const int first = int(item / unsigned(split)) * ROWS, part = int(item % unsigned(split)), many = min(ROWS, rows - first);
    const typename TW::Elem* from[ROWS];
    bool there[ROWS];
    float fill[ROWS];
#pragma unroll
    for (int q = 0; q < ROWS; ++q) {
      const long long r = first + (q < many ? q : 0);
      const long long t = bits == 64 ? static_cast<const long long*>(tokens)[r] : (long long)static_cast<const int*>(tokens)[r];
      there[q] = t >= 0 && t < classes;
      from[q] = weight + (there[q] ? t : 0) * weight_stride;
      fill[q] = t < 0 ? 0.f : __builtin_nanf("");
    }
#pragma unroll 2
    for (int col = part * kSpan; col < width; col += split * kSpan) {
      const Columns<kApart<TW, TO>> at(col, lane, width);
      float v[ROWS][kEight];
#pragma unroll
      for (int q = 0; q < ROWS; ++q)
        if (q < many) at.template load<TW>(from[q], v[q]);
#pragma unroll
      for (int q = 0; q < ROWS; ++q) {
        if (q >= many) continue;
#pragma unroll
        for (int i = 0; i < kEight; ++i) v[q][i] = there[q] ? v[q][i] * scale : fill[q];
        at.template store<TO>(out + (long long)(first + q) * out_stride, v[q]);
      }
    }
  }
}

// ------------------------------------------------------------------- the sort

// Stable, least digit first, in passes of up to ten bits: 1000 classes take one, 2^20 two.
struct Sorted {
  int* key;
  int* row;
};
constexpr int kMostBits = 10, kDigits = 1 << kMostBits;

// next[wave][digit] goes from how many pairs of the digit a wave has to how many the waves
// before it have; returns how many all have.
template <int WAVES>
__device__ __forceinline__ int digit_total(int (&next)[WAVES][kDigits], int digit) {
  int all = 0;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) {
    const int c = next[w][digit];
    next[w][digit] = all;
    all += c;
  }
  return all;
}
// The exclusive sums of kDigits totals, EACH digits that follow one another for each of the
// first threads; the whole workgroup calls it.
template <int EACH>
__device__ __forceinline__ void digit_bases(const int (&total)[EACH], int (&base)[EACH], int* slots) {
  const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
  int mine = 0;
#pragma unroll
  for (int q = 0; q < EACH; ++q) mine += total[q];
  int sum = mine;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int up = __shfl_up(sum, o);
    if (lane >= o) sum += up;
  }
  constexpr int WAVES = kDigits / EACH / 64;
  if (wave < WAVES && lane == 63) slots[wave] = sum;
  __syncthreads();
  int at = sum - mine;
#pragma unroll
  for (int w = 0; w < WAVES; ++w)
    if (w < wave) at += slots[w];
#pragma unroll
  for (int q = 0; q < EACH; ++q) {
    base[q] = at;
    at += total[q];
  }
}
// The place of a pair among its wave's of the same digit; a wave's pairs come in rounds of 64.
__device__ __forceinline__ int place_of(int* next, bool here, int digit, int bits) {
  const int lane = threadIdx.x % 64;
  unsigned long long same = __ballot(here);  // the lanes of this round with the same digit
  for (int b = 0; b < bits; ++b) {
    const unsigned long long set = __ballot(here && (digit >> b & 1));
    same &= (digit >> b & 1) ? set : ~set;
  }
  const int rank = __popcll(same & ((1ull << lane) - 1)), many = __popcll(same);
  int to = 0;
  if (here) to = next[digit] + rank;
  wave_sync();  // everyone has read before the last of a digit writes
  if (here && rank == many - 1) next[digit] = to + 1;
  wave_sync();
  return to;
}

// Zeros over the rows v, v + step, ... of the gradient, by a wave.
template <class TW>
__device__ __forceinline__ void fill_zeros(typename TW::Elem* weight, long long stride, int width, int classes, long long v, int step) {
  const float zero[kEight] = {};
  for (; v < classes; v += step)
    for (int col = 0; col < width; col += kSpan)
      Columns<kApart<TW, TW>>(col, threadIdx.x % 64, width).template store<TW>(weight + v * stride, zero);
}

// Up to 8192 rows by the first workgroup, in LDS, while the others (if there are any) write
// zeros over the gradient.
constexpr int kSmallThreads = 1024, kSmallEach = 8, kSmall = kSmallThreads * kSmallEach;
template <class TW>
__global__ __launch_bounds__(kSmallThreads) void k_sort_small(const void* __restrict__ tokens, int bits, int classes, Sorted out,
                                                             int n, int digit_bits, int passes,
                                                             typename TW::Elem* __restrict__ weight, long long weight_stride, int width) {
  constexpr int WAVES = kSmallThreads / 64;
  __shared__ int next[WAVES][kDigits];
  __shared__ int keys[kSmall], rows[kSmall], slots[WAVES];
  const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64, base = wave * (64 * kSmallEach);
  if (blockIdx.x > 0) {
    fill_zeros<TW>(weight, weight_stride, width, classes, (blockIdx.x - 1) * WAVES + wave, (gridDim.x - 1) * WAVES);
    return;
  }
  int key[kSmallEach], row[kSmallEach];
#pragma unroll
  for (int q = 0; q < kSmallEach; ++q) {
    const int i = base + q * 64 + lane;
    key[q] = i < n ? key_of(tokens, bits, i, classes) : 0;
    row[q] = i;
  }
  const int mask = (1 << digit_bits) - 1;
  for (int pass = 0; pass < passes; ++pass) {
    const int shift = pass * digit_bits;
    for (int i = tid; i < WAVES * kDigits; i += kSmallThreads) next[i / kDigits][i % kDigits] = 0;
    __syncthreads();
#pragma unroll
    for (int q = 0; q < kSmallEach; ++q)
      if (base + q * 64 + lane < n) atomicAdd(&next[wave][(key[q] >> shift) & mask], 1);  // (whole numbers: any order gives the same)
    __syncthreads();
    int total[1] = {0}, first[1];
    if (tid < kDigits) total[0] = digit_total<WAVES>(next, tid);
    digit_bases<1>(total, first, slots);
    if (tid < kDigits) {
#pragma unroll
      for (int w = 0; w < WAVES; ++w) next[w][tid] += first[0];
    }
    __syncthreads();
#pragma unroll
    for (int q = 0; q < kSmallEach; ++q) {
      if (base + q * 64 >= n) break;
      const bool here = base + q * 64 + lane < n;
      const int to = place_of(next[wave], here, (key[q] >> shift) & mask, digit_bits);
      if (here) {
        keys[to] = key[q];
        rows[to] = row[q];
      }
    }
    __syncthreads();
#pragma unroll
    for (int q = 0; q < kSmallEach; ++q) {
      const int i = base + q * 64 + lane;
      key[q] = keys[i];  // (behind the last: anything, not used)
      row[q] = rows[i];
    }
    __syncthreads();
  }
#pragma unroll
  for (int q = 0; q < kSmallEach; ++q) {
    const int i = base + q * 64 + lane;
    if (i < n) {
      out.key[i] = key[q];
      out.row[i] = row[q];
    }
  }
}

// More rows, in tiles: counts[tile][digit], their sums over the tiles before, and each pair
// to its place, a pass in three launches.
constexpr int kPerThread = kDigits / kThreads;

// The tokens that are there are marked in `there` or, where that is null, the workgroups past
// the tiles (if there are any) write zeros over the gradient.
template <class TW, int EACH>
__global__ __launch_bounds__(kThreads) void k_sort_count(const void* __restrict__ tokens, int bits, int classes, Sorted in, int n,
                                                         int shift, int mask, int* __restrict__ counts,
                                                         unsigned char* __restrict__ there, int tiles,
                                                         typename TW::Elem* __restrict__ weight, long long weight_stride, int width) {
  __shared__ int bins[kDigits];
  if (int(blockIdx.x) >= tiles) {
    fill_zeros<TW>(weight, weight_stride, width, classes, (blockIdx.x - tiles) * kWaves + threadIdx.x / 64, (gridDim.x - tiles) * kWaves);
    return;
  }
#pragma unroll
  for (int d = 0; d < kPerThread; ++d) bins[d * kThreads + threadIdx.x] = 0;
  __syncthreads();
#pragma unroll
  for (int q = 0; q < EACH; ++q) {
    const int i = (blockIdx.x * EACH + q) * kThreads + threadIdx.x;
    if (i < n) {
      // in the first pass the keys come from the tokens, and are marked as there
      const int k = tokens != nullptr ? key_of(tokens, bits, i, classes) : in.key[i];
      if (there != nullptr && k < classes) there[k] = 1;
      atomicAdd(&bins[(k >> shift) & mask], 1);
    }
  }
  __syncthreads();
#pragma unroll
  for (int d = 0; d < kPerThread; ++d)
    counts[(long long)blockIdx.x * kDigits + d * kThreads + threadIdx.x] = bins[d * kThreads + threadIdx.x];
}

// 64 digits a workgroup, 16 waves along the tiles: counts become what the tiles before
// hold, totals[digit] what all do.
constexpr int kSumWaves = 16;
__global__ __launch_bounds__(64 * kSumWaves) void k_sort_sums(int* __restrict__ counts, int tiles, int* __restrict__ totals) {
  __shared__ int slots[kSumWaves][64];
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, digit = blockIdx.x * 64 + lane;
  const int per = (tiles + kSumWaves - 1) / kSumWaves, from = min(tiles, wave * per), to = min(tiles, from + per);
  int sum = 0;
#pragma unroll 8
  for (int t = from; t < to; ++t) sum += counts[(long long)t * kDigits + digit];
  slots[wave][lane] = sum;
  __syncthreads();
  int before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kSumWaves; ++w) {
    if (w < wave) before += slots[w][lane];
    all += slots[w][lane];
  }
  if (wave == 0) totals[digit] = all;
#pragma unroll 8
  for (int t = from; t < to; ++t) {
    const int c = counts[(long long)t * kDigits + digit];
    counts[(long long)t * kDigits + digit] = before;
    before += c;
  }
}

// A pair comes after those of lower digits, of earlier tiles, of earlier waves, of earlier
// rounds and of lower lanes with the same digit.
template <int EACH>
__global__ __launch_bounds__(kThreads) void k_sort_move(const void* __restrict__ tokens, int bits, int classes, Sorted in,
                                                        Sorted out, int n, int shift, int digit_bits,
                                                        const int* __restrict__ counts, const int* __restrict__ totals) {
  __shared__ int next[kWaves][kDigits], slots[kWaves];
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, mask = (1 << digit_bits) - 1;
  const int base = (blockIdx.x * kThreads + wave * 64) * EACH;
  for (int i = threadIdx.x; i < kWaves * kDigits; i += kThreads) next[i / kDigits][i % kDigits] = 0;
  __syncthreads();
  int key[EACH], row[EACH];
#pragma unroll
  for (int q = 0; q < EACH; ++q) {
    const int i = base + q * 64 + lane;
    key[q] = row[q] = 0;
    if (i < n) {
      key[q] = tokens != nullptr ? key_of(tokens, bits, i, classes) : in.key[i];
      row[q] = tokens != nullptr ? i : in.row[i];
      atomicAdd(&next[wave][(key[q] >> shift) & mask], 1);
    }
  }
  int total[kPerThread], first[kPerThread];
#pragma unroll
  for (int d = 0; d < kPerThread; ++d) total[d] = totals[threadIdx.x * kPerThread + d];
  __syncthreads();
  digit_bases<kPerThread>(total, first, slots);
#pragma unroll
  for (int d = 0; d < kPerThread; ++d) {
    const int digit = threadIdx.x * kPerThread + d;
    digit_total<kWaves>(next, digit);
    const int at = first[d] + counts[(long long)blockIdx.x * kDigits + digit];
#pragma unroll
    for (int w = 0; w < kWaves; ++w) next[w][digit] += at;
  }
  __syncthreads();
#pragma unroll
  for (int q = 0; q < EACH; ++q) {
    const bool here = base + q * 64 + lane < n;
    const int to = place_of(next[wave], here, (key[q] >> shift) & mask, digit_bits);
    if (here) {
      out.key[to] = key[q];
      out.row[to] = row[q];
    }
  }
}

// --------------------------------------------------------------- the gradient

constexpr int kPiece = 64, kShort = 16;  // sorted rows that are summed together, at the most and at the least

struct SumArgs {
  const int* key;
  const int* row;
  int rows, classes, width, piece, pieces, blocks;
  float scale;
  long long grad_stride, weight_stride;
  float* partial;  // [pieces][2][width]: the sum that the piece begins with, and the one it ends with
  bool add;
};

template <class TW, class C>
__device__ __forceinline__ void put_class(typename TW::Elem* row, const C& at, const float (&v)[kEight], float scale, bool add) {
  float o[kEight] = {};
  if (add) at.template load<TW>(row, o);
#pragma unroll
  for (int i = 0; i < kEight; ++i) o[i] += scale * v[i];
  at.template store<TW>(row, o);
}

// A wave sums a piece of the sorted rows in 512 columns.
template <class TG, class TW>
__global__ __launch_bounds__(kThreads) void k_embed_sums(SumArgs a, const typename TG::Elem* __restrict__ grad,
                                                         typename TW::Elem* __restrict__ weight) {
  const int lane = threadIdx.x % 64;
  const long long item = (long long)blockIdx.x * kWaves + uniform(int(threadIdx.x / 64));
  if (item >= (long long)a.pieces * a.blocks) return;
  const int piece = int(item / a.blocks);
  const Columns<kApart<TG, TW>> at(int(item % a.blocks) * kSpan, lane, a.width);
  const int from = piece * a.piece, to = min(a.rows, from + a.piece);
  // one sorted row a lane; the loop passes them on
  const int mine = from + lane < to ? a.key[from + lane] : a.classes;
  const int mine_row = from + lane < to ? a.row[from + lane] : 0;
  const int before = from > 0 ? a.key[from - 1] : -1, after = to < a.rows ? a.key[to] : -1;
  float s[kEight] = {};
  int current = uniform(mine);
  bool began = current != before;  // the class begins in this piece
  constexpr int AHEAD = 8;
  for (int i = 0; i < to - from; i += AHEAD) {
    float v[AHEAD][kEight];
    int key[AHEAD];
#pragma unroll
    for (int q = 0; q < AHEAD; ++q) {
      const int k = min(i + q, to - from - 1);
      key[q] = __builtin_amdgcn_readlane(mine, k);
      const long long r = __builtin_amdgcn_readlane(mine_row, k);
      if (key[q] < a.classes && at.any()) at.template load<TG>(grad + r * a.grad_stride, v[q]);
    }
#pragma unroll
    for (int q = 0; q < AHEAD; ++q) {
      if (i + q >= to - from) break;
      if (key[q] != current) {  // the class before ends here
        if (at.any()) {
          if (began) put_class<TW>(weight + current * a.weight_stride, at, s, a.scale, a.add);
          else at.template store<F32, false>(a.partial + (long long)piece * 2 * a.width, s);
        }
#pragma unroll
        for (int c = 0; c < kEight; ++c) s[c] = 0.f;
        current = key[q];
        began = true;
      }
      if (current >= a.classes) return;  // nothing but rows that take no part from here on
#pragma unroll
      for (int c = 0; c < kEight; ++c) s[c] += v[q][c];
    }
  }
  if (current >= a.classes || !at.any()) return;
  if (current == after || !began) at.template store<F32, false>(a.partial + ((long long)piece * 2 + (began ? 1 : 0)) * a.width, s);
  else put_class<TW>(weight + current * a.weight_stride, at, s, a.scale, a.add);
}

// The class that begins in a piece and goes on behind it: its partial sums together.  A
// wave does that for its piece; more than kAlone of them are shared by the waves of the
// workgroup, which each take some that follow one another.
constexpr int kJoinWaves = 8, kAlone = 8;
template <class TW>
__global__ __launch_bounds__(64 * kJoinWaves) void k_embed_join(SumArgs a, typename TW::Elem* __restrict__ weight) {
  __shared__ float slots[kJoinWaves][kEight][64];
  __shared__ int shared[kJoinWaves];  // pieces that a wave's class goes on for, where that is shared
  const int lane = threadIdx.x % 64, wave = uniform(int(threadIdx.x / 64));
  const int first_piece = int(blockIdx.x / unsigned(a.blocks)) * kJoinWaves;
  const Columns<true> at(int(blockIdx.x % unsigned(a.blocks)) * kSpan, lane, a.width);
  // the class that begins in a piece and the pieces behind it that begin with it: 0, none
  auto goes_on = [&](int piece) {
    const long long from = (long long)piece * a.piece, to = from + a.piece;
    if (to >= a.rows) return 0;
    const int key = a.key[to];
    if (key >= a.classes || a.key[to - 1] != key) return 0;                  // nothing goes on
    if (a.key[from] == key && from > 0 && a.key[from - 1] == key) return 0;  // it began before
    // (those that do follow one another: of 64 at `step` from each other the first ones)
    auto count = [&](int first, int step) {
      const long long p = (long long)piece + first + (long long)(lane + 1) * step;
      const unsigned long long same = __ballot(p < a.pieces && a.key[min(p, (long long)a.pieces - 1) * a.piece] == key);
      return ~same == 0ull ? 64 : __ffsll((long long)~same) - 1;
    };
    int many = count(0, 1);
    if (many < 64) return many;
    for (int more = 64; more == 64; many += more * 64) more = count(many, 64);
    return many + count(many, 1);
  };
  // partial sums first .. last - 1 of those behind `piece` on top of s
  auto add = [&](int piece, int first, int last, float (&s)[kEight]) {
    constexpr int AHEAD = 8;
    for (int p = first; p < last; p += AHEAD) {
      float v[AHEAD][kEight];
#pragma unroll
      for (int q = 0; q < AHEAD; ++q) at.template load<F32>(a.partial + (long long)(piece + 1 + min(p + q, last - 1)) * 2 * a.width, v[q]);
#pragma unroll
      for (int q = 0; q < AHEAD; ++q)
#pragma unroll
        for (int c = 0; c < kEight; ++c) s[c] += p + q < last ? v[q][c] : 0.f;
    }
  };
  auto begin = [&](int piece, float (&s)[kEight]) { at.template load<F32>(a.partial + ((long long)piece * 2 + 1) * a.width, s); };
  auto put = [&](int piece, const float (&s)[kEight]) {
    put_class<TW>(weight + a.key[(long long)(piece + 1) * a.piece] * a.weight_stride, at, s, a.scale, a.add);
  };
  const int mine = first_piece + wave, many = goes_on(mine);
  if (lane == 0) shared[wave] = many > kAlone ? many : 0;
  if (many > 0 && many <= kAlone && at.any()) {
    float s[kEight];
    begin(mine, s);
    add(mine, 0, many, s);
    put(mine, s);
  }
  __syncthreads();
  for (int w = 0; w < kJoinWaves; ++w) {
    const int all = shared[w], piece = first_piece + w;
    if (all == 0) continue;
    float s[kEight] = {};
    const int per = (all + kJoinWaves - 1) / kJoinWaves, first = min(all, wave * per);
    if (at.any()) {
      if (wave == 0) begin(piece, s);
      add(piece, first, min(all, first + per), s);
    }
    __syncthreads();  // the slots of the class before have been read
#pragma unroll
    for (int c = 0; c < kEight; ++c) slots[wave][c][lane] = s[c];
    __syncthreads();
    if (wave != 0 || !at.any()) continue;
#pragma unroll
    for (int k = 1; k < kJoinWaves; ++k)
#pragma unroll
      for (int c = 0; c < kEight; ++c) s[c] += slots[k][c][lane];
    put(piece, s);
  }
}

__global__ __launch_bounds__(kThreads) void k_embed_clear(unsigned char* there, int classes) {
  for (int i = blockIdx.x * kThreads + threadIdx.x; i < classes; i += gridDim.x * kThreads) there[i] = 0;
}

// Zeros for the classes without a row.
template <class TW>
__global__ __launch_bounds__(kThreads) void k_embed_zeros(const unsigned char* __restrict__ there, int classes, int width,
                                                          typename TW::Elem* __restrict__ weight, long long weight_stride) {
  const int lane = threadIdx.x % 64;
  const float zero[kEight] = {};
  for (int v = blockIdx.x * kWaves + threadIdx.x / 64; v < classes; v += gridDim.x * kWaves) {
    if (there[v] != 0) continue;
    for (int col = 0; col < width; col += kSpan) Columns<kApart<TW, TW>>(col, lane, width).template store<TW>(weight + v * weight_stride, zero);
  }
}

// ------------------------------------------------------------------ on the host

constexpr int64_t kMostRows = (1 << 28) - kPiece, kMostClasses = 1 << 30, kMostWidth = 1 << 20, kMostStride = int64_t(1) << 40;

int done() {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? ACDC_OK : hip_fail(e);
}
size_t up256(size_t n) { return (n + 255) & ~size_t(255); }
int blocks_of(int32_t width) { return int((int64_t(width) + kSpan - 1) / kSpan); }
// Shorter pieces where long ones would leave most of the card idle (131072 rows of 257: in
// pieces of 32 88 us lookup and gradient, of 64 95, of 16 100).
int piece_of(int64_t rows, int32_t width) {
  int piece = kPiece;
  while (piece > kShort && rows / piece * blocks_of(width) < 4096) piece /= 2;
  return piece;
}
// Pairs of a thread in a tile of the sort: fewer where that gives more CUs a tile (131072
// rows of 256: 42 us a gradient for 50; 2^20 of 64: 200 for 194).
int each_of(int64_t rows) { return rows >= 256 * kThreads * 8 ? 8 : 2; }
struct Layout {
  size_t key[2], row[2], counts, totals, there, partial, bytes;
};
Layout layout(int64_t rows, int32_t width, int32_t classes) {
  Layout w{};
  size_t next = 0;
  auto take = [&](size_t bytes) {
    const size_t o = next;
    next += up256(bytes);
    return o;
  };
  const size_t n = size_t(rows);
  for (int k = 0; k < 2; ++k) {
    w.key[k] = take(n * 4);
    w.row[k] = take(n * 4);
  }
  const size_t tile = size_t(kThreads) * each_of(rows);
  w.counts = take((n + tile - 1) / tile * kDigits * 4);
  w.totals = take(kDigits * 4);
  w.there = take(size_t(classes));
  w.partial = take((n + piece_of(rows, width) - 1) / piece_of(rows, width) * 2 * size_t(width) * 4);
  w.bytes = next;
  return w;
}
bool sizes_ok(int64_t rows, int32_t width, int32_t classes) {
  // (a grid has fewer than 2^32 lanes)
  if (rows >= 0 && rows <= kMostRows && width >= 1 && (rows / kPiece + 1) * (int64_t(width) / kSpan + 1) > (1 << 22)) return false;
  return rows >= 0 && rows <= kMostRows && width >= 1 && width <= kMostWidth && classes >= 1 && classes <= kMostClasses;
}
bool matrix_ok(const void* p, int32_t dtype, int64_t stride, int64_t rows, int32_t width) {
  const size_t e = dtype_bytes(dtype);
  return e != 0 && stride >= width && stride <= kMostStride && aligned_to(p, e) && (rows == 0 || p != nullptr);
}
bool tokens_ok(const void* tokens, int32_t bits, int64_t rows) {
  return (bits == 32 || bits == 64) && aligned_to(tokens, size_t(bits) / 8) && (rows == 0 || tokens != nullptr);
}
template <class F>
void with_types(int32_t a, int32_t b, F&& f) {
  if (a == ACDC_F32) {
    if (b == ACDC_F32) f.template operator()<F32, F32>();
    else f.template operator()<F32, BF16>();
  } else {
    if (b == ACDC_F32) f.template operator()<BF16, F32>();
    else f.template operator()<BF16, BF16>();
  }
}

}  // namespace
}  // namespace acdc

using namespace acdc;

extern "C" int acdc_embedding_forward(const void* tokens, int32_t token_bits, const void* weight, int32_t weight_type,
                                      int64_t weight_stride, float scale, void* out, int32_t out_type, int64_t out_stride,
                                      int64_t rows, int32_t width, int32_t classes, acdc_stream_t stream) {
  if (!sizes_ok(rows, width, classes) || !tokens_ok(tokens, token_bits, rows) ||
      !matrix_ok(weight, weight_type, weight_stride, classes, width) || !matrix_ok(out, out_type, out_stride, rows, width) ||
      !(scale - scale == 0.f) ||
      !all_apart({span_of(out, rows, out_stride, width, dtype_bytes(out_type))},
                 {span_of(weight, classes, weight_stride, width, dtype_bytes(weight_type)), span_of(tokens, rows, size_t(token_bits) / 8)}))
    return ACDC_ERR_INVALID_ARG;
  if (rows == 0) return ACDC_OK;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  // parts of a row where few rows would leave the card idle
  const int64_t most = (width + kSpan - 1) / kSpan;
  const int split = int(std::clamp<int64_t>((rows >= 8192 ? 32768 : 2048) / rows, 1, most));
  with_types(weight_type, out_type, [&]<class TW, class TO>() {
    auto go = [&]<int ROWS>() {
      const int64_t items = (rows + ROWS - 1) / ROWS * split;
      hipLaunchKernelGGL((k_embed<TW, TO, ROWS>), dim3(unsigned(std::min<int64_t>((items + kWaves - 1) / kWaves, 1 << 16))),
                         dim3(kThreads), 0, s, tokens, token_bits, static_cast<const typename TW::Elem*>(weight),
                         (long long)weight_stride, scale, static_cast<typename TO::Elem*>(out), (long long)out_stride, int(rows),
                         width, classes, split);
    };
    // four rows a wave where a row is too short to keep one busy (131072 rows of 257 32 us for
    // 37, 65536 of 256 12 for 19; but 32768 of 512 13 for 11, of 1024 34 for 24)
    if (rows >= 8192 && width <= kSpan / 4 * 3) go.template operator()<4>();
    else go.template operator()<1>();
  });
  return done();
}

extern "C" size_t acdc_embedding_workspace_size(int64_t rows, int32_t width, int32_t classes) {
  return sizes_ok(rows, width, classes) ? std::max<size_t>(256, layout(rows, width, classes).bytes) : 0;
}

extern "C" int acdc_embedding_backward(const void* tokens, int32_t token_bits, const void* grad_out, int32_t out_type,
                                       int64_t out_stride, float scale, void* grad_weight, int32_t weight_type,
                                       int64_t weight_stride, int32_t accumulate, int64_t rows, int32_t width,
                                       int32_t classes, void* workspace, size_t workspace_bytes, acdc_stream_t stream) {
  if (!sizes_ok(rows, width, classes) || !tokens_ok(tokens, token_bits, rows) ||
      !matrix_ok(grad_out, out_type, out_stride, rows, width) || !matrix_ok(grad_weight, weight_type, weight_stride, classes, width) ||
      !(scale - scale == 0.f) || !aligned_to(workspace, 256))
    return ACDC_ERR_INVALID_ARG;
  const Span gw = span_of(grad_weight, classes, weight_stride, width, dtype_bytes(weight_type)),
             g = span_of(grad_out, rows, out_stride, width, dtype_bytes(out_type)), t = span_of(tokens, rows, size_t(token_bits) / 8);
  if (!all_apart({gw}, {g, t})) return ACDC_ERR_INVALID_ARG;
  const Layout w = layout(rows, width, classes);
  if (workspace == nullptr || workspace_bytes < w.bytes) return ACDC_ERR_WORKSPACE;
  if (!all_apart({span_of(workspace, int64_t(w.bytes), 1)}, {gw, g, t})) return ACDC_ERR_INVALID_ARG;
  if (rows == 0 && accumulate != 0) return ACDC_OK;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  char* ws = static_cast<char*>(workspace);
  unsigned char* there = reinterpret_cast<unsigned char*>(ws + w.there);
  int* counts = reinterpret_cast<int*>(ws + w.counts);
  int* totals = reinterpret_cast<int*>(ws + w.totals);
  Sorted pairs[2];
  for (int k = 0; k < 2; ++k) pairs[k] = Sorted{reinterpret_cast<int*>(ws + w.key[k]), reinterpret_cast<int*>(ws + w.row[k])};
  // passes of as many bits each; `classes` is a key too
  int key_bits = 0;
  while ((int64_t(classes) >> key_bits) != 0) ++key_bits;
  const int passes = (key_bits + kMostBits - 1) / kMostBits, digit_bits = (key_bits + passes - 1) / passes, n = int(rows);
  int at = 0;
  const bool small = rows <= kSmall;
  // zeros over everything before the sums are written, or only where no token is: the first
  // writes up to `rows` rows twice, the second takes two launches (16384 rows of 1024 over
  // 5000 classes: 41 and 43 us; over 20000 55 and 53)
  const bool mark = !small && accumulate == 0 && classes > rows / 2;
  if (small) {
    const int64_t fill = accumulate != 0 ? 0 : std::min<int64_t>((classes + 15) / 16, 1023);
    with_types(out_type, weight_type, [&]<class TG, class TW>() {
      hipLaunchKernelGGL(k_sort_small<TW>, dim3(unsigned(1 + fill)), dim3(kSmallThreads), 0, s, tokens, token_bits, classes, pairs[0], n,
                         digit_bits, passes, static_cast<typename TW::Elem*>(grad_weight), (long long)weight_stride, width);
    });
  } else {
    if (mark)
      hipLaunchKernelGGL(k_embed_clear, dim3(unsigned(std::min<int64_t>((classes + kThreads - 1) / kThreads, 1024))), dim3(kThreads), 0,
                         s, there, classes);
    const int each = each_of(rows), tile = kThreads * each, tiles = (n + tile - 1) / tile;
    for (int pass = 0; pass < passes; ++pass, at ^= 1) {
      const void* from = pass == 0 ? tokens : nullptr;
      const int fill = pass == 0 && accumulate == 0 && !mark ? int(std::min<int64_t>((classes + kWaves - 1) / kWaves, 2048)) : 0;
      with_types(out_type, weight_type, [&]<class TG, class TW>() {
        hipLaunchKernelGGL((each == 8 ? k_sort_count<TW, 8> : k_sort_count<TW, 2>), dim3(unsigned(tiles + fill)), dim3(kThreads), 0, s, from, token_bits, classes, pairs[at], n,
                           pass * digit_bits, (1 << digit_bits) - 1, counts, pass == 0 && mark ? there : nullptr, tiles,
                           static_cast<typename TW::Elem*>(grad_weight), (long long)weight_stride, width);
      });
      hipLaunchKernelGGL(k_sort_sums, dim3(kDigits / 64), dim3(64 * kSumWaves), 0, s, counts, tiles, totals);
      hipLaunchKernelGGL((each == 8 ? k_sort_move<8> : k_sort_move<2>), dim3(unsigned(tiles)), dim3(kThreads), 0, s, from, token_bits, classes, pairs[at], pairs[at ^ 1],
                         n, pass * digit_bits, digit_bits, counts, totals);
    }
  }
  with_types(out_type, weight_type, [&]<class TG, class TW>() {
    typename TW::Elem* out = static_cast<typename TW::Elem*>(grad_weight);
    if (mark)
      hipLaunchKernelGGL(k_embed_zeros<TW>, dim3(unsigned(std::min<int64_t>((classes + kWaves - 1) / kWaves, 8192))), dim3(kThreads),
                         0, s, there, classes, width, out, (long long)weight_stride);
    if (rows == 0) return;
    const int blocks = blocks_of(width), piece = piece_of(rows, width), pieces = int((rows + piece - 1) / piece);
    const SumArgs a{pairs[at].key, pairs[at].row, int(rows), classes, width, piece, pieces, blocks, scale, out_stride, weight_stride,
                    reinterpret_cast<float*>(ws + w.partial), accumulate != 0};
    const unsigned groups = unsigned((int64_t(pieces) * blocks + kWaves - 1) / kWaves);
    hipLaunchKernelGGL((k_embed_sums<TG, TW>), dim3(groups), dim3(kThreads), 0, s, a, static_cast<const typename TG::Elem*>(grad_out), out);
    if (pieces > 1)
      hipLaunchKernelGGL(k_embed_join<TW>, dim3(unsigned(int64_t((pieces + kJoinWaves - 1) / kJoinWaves) * blocks)),
                         dim3(64 * kJoinWaves), 0, s, a, out);
  });
  return done();
}
