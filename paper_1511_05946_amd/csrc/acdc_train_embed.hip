// Rows of a weight looked up by tokens, and the weight's gradient
// (acdc_train_lm.h).
//
// The gradient of a class is the sum of the gradients of its rows.  The rows
// are sorted by token (a stable radix sort of eight bits a pass), so that those
// of a class follow one another, in their order; then 64 sorted rows at a
// time are summed class by class.  A class that begins and ends within the 64
// is written at once; of one that goes on, each 64 leave a partial sum, which
// a second launch adds up in order.  No sum depends on the order in which
// anything runs.  Bound by HBM: each gradient row is read once, each row of
// the weight's gradient written once.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "acdc_train_lm.h"
#include "acdc_train_rows.hpp"

namespace acdc {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;

// `classes` for a row that takes no part: sorted behind all others.
__device__ __forceinline__ int key_of(const void* tokens, int bits, long long r, int classes) {
  const long long t = bits == 64 ? static_cast<const long long*>(tokens)[r] : (long long)static_cast<const int*>(tokens)[r];
  return t < 0 || t >= classes ? classes : int(t);
}

// ----------------------------------------------------------------- the lookup

// A wave takes one of `split` parts of a row.
template <class TW, class TO>
__global__ __launch_bounds__(kThreads) void k_embed(const void* __restrict__ tokens, int bits,
                                                    const typename TW::Elem* __restrict__ weight, long long weight_stride,
                                                    float scale, typename TO::Elem* __restrict__ out, long long out_stride,
                                                    int rows, int width, int classes, int split) {
  const int lane = threadIdx.x % 64;
  const unsigned items = unsigned(rows) * unsigned(split);
  for (unsigned item = blockIdx.x * kWaves + uniform(int(threadIdx.x / 64)); item < items; item += gridDim.x * kWaves) {
    const long long r = item / unsigned(split);
    const int part = int(item % unsigned(split));
    const long long t = bits == 64 ? static_cast<const long long*>(tokens)[r] : (long long)static_cast<const int*>(tokens)[r];
    const float fill = t < 0 ? 0.f : __builtin_nanf("");
    const bool there = t >= 0 && t < classes;
    const typename TW::Elem* from = weight + (there ? t : 0) * weight_stride;
    typename TO::Elem* to = out + r * out_stride;
#pragma unroll 4
    for (int col = (part * 64 + lane) * kEight; col < width; col += split * 64 * kEight) {
      float v[kEight];
      if (there) load_some<TW>(from + col, width - col, 0.f, v);
#pragma unroll
      for (int i = 0; i < kEight; ++i) v[i] = there ? v[i] * scale : fill;
      store_some<TO>(to + col, width - col, v);
    }
  }
}

// ------------------------------------------------------------------- the sort

// Pairs of a key and its row in tiles of kTile, a wave's kEach x 64 of them following
// one another.
constexpr int kEach = 8, kTile = kThreads * kEach, kDigits = 256;
struct Pairs {
  int* key;
  int* row;
};

// How often each digit comes in each tile: counts[digit][tile].  In the first pass
// the keys come from the tokens, and each token is marked as one that is there.
__global__ __launch_bounds__(kThreads) void k_sort_count(const void* __restrict__ tokens, int bits, int classes, Pairs in,
                                                         int n, int shift, int tiles, int* __restrict__ counts,
                                                         unsigned char* __restrict__ there) {
  __shared__ int bins[kDigits];
  bins[threadIdx.x] = 0;
  __syncthreads();
#pragma unroll
  for (int q = 0; q < kEach; ++q) {
    const int i = blockIdx.x * kTile + q * kThreads + threadIdx.x;
    if (i < n) {
      const int k = tokens != nullptr ? key_of(tokens, bits, i, classes) : in.key[i];
      if (tokens != nullptr && k < classes) there[k] = 1;
      atomicAdd(&bins[(k >> shift) & (kDigits - 1)], 1);  // (whole numbers: any order gives the same)
    }
  }
  __syncthreads();
  counts[threadIdx.x * tiles + blockIdx.x] = bins[threadIdx.x];
}

// Exclusive sums of `n` counts, in place, by one workgroup.
constexpr int kScan = 1024;
__global__ __launch_bounds__(kScan) void k_sort_scan(int* __restrict__ counts, int n) {
  __shared__ int waves[kScan / 64];
  constexpr int EACH = 8;
  const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
  int before = 0;
  for (int base = 0; base < n; base += kScan * EACH) {
    int v[EACH], mine = 0;
    const int first = base + tid * EACH;
#pragma unroll
    for (int q = 0; q < EACH; ++q) {
      v[q] = first + q < n ? counts[first + q] : 0;
      mine += v[q];
    }
    int sum = mine;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int up = __shfl_up(sum, o);
      if (lane >= o) sum += up;
    }
    if (lane == 63) waves[wave] = sum;
    __syncthreads();
    int at = before + sum - mine;
#pragma unroll
    for (int w = 0; w < kScan / 64; ++w) {
      if (w < wave) at += waves[w];
      before += waves[w];
    }
    __syncthreads();
#pragma unroll
    for (int q = 0; q < EACH; ++q)
      if (first + q < n) {
        counts[first + q] = at;
        at += v[q];
      }
  }
}

// Each pair to its place: after those of lower digits, of earlier tiles, of earlier
// waves, of earlier rounds and of lower lanes with the same digit.
__global__ __launch_bounds__(kThreads) void k_sort_move(const void* __restrict__ tokens, int bits, int classes, Pairs in,
                                                        Pairs out, int n, int shift, int tiles, const int* __restrict__ counts) {
  __shared__ int next[kWaves][kDigits];
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const int base = blockIdx.x * kTile + wave * (64 * kEach);
#pragma unroll
  for (int w = 0; w < kWaves; ++w) next[w][threadIdx.x] = 0;
  __syncthreads();
  int key[kEach], row[kEach];
#pragma unroll
  for (int q = 0; q < kEach; ++q) {
    const int i = base + q * 64 + lane;
    if (i < n) {
      key[q] = tokens != nullptr ? key_of(tokens, bits, i, classes) : in.key[i];
      row[q] = tokens != nullptr ? i : in.row[i];
      atomicAdd(&next[wave][(key[q] >> shift) & (kDigits - 1)], 1);
    }
  }
  __syncthreads();
  {
    int at = counts[threadIdx.x * tiles + blockIdx.x];
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const int c = next[w][threadIdx.x];
      next[w][threadIdx.x] = at;
      at += c;
    }
  }
  __syncthreads();
#pragma unroll
  for (int q = 0; q < kEach; ++q) {
    const bool here = base + q * 64 + lane < n;
    const int digit = (key[q] >> shift) & (kDigits - 1);
    // the lanes of this round with the same digit
    unsigned long long same = __ballot(here);
#pragma unroll
    for (int b = 0; b < 8; ++b) {
      const unsigned long long set = __ballot(here && (digit >> b & 1));
      same &= (digit >> b & 1) ? set : ~set;
    }
    const int rank = __popcll(same & ((1ull << lane) - 1)), many = __popcll(same);
    int to = 0;
    if (here) to = next[wave][digit] + rank;
    wave_sync();  // everyone has read before the last of a digit writes
    if (here && rank == many - 1) next[wave][digit] = to + 1;
    wave_sync();
    if (here) {
      out.key[to] = key[q];
      out.row[to] = row[q];
    }
  }
}

// --------------------------------------------------------------- the gradient

constexpr int kPiece = 64;  // sorted rows that are summed together

struct SumArgs {
  const int* key;
  const int* row;
  int rows, classes, width, pieces, blocks;
  float scale;
  long long grad_stride, weight_stride;
  float* partial;  // [pieces][2][width]: the sum that the piece begins with, and the one it ends with
  bool add;
};

template <class TW>
__device__ __forceinline__ void put_class(typename TW::Elem* to, int left, const float (&v)[kEight], float scale, bool add) {
  float o[kEight] = {};
  if (add) load_some<TW>(to, left, 0.f, o);
#pragma unroll
  for (int i = 0; i < kEight; ++i) o[i] += scale * v[i];
  store_some<TW>(to, left, o);
}

// A wave sums 64 sorted rows in 512 columns.
template <class TG, class TW>
__global__ __launch_bounds__(kThreads) void k_embed_sums(SumArgs a, const typename TG::Elem* __restrict__ grad,
                                                         typename TW::Elem* __restrict__ weight) {
  const int lane = threadIdx.x % 64;
  const long long item = (long long)blockIdx.x * kWaves + uniform(int(threadIdx.x / 64));
  if (item >= (long long)a.pieces * a.blocks) return;
  const int piece = int(item / a.blocks), col = (int(item % a.blocks) * 64 + lane) * kEight, left = a.width - col;
  const int from = piece * kPiece, to = min(a.rows, from + kPiece);
  // one sorted row a lane; the loop passes them on
  const int mine = from + lane < to ? a.key[from + lane] : a.classes;
  const int mine_row = from + lane < to ? a.row[from + lane] : 0;
  const int before = from > 0 ? a.key[from - 1] : -1, after = to < a.rows ? a.key[to] : -1;
  float s[kEight] = {};
  int current = uniform(mine);
  bool began = current != before;  // the class begins in this piece
  constexpr int AHEAD = 4;
  for (int i = 0; i < to - from; i += AHEAD) {
    float v[AHEAD][kEight];
    int key[AHEAD];
#pragma unroll
    for (int q = 0; q < AHEAD; ++q) {
      const int at = min(i + q, to - from - 1);
      key[q] = __builtin_amdgcn_readlane(mine, at);
      const long long r = __builtin_amdgcn_readlane(mine_row, at);
      if (key[q] < a.classes && left > 0) load_some<TG>(grad + r * a.grad_stride + col, left, 0.f, v[q]);
    }
#pragma unroll
    for (int q = 0; q < AHEAD; ++q) {
      if (i + q >= to - from) break;
      if (key[q] != current) {  // the class before ends here
        if (left > 0) {
          if (began) put_class<TW>(weight + current * a.weight_stride + col, left, s, a.scale, a.add);
          else store_some<F32, false>(a.partial + (long long)piece * 2 * a.width + col, left, s);
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
  if (current >= a.classes || left <= 0) return;
  if (current == after || !began)
    store_some<F32, false>(a.partial + ((long long)piece * 2 + (began ? 1 : 0)) * a.width + col, left, s);
  else
    put_class<TW>(weight + current * a.weight_stride + col, left, s, a.scale, a.add);
}

// The class that begins in a piece and goes on behind it: its partial sums together.
template <class TW>
__global__ __launch_bounds__(kThreads) void k_embed_join(SumArgs a, typename TW::Elem* __restrict__ weight) {
  const int lane = threadIdx.x % 64;
  const long long item = (long long)blockIdx.x * kWaves + uniform(int(threadIdx.x / 64));
  if (item >= (long long)a.pieces * a.blocks) return;
  const int piece = int(item / a.blocks), col = (int(item % a.blocks) * 64 + lane) * kEight, left = a.width - col;
  const int from = piece * kPiece, to = from + kPiece;
  if (to >= a.rows || left <= 0) return;
  const int key = a.key[to];
  if (key >= a.classes || a.key[to - 1] != key) return;        // nothing goes on
  if (a.key[from] == key && from > 0 && a.key[from - 1] == key) return;  // it began before
  float s[kEight];
  load_some<F32>(a.partial + ((long long)piece * 2 + 1) * a.width + col, left, 0.f, s);
#pragma unroll 4
  for (int p = piece + 1; p < a.pieces && a.key[p * kPiece] == key; ++p) {
    float v[kEight];
    load_some<F32>(a.partial + (long long)p * 2 * a.width + col, left, 0.f, v);
#pragma unroll
    for (int c = 0; c < kEight; ++c) s[c] += v[c];
  }
  put_class<TW>(weight + key * a.weight_stride + col, left, s, a.scale, a.add);
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
    for (int col = lane * kEight; col < width; col += 64 * kEight) store_some<TW>(weight + v * weight_stride + col, width - col, zero);
  }
}

// ------------------------------------------------------------------ on the host

constexpr int64_t kMostRows = 1 << 28, kMostClasses = 1 << 30, kMostWidth = 1 << 20, kMostStride = int64_t(1) << 40;

int done() {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? ACDC_OK : hip_fail(e);
}
size_t up256(size_t n) { return (n + 255) & ~size_t(255); }
struct Layout {
  size_t key[2], row[2], counts, there, partial, bytes;
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
  w.counts = take((n + kTile - 1) / kTile * kDigits * 4);
  w.there = take(size_t(classes));
  w.partial = take((n + kPiece - 1) / kPiece * 2 * size_t(width) * 4);
  w.bytes = next;
  return w;
}
bool sizes_ok(int64_t rows, int32_t width, int32_t classes) {
  return rows >= 0 && rows <= kMostRows && width >= 1 && width <= kMostWidth && classes >= 1 && classes <= kMostClasses;
}
bool matrix_ok(const void* p, int32_t dtype, int64_t stride, int64_t rows, int32_t width) {
  const size_t e = dtype_bytes(dtype);
  return e != 0 && stride >= width && stride <= kMostStride && aligned_to(p, e) && (rows == 0 || p != nullptr);
}
bool tokens_ok(const void* tokens, int32_t bits, int64_t rows) {
  return (bits == 32 || bits == 64) && aligned_to(tokens, size_t(bits) / 8) && (rows == 0 || tokens != nullptr);
}
bool apart(const void* p, int64_t rows, int64_t stride, int32_t type, const void* q, int64_t others, int64_t other_stride,
           int32_t other_type, int64_t width) {
  if (rows == 0 || others == 0) return true;
  const char *a = static_cast<const char*>(p), *b = static_cast<const char*>(q);
  const char* a_end = a + (size_t(rows - 1) * size_t(stride) + size_t(width)) * dtype_bytes(type);
  const char* b_end = b + (size_t(others - 1) * size_t(other_stride) + size_t(width)) * dtype_bytes(other_type);
  return a_end <= b || b_end <= a;
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
      !(scale - scale == 0.f) || !apart(out, rows, out_stride, out_type, weight, classes, weight_stride, weight_type, width))
    return ACDC_ERR_INVALID_ARG;
  if (rows == 0) return ACDC_OK;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  // parts of a row where few rows would leave the card idle
  const int64_t most = (width + 64 * kEight - 1) / (64 * kEight);
  const int split = int(std::clamp<int64_t>(2048 / rows, 1, most));
  const unsigned blocks = unsigned(std::min<int64_t>((rows * split + kWaves - 1) / kWaves, 1 << 16));
  with_types(weight_type, out_type, [&]<class TW, class TO>() {
    hipLaunchKernelGGL((k_embed<TW, TO>), dim3(blocks), dim3(kThreads), 0, s, tokens, token_bits,
                       static_cast<const typename TW::Elem*>(weight), (long long)weight_stride, scale,
                       static_cast<typename TO::Elem*>(out), (long long)out_stride, int(rows), width, classes, split);
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
      !(scale - scale == 0.f) || !aligned_to(workspace, 256) ||
      !apart(grad_weight, classes, weight_stride, weight_type, grad_out, rows, out_stride, out_type, width))
    return ACDC_ERR_INVALID_ARG;
  const Layout w = layout(rows, width, classes);
  if (workspace == nullptr || workspace_bytes < w.bytes) return ACDC_ERR_WORKSPACE;
  if (rows == 0 && accumulate != 0) return ACDC_OK;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  char* ws = static_cast<char*>(workspace);
  unsigned char* there = reinterpret_cast<unsigned char*>(ws + w.there);
  int* counts = reinterpret_cast<int*>(ws + w.counts);
  Pairs pairs[2];
  for (int k = 0; k < 2; ++k) pairs[k] = Pairs{reinterpret_cast<int*>(ws + w.key[k]), reinterpret_cast<int*>(ws + w.row[k])};
  hipLaunchKernelGGL(k_embed_clear, dim3(unsigned(std::min<int64_t>((classes + kThreads - 1) / kThreads, 1024))), dim3(kThreads), 0, s,
                     there, classes);
  int at = 0;
  if (rows > 0) {
    const int n = int(rows), tiles = (n + kTile - 1) / kTile;
    for (int shift = 0; shift == 0 || (classes >> shift) != 0; shift += 8, at ^= 1) {
      const void* from = shift == 0 ? tokens : nullptr;
      hipLaunchKernelGGL(k_sort_count, dim3(unsigned(tiles)), dim3(kThreads), 0, s, from, token_bits, classes, pairs[at], n, shift,
                         tiles, counts, there);
      hipLaunchKernelGGL(k_sort_scan, dim3(1), dim3(kScan), 0, s, counts, tiles * kDigits);
      hipLaunchKernelGGL(k_sort_move, dim3(unsigned(tiles)), dim3(kThreads), 0, s, from, token_bits, classes, pairs[at],
                         pairs[at ^ 1], n, shift, tiles, counts);
    }
  }
  with_types(out_type, weight_type, [&]<class TG, class TW>() {
    typename TW::Elem* out = static_cast<typename TW::Elem*>(grad_weight);
    if (accumulate == 0)
      hipLaunchKernelGGL(k_embed_zeros<TW>, dim3(unsigned(std::min<int64_t>((classes + kWaves - 1) / kWaves, 8192))), dim3(kThreads),
                         0, s, there, classes, width, out, (long long)weight_stride);
    if (rows == 0) return;
    const int blocks = (width + 64 * kEight - 1) / (64 * kEight), pieces = int((rows + kPiece - 1) / kPiece);
    const SumArgs a{pairs[at].key, pairs[at].row, int(rows), classes, width, pieces, blocks, scale, out_stride, weight_stride,
                    reinterpret_cast<float*>(ws + w.partial), accumulate != 0};
    const unsigned groups = unsigned((int64_t(pieces) * blocks + kWaves - 1) / kWaves);
    hipLaunchKernelGGL((k_embed_sums<TG, TW>), dim3(groups), dim3(kThreads), 0, s, a, static_cast<const typename TG::Elem*>(grad_out), out);
    if (pieces > 1) hipLaunchKernelGGL(k_embed_join<TW>, dim3(groups), dim3(kThreads), 0, s, a, out);
  });
  return done();
}
