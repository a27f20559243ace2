// The optimiser's operators (acdc_train.h): an AdamW step over a list of
// tensors and the global norm of their gradients.
//
// Mathematics.  Every element is on its own (m, v, w of one element), but for
// the scales of 8-bit moments, one per 256 elements: the block's maximum has
// to be known before its first code is written.
//
// The tensors' addresses travel in the kernels' arguments, 62 to 104 tensors a
// launch and as offsets 103 to 156: nothing is uploaded, and no table outlives
// the call.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstring>
#include <type_traits>

#include "acdc_train.hpp"

namespace acdc {
namespace {

constexpr int kThreads = 256;
constexpr int kBlock = 256;     // elements that share a scale: 4 of each lane of a wave
constexpr int kChunk = kThreads * 4;  // elements a workgroup: four a thread, and no loop
constexpr float kPerTop = 1.f / 448.f;  // 448: largest e4m3 value
constexpr float kTiny = 0x1p-9f;  // smallest positive one

// A tensor is a few words of an address each, below 2^48: param, grad, m, v, then
// m_scale and v_scale (8 bits), master.  Three words have 16 bits of its length
// on top, the fourth the index of its rate.  More tensors fit a launch's arguments
// that way, and fewer launches drain and fill the card: 300 tensors, 560 MB, took
// 118 us with 48 whole records a launch, and 106 so.
constexpr int kArguments = 3840;  // bytes, of the 4 KB that a launch has
constexpr int kFewArguments = 480;
constexpr int kRates = 8;
constexpr unsigned long long kAddress = (1ull << 48) - 1;
struct Rate {
  float rate, decay;  // lr / (1 - beta1^step), 1 - lr * weight_decay
};
// A list that fits an eighth of the arguments goes in as many: they are copied
// whole at each launch, and three tensors of 256 floats, step after step, take
// 4.8 us so and 6.2 with the long ones (eleven 4.8 and 5.2, and with 1024 bytes
// 5.1).
template <int WORDS, int BYTES>
struct Batch {
  static constexpr int kMost = int((BYTES - kRates * sizeof(Rate)) / (4 + 8 * WORDS));
  unsigned long long word[kMost][WORDS];
  Rate rate[kRates];
  int first[kMost];  // first workgroup of each tensor
  void put(int i, const void* const (&p)[WORDS], unsigned long long n, int begin, int r) {
    for (int k = 0; k < WORDS; ++k) {
      const unsigned long long top = k < 3 ? n >> 16 * k & 0xffff : k == 3 ? (unsigned long long)r : 0;
      word[i][k] = (unsigned long long)reinterpret_cast<uintptr_t>(p[k]) | top << 48;
    }
    first[i] = begin;
  }
  __device__ __forceinline__ unsigned long long address(int i, int k) const { return word[i][k] & kAddress; }
  __device__ __forceinline__ long long length(int i) const {
    return (long long)(word[i][0] >> 48 | word[i][1] >> 48 << 16 | word[i][2] >> 48 << 32);
  }
  __device__ __forceinline__ int rate_of(int i) const { return int(word[i][3] >> 48); }
};
// Longer lists go as 32-bit offsets from the lowest address of each kind where
// those reach: in units of 16 bytes, and of 4 for the scales.  300 tensors with
// 8-bit moments, 327 MB, take three launches for five so, 70 us for 75, and 200
// with copies two for three, 765 us for 768.  In both forms the rate's index
// lies with what is loaded anyway: beside the first workgroup, where its load
// begins a little later, 400 M elements with 8-bit moments took 1050 us for 1032.
template <int WORDS>
struct NearBatch {
  static constexpr int kMost = int((kArguments - kRates * sizeof(Rate) - 8 * WORDS) / (8 + 4 * WORDS));
  static constexpr int shift(int k) { return WORDS >= 6 && (k == 4 || k == 5) ? 2 : 4; }
  unsigned long long base[WORDS];
  Rate rate[kRates];
  unsigned offset[kMost][WORDS];
  unsigned n[kMost];  // length | index of the rate << 29
  int first[kMost];
  void put(int i, const void* const (&p)[WORDS], unsigned long long length, int begin, int r) {
    for (int k = 0; k < WORDS; ++k) offset[i][k] = unsigned((reinterpret_cast<uintptr_t>(p[k]) - base[k]) >> shift(k));
    n[i] = unsigned(length) | unsigned(r) << 29;
    first[i] = begin;
  }
  __device__ __forceinline__ unsigned long long address(int i, int k) const {
    return base[k] + ((unsigned long long)offset[i][k] << shift(k));
  }
  __device__ __forceinline__ long long length(int i) const { return n[i] & ((1u << 29) - 1); }
  __device__ __forceinline__ int rate_of(int i) const { return int(n[i] >> 29); }
};
constexpr int words_of(int bits, bool master) { return 4 + (bits == 8 ? 2 : 0) + (master ? 1 : 0); }
template <int WORDS>
constexpr bool fits = sizeof(Batch<WORDS, kArguments>) <= kArguments &&
                      sizeof(Batch<WORDS, kFewArguments>) <= kFewArguments && sizeof(NearBatch<WORDS>) <= kArguments;
static_assert(kRates <= 8 && fits<4> && fits<5> && fits<6> && fits<7>);
static_assert(Batch<7, kArguments>::kMost == 62 && Batch<4, kArguments>::kMost == 104 && NearBatch<7>::kMost == 103 &&
              NearBatch<4>::kMost == 156);

struct Step {
  double one1, one2;      // 1 - beta
  float c1, c2;           // the same, for gradients without a scale
  float beta1, beta2;
  float root_scale, eps;  // 1 / sqrt(1 - beta2^step)
  const float* grad_scale;
};

// The tensor that a workgroup works on: the last one whose first workgroup is
// not after it.  One load per lane and a ballot for 64 tensors at a time.
__device__ __forceinline__ int tensor_of(const int* first, int count, int block) {
  int i = -1;
  for (int base = 0; base < count; base += 64) {
    const int k = base + int(threadIdx.x) % 64;
    i += __popcll(__ballot(k < count ? first[k] <= block : false));
  }
  return __builtin_amdgcn_readfirstlane(i);
}

// Four elements, the first of them at p; `have` of them exist.
template <class T, bool NT>
__device__ __forceinline__ void load4(const void* base, long long at, int have, float (&v)[4]) {
  typedef typename T::Elem V4 __attribute__((ext_vector_type(4), aligned(sizeof(typename T::Elem))));
  const typename T::Elem* p = static_cast<const typename T::Elem*>(base) + at;
  if (have == 4) {
    const V4 r = load_as<NT>(reinterpret_cast<const V4*>(p));
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = float(r[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = i < have ? float(p[i]) : 0.f;
  }
}
template <class T, bool NT>
__device__ __forceinline__ void store4(void* base, long long at, int have, const float (&v)[4]) {
  typedef typename T::Elem V4 __attribute__((ext_vector_type(4), aligned(sizeof(typename T::Elem))));
  typename T::Elem* p = static_cast<typename T::Elem*>(base) + at;
  if (have == 4) {
    store_as<NT>(reinterpret_cast<V4*>(p), V4{T::to(v[0]), T::to(v[1]), T::to(v[2]), T::to(v[3])});
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < have) p[i] = T::to(v[i]);
  }
}

// Four e4m3 codes as one word.
typedef unsigned Word1 __attribute__((aligned(1)));
template <bool NT>
__device__ __forceinline__ unsigned load_codes(const void* base, long long at, int have) {
  const unsigned char* p = static_cast<const unsigned char*>(base) + at;
  if (have == 4) return load_as<NT>(reinterpret_cast<const Word1*>(p));
  unsigned w = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (i < have) w |= unsigned(p[i]) << (8 * i);
  return w;
}
template <bool NT>
__device__ __forceinline__ void store_codes(void* base, long long at, int have, unsigned w) {
  unsigned char* p = static_cast<unsigned char*>(base) + at;
  if (have == 4) {
    store_as<NT>(reinterpret_cast<Word1*>(p), Word1(w));
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < have) p[i] = (unsigned char)(w >> (8 * i));
  }
}
__device__ __forceinline__ void decode4(unsigned w, float scale, float (&v)[4]) {
  const auto a = __builtin_amdgcn_cvt_pk_f32_fp8(int(w), false), b = __builtin_amdgcn_cvt_pk_f32_fp8(int(w), true);
  v[0] = a[0] * scale;
  v[1] = a[1] * scale;
  v[2] = b[0] * scale;
  v[3] = b[1] * scale;
}
// Codes of four values of a block with this scale; positive values stay
// positive with POSITIVE.  A NaN keeps its own code.  The quotient v / scale is
// correctly rounded: with r the rounded reciprocal, q + r (v - q scale) of q = v r
// is (Markstein's division), three instructions a value and one division a block.
template <bool POSITIVE>
__device__ __forceinline__ unsigned encode4(const float (&v)[4], float scale) {
  const float s = scale, r = s > 0.f ? 1.f / s : 0.f;  // (a scale of 0 has codes of 0, and NaN)
  float q[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float q0 = v[i] * r;
    q[i] = fmaf(fmaf(-q0, s, v[i]), r, q0);
    if (POSITIVE) q[i] = v[i] > 0.f ? fmaxf(q[i], kTiny) : q[i];
  }
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(q[0], q[1], 0, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(q[2], q[3], w, true);
  return unsigned(w);
}
// Square roots of four values, correctly rounded but for rare cases a unit in
// the last place off: s = v rsq(v), then s + rsq(v) / 2 (v - s s).  Denormal
// values, infinities and NaN, which the instruction does not take, go the long
// way, all lanes together.
__device__ __forceinline__ void roots4(const float (&v)[4], float (&root)[4]) {
  constexpr int kOdd = 0x3 | 0x204 | 0x90;  // NaN, infinities, denormals
  bool odd = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) odd |= __builtin_amdgcn_classf(v[i], kOdd);
  if (__any(odd)) {
#pragma unroll 1
    for (int i = 0; i < 4; ++i) root[i] = sqrtf(v[i]);
    return;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float r = __builtin_amdgcn_rsqf(fmaxf(v[i], 0x1p-126f)), s = v[i] * r;
    root[i] = fmaf(fmaf(-s, s, v[i]), 0.5f * r, s);
  }
}
// Scale of a wave's block out of each lane's four values.  Blocks below 2^-100
// are 0: their scale would leave the normal numbers.  (The product may leave the
// largest element a rounding away from 448, which its code does not see.)
// Infinities become NaN, which no maximum sees: their block keeps a scale for
// the others.
__device__ __forceinline__ float block_top(const float (&v)[4]) {
  return wave_max(fmaxf(fmaxf(fabsf(v[0]), fabsf(v[1])), fmaxf(fabsf(v[2]), fabsf(v[3]))));
}
__device__ __forceinline__ float scale_of(float (&v)[4]) {
  float top = block_top(v);
  if (top == __builtin_inff()) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (fabsf(v[i]) == __builtin_inff()) v[i] = __builtin_nanf("");
    top = block_top(v);
  }
  return top < 0x1p-100f ? 0.f : top * kPerTop;
}

// The step of 1024 elements, four a thread.  Bound by HBM: 100 M floats with
// 32-bit moments, 2.8 GB, in 470 us (6.0 TB/s), 400 M with 8-bit ones, 6.4 GB, in
// 1043 us (6.2 TB/s).  No loop in a workgroup: with two and four times the
// elements in flight a thread, 20 M elements in 300 tensors took 105 and 121 us
// instead of 93.  8-bit: a wave's 64 x 4 elements are one block, whose maximum is
// a reduction by lane swaps; its scales are one scalar load each.  With the
// compiler's quotients and roots the vector unit bound it (106 % of its cycles
// at 1138 us); the step itself needs neither to the last bit.
template <class P, class G, int BITS, bool MASTER, bool NT, class LIST>
__global__ __launch_bounds__(kThreads) void k_adamw(LIST b, int count, Step s) {
  const int i = tensor_of(b.first, count, blockIdx.x);
  // (named as global memory: of a pointer made out of a number the compiler would not know)
  auto address = [&](int k) {
    return (void*)reinterpret_cast<__attribute__((address_space(1))) void*>(b.address(i, k));
  };
  struct {
    void *param, *grad, *m, *v;
    float *m_scale, *v_scale;
    void* master;
    long long n;
    float rate, decay;
  } t;
  t.param = address(0);
  t.grad = address(1);
  t.m = address(2);
  t.v = address(3);
  if constexpr (BITS == 8) {
    t.m_scale = static_cast<float*>(address(4));
    t.v_scale = static_cast<float*>(address(5));
  }
  if constexpr (MASTER) t.master = address(words_of(BITS, MASTER) - 1);
  t.n = b.length(i);
  const Rate rate = b.rate[b.rate_of(i)];
  t.rate = rate.rate;
  t.decay = rate.decay;
  float c1 = s.c1, c2 = s.c2, first = 1.f;
  if (s.grad_scale != nullptr) {
    const float gs = *s.grad_scale;
    // not finite, or -0: a gradient is NaN or infinite, and 0 * inf would spoil its element
    if (!(gs - gs == 0.f) || __float_as_uint(gs) == 0x80000000u) return;
    // The gradient's scale goes into the factors of g and g^2, each rounded once.
    // Where a factor is not a normal number (the scale's square leaves 32 bits from
    // about 1e-18 and 1e20 on), the gradient is scaled first and rounded itself.
    c1 = float(s.one1 * double(gs));
    c2 = float(s.one2 * (double(gs) * double(gs)));
    auto normal = [](float c) { return fabsf(c) >= 0x1p-126f && fabsf(c) < __builtin_inff(); };
    if (!normal(c1) || !normal(c2)) {
      first = gs;
      c1 = s.c1;
      c2 = s.c2;
    }
  }
  // a wave's 256 elements are one block of scales
  const long long base = (long long)(int(blockIdx.x) - b.first[i]) * kChunk + (threadIdx.x / 64) * kBlock;
  if (base >= t.n) return;
  const int lane = (threadIdx.x % 64) * 4;
  const long long at = base + lane, left = t.n - at;
  const int have = left >= 4 ? 4 : left > 0 ? int(left) : 0;
  float g[4], m[4], v[4], w[4];
  load4<G, NT>(t.grad, at, have, g);
  if constexpr (MASTER) load4<F32, NT>(t.master, at, have, w);
  else load4<P, NT>(t.param, at, have, w);
  if constexpr (BITS == 32) {
    load4<F32, NT>(t.m, at, have, m);
    load4<F32, NT>(t.v, at, have, v);
  } else {
    decode4(load_codes<NT>(t.m, at, have), t.m_scale[base / kBlock], m);
    decode4(load_codes<NT>(t.v, at, have), t.v_scale[base / kBlock], v);
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    // each product and sum rounded on its own, as the formula written out in
    // 32 bits is: an 8-bit code that a fused product turned the other way would
    // stand a whole step of its format off
#pragma clang fp contract(off)
    if constexpr (BITS == 8) v[k] *= v[k];
    const float x = first * g[k];
    m[k] = s.beta1 * m[k] + c1 * x;
    v[k] = s.beta2 * v[k] + c2 * x * x;
  }
  float root[4];
  roots4(v, root);
#pragma unroll
  for (int k = 0; k < 4; ++k)
    w[k] = w[k] * t.decay - t.rate * (m[k] * __builtin_amdgcn_rcpf(root[k] * s.root_scale + s.eps));
  if constexpr (MASTER) store4<F32, NT>(t.master, at, have, w);
  store4<P, NT>(t.param, at, have, w);
  if constexpr (BITS == 32) {
    store4<F32, NT>(t.m, at, have, m);
    store4<F32, NT>(t.v, at, have, v);
  } else {
    const float ms = scale_of(m), vs = scale_of(root);
    store_codes<NT>(t.m, at, have, encode4<false>(m, ms));
    store_codes<NT>(t.v, at, have, encode4<true>(root, vs));
    if (lane == 0) {
      t.m_scale[base / kBlock] = ms;
      t.v_scale[base / kBlock] = vs;
    }
  }
}

// ------------------------------------------------------------ gradient norm

constexpr int kNormBatch = 180;
constexpr int kNormRounds = 4;     // chunks of 16 bytes that a thread asks for at a time
// Elements a workgroup takes, a power of two by the list's whole size: long
// enough that finding its tensor is a small part of its time, and short enough
// that there are thousands of workgroups (about 4096 where the list allows it).
constexpr long long kNormLeast = 4096, kNormMost = 65536;
long long norm_chunk(const int64_t* sizes, int32_t count) {
  long long all = 0;
  for (int32_t i = 0; i < count; ++i) all += sizes[i];
  long long chunk = kNormLeast;
  while (chunk < kNormMost && all / (2 * chunk) >= 4096) chunk *= 2;
  return chunk;
}
struct NormTensor {
  const void* grad;
  unsigned long long n_type;  // elements << 1 | bfloat16
};
struct NormBatch {
  int first[kNormBatch];
  NormTensor t[kNormBatch];
};
static_assert(sizeof(NormBatch) <= 3840, "kernel arguments");

// Sum over the workgroup's waves in a fixed order, for thread 0.
__device__ __forceinline__ double sum_workgroup(double v, double* part, int waves) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
  if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = v;
  __syncthreads();
  double s = 0.0;
  for (int w = 0; w < waves; ++w) s += part[w];
  return s;
}

template <class G>
__device__ __forceinline__ double square_sum(const typename G::Elem* p, int count) {
  constexpr int kStep = kThreads * G::kPer;
  const int full = count / G::kPer * G::kPer;
  double total = 0.0;
  for (int base = 0; base < full; base += kStep * kNormRounds) {
    typename G::Raw raw[kNormRounds];
    const int at = base + int(threadIdx.x) * G::kPer;
#pragma unroll
    for (int q = 0; q < kNormRounds; ++q) {
      raw[q] = typename G::Raw{};
      if (at + q * kStep < full) raw[q] = load_chunk<G>(p + at + q * kStep);
    }
    // in 64 bits, which no square of a gradient leaves: 32 end at 1.8e19 and 1e-23
#pragma unroll
    for (int q = 0; q < kNormRounds; ++q)
#pragma unroll
      for (int i = 0; i < G::kPer; ++i) {
        const double v = G::get(raw[q], i);
        total += v * v;
      }
  }
  if (full + int(threadIdx.x) < count) {
    const double v = G::one(p[full + threadIdx.x]);
    total += v * v;
  }
  return total;
}

// Sum of squares of a workgroup's chunk, in 64 bits; bound by HBM: 156 M bfloat16,
// 311 MB, in 54 us (5.7 TB/s; the vector unit 23 % busy, and 18 % with squares in
// 32 bits).  Right after a step without the streaming hint it took 94: the
// Infinity Cache then writes back 256 MB of the step's before it takes what is read.
__global__ __launch_bounds__(kThreads) void k_square_sums(NormBatch b, int count, int chunk, double* __restrict__ sums) {
  __shared__ double part[kThreads / 64];
  const int i = tensor_of(b.first, count, blockIdx.x);
  const long long begin = (long long)(int(blockIdx.x) - b.first[i]) * chunk;
  const long long left = (long long)(b.t[i].n_type >> 1) - begin;
  const int n = left < chunk ? int(left) : chunk;
  const double s = b.t[i].n_type & 1 ? square_sum<BF16>(static_cast<const __bf16*>(b.t[i].grad) + begin, n)
                                     : square_sum<F32>(static_cast<const float*>(b.t[i].grad) + begin, n);
  const double total = sum_workgroup(s, part, kThreads / 64);
  if (threadIdx.x == 0) sums[blockIdx.x] = total;
}

constexpr int kWide = 1024;
// The norm and the clip coefficient out of all sums, in a fixed order: one workgroup,
// 4 us for 5000 sums.
__global__ __launch_bounds__(kWide) void k_norm(const double* __restrict__ sums, long long n, float max_norm,
                                                float* __restrict__ out) {
  __shared__ double part[kWide / 64];
  double s = 0.0;
#pragma unroll 8
  for (long long i = threadIdx.x; i < n; i += kWide) s += sums[i];
  s = sum_workgroup(s, part, kWide / 64);
  if (threadIdx.x == 0) {
    const double norm = sqrt(s);
    out[0] = float(norm);
    // (of the norm in 64 bits: one past what a float holds still clips to max_norm)
    const double c = double(max_norm) / (norm + 1e-6);
    // NaN stays; the 0 of an infinite norm goes as -0, which the step knows
    out[1] = max_norm > 0.f ? (norm == double(__builtin_inff()) ? -0.f : float(c > 1.0 ? 1.0 : c)) : 1.f;
  }
}

// ------------------------------------------------------------------ host side

int done() {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? ACDC_OK : hip_fail(e);
}

// Workgroups of a launch: a grid holds fewer than 2^32 lanes.
constexpr long long kMaxBlocks = (1LL << 32) / kThreads - 1;
constexpr int64_t kMaxElements = kMaxBlocks * kChunk;  // of a tensor

// The kernel of a class of tensors: parameter and gradient types, moments, master.
int class_of(const acdc_adamw_tensor& t) {
  return t.param_type * 8 + t.grad_type * 4 + (t.m_scale != nullptr ? 2 : 0) + (t.master != nullptr ? 1 : 0);
}
constexpr int kClasses = 16;

// Bytes of a step's tensors from which on they are not to stay in the caches: half
// of the 256 MB Infinity Cache, as the passes between two steps use it too.  (With
// the hint 160 MB of float tensors took 49 us instead of 56, 4.5 GB of bfloat16
// ones with masters 775 instead of 900; without it 80 MB took 23 instead of 26.)
constexpr double kKeepBytes = 128e6;

// f.template operator()<P, G, BITS, MASTER>() for a class.
template <class F>
void with_class(int cls, F&& f) {
  auto moments = [&]<class P, class G, bool MASTER>() {
    if (cls & 2) f.template operator()<P, G, 8, MASTER>();
    else f.template operator()<P, G, 32, MASTER>();
  };
  auto grads = [&]<class P, bool MASTER>() {
    if (cls & 4) moments.template operator()<P, BF16, MASTER>();
    else moments.template operator()<P, F32, MASTER>();
  };
  if (!(cls & 8)) grads.template operator()<F32, false>();
  else if (cls & 1) grads.template operator()<BF16, true>();
  else grads.template operator()<BF16, false>();
}

bool low48(const void* p) { return reinterpret_cast<uintptr_t>(p) <= kAddress; }

bool tensor_ok(const acdc_adamw_tensor& t) {
  const size_t pb = dtype_bytes(t.param_type), gb = dtype_bytes(t.grad_type);
  if (pb == 0 || gb == 0 || t.n < 0 || t.n > kMaxElements) return false;
  if (!(t.lr - t.lr == 0.f) || !(t.weight_decay - t.weight_decay == 0.f)) return false;
  if ((t.m_scale == nullptr) != (t.v_scale == nullptr)) return false;
  if (t.master != nullptr && t.param_type != ACDC_BF16) return false;
  if (t.n == 0) return true;
  const size_t mb = t.m_scale != nullptr ? 1 : 4;
  if (t.param == nullptr || t.grad == nullptr || t.m == nullptr || t.v == nullptr) return false;
  if (t.param == t.grad || t.m == t.v || t.m == t.param || t.v == t.param || t.master == t.param) return false;
  if (!low48(t.param) || !low48(t.grad) || !low48(t.m) || !low48(t.v) || !low48(t.m_scale) || !low48(t.v_scale) ||
      !low48(t.master))
    return false;
  return aligned_to(t.param, pb) && aligned_to(t.grad, gb) && aligned_to(t.master, 4) && aligned_to(t.m, mb) &&
         aligned_to(t.v, mb) && aligned_to(t.m_scale, 4) && aligned_to(t.v_scale, 4);
}

}  // namespace
}  // namespace acdc

using namespace acdc;

extern "C" int acdc_adamw_step(const acdc_adamw_tensor* tensors, int32_t count, double beta1, double beta2, double eps,
                               int64_t step, const float* grad_scale, acdc_stream_t stream) {
  if (count < 0 || (count > 0 && tensors == nullptr) || step < 1 || !aligned_to(grad_scale, 4))
    return ACDC_ERR_INVALID_ARG;
  if (!(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0) || !(eps >= 0.0) || !(eps - eps == 0.0))
    return ACDC_ERR_INVALID_ARG;
  for (int32_t i = 0; i < count; ++i)
    if (!tensor_ok(tensors[i])) return ACDC_ERR_INVALID_ARG;
  const double c1 = 1.0 - std::pow(beta1, double(step)), c2 = 1.0 - std::pow(beta2, double(step));
  const Step s{1.0 - beta1, 1.0 - beta2, float(1.0 - beta1), float(1.0 - beta2), float(beta1), float(beta2),
               float(1.0 / std::sqrt(c2)), float(eps), grad_scale};
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  unsigned seen = 0;
  double bytes = 0.0;
  for (int32_t i = 0; i < count; ++i) {
    const acdc_adamw_tensor& t = tensors[i];
    seen |= 1u << class_of(t);
    bytes += double(t.n) * double(dtype_bytes(t.param_type) + dtype_bytes(t.grad_type) + (t.master != nullptr ? 4 : 0) +
                                  (t.m_scale != nullptr ? 2 : 8));
  }
  int rc = ACDC_OK;
  for (int cls = 0; cls < kClasses && rc == ACDC_OK; ++cls) {
    if (!(seen >> cls & 1)) continue;
    with_class(cls, [&]<class P, class G, int BITS, bool MASTER>() {
      constexpr int kWords = words_of(BITS, MASTER);
      using Long = Batch<kWords, kArguments>;
      using Few = Batch<kWords, kFewArguments>;
      using Near = NearBatch<kWords>;
      auto launch = [&]<class LIST>(const LIST& b, int used, long long blocks) {
        const dim3 grid(static_cast<unsigned>(blocks)), block(kThreads);
        if constexpr (!std::is_same_v<LIST, Few>) {
          if (bytes >= kKeepBytes) {
            hipLaunchKernelGGL((k_adamw<P, G, BITS, MASTER, true, LIST>), grid, block, 0, st, b, used, s);
            return;
          }
        }
        hipLaunchKernelGGL((k_adamw<P, G, BITS, MASTER, false, LIST>), grid, block, 0, st, b, used, s);
      };
      auto addresses = [](const acdc_adamw_tensor& t, const void* (&p)[kWords]) {
        p[0] = t.param;
        p[1] = t.grad;
        p[2] = t.m;
        p[3] = t.v;
        if constexpr (BITS == 8) {
          p[4] = t.m_scale;
          p[5] = t.v_scale;
        }
        if constexpr (MASTER) p[kWords - 1] = t.master;
      };
      auto all = [&]<class LIST>(LIST& b) {
        int used = 0, rates = 0;
        long long blocks = 0;
        auto flush = [&] {
          if (used == 0) return;
          bool launched = false;
          if constexpr (std::is_same_v<LIST, Long>) {
            if (used <= Few::kMost && bytes < kKeepBytes) {
              Few few;
              std::memcpy(few.word, b.word, size_t(used) * sizeof few.word[0]);
              std::memcpy(few.rate, b.rate, size_t(rates) * sizeof few.rate[0]);
              std::memcpy(few.first, b.first, size_t(used) * sizeof few.first[0]);
              launch(few, used, blocks);
              launched = true;
            }
          }
          if (!launched) launch(b, used, blocks);
          used = rates = 0;
          blocks = 0;
          rc = done();
        };
        for (int32_t i = 0; i < count; ++i) {
          const acdc_adamw_tensor& t = tensors[i];
          if (t.n == 0 || class_of(t) != cls) continue;
          const Rate rate{float(double(t.lr) / c1), float(1.0 - double(t.lr) * double(t.weight_decay))};
          const long long need = (t.n + kChunk - 1) / kChunk;
          int k = 0;
          while (k < rates && !(b.rate[k].rate == rate.rate && b.rate[k].decay == rate.decay)) ++k;
          if (used == LIST::kMost || blocks + need > kMaxBlocks || k == kRates) {
            flush();
            if (rc != ACDC_OK) return;
            k = 0;
          }
          if (k == rates) b.rate[rates++] = rate;
          const void* p[kWords];
          addresses(t, p);
          b.put(used, p, (unsigned long long)t.n, int(blocks), k);
          ++used;
          blocks += need;
        }
        flush();
      };
      int of_class = 0;
      bool near = count > Long::kMost;
      uintptr_t low[kWords], high[kWords];
      for (int k = 0; k < kWords; ++k) low[k] = ~uintptr_t(0), high[k] = 0;
      for (int32_t i = 0; near && i < count; ++i) {
        const acdc_adamw_tensor& t = tensors[i];
        if (t.n == 0 || class_of(t) != cls) continue;
        ++of_class;
        near = near && t.n < 1ll << 29;
        const void* p[kWords];
        addresses(t, p);
        for (int k = 0; k < kWords; ++k) {
          const uintptr_t a = reinterpret_cast<uintptr_t>(p[k]);
          near = near && (a & ((1u << Near::shift(k)) - 1)) == 0;
          low[k] = a < low[k] ? a : low[k];
          high[k] = a > high[k] ? a : high[k];
        }
      }
      for (int k = 0; k < kWords; ++k) near = near && (high[k] - low[k]) >> Near::shift(k) >> 32 == 0;
      if (near && of_class > Long::kMost) {
        Near b;
        for (int k = 0; k < kWords; ++k) b.base[k] = low[k];
        all(b);
      } else {
        Long b;
        all(b);
      }
    });
  }
  return rc;
}

static long long norm_blocks(const int64_t* sizes, int32_t count) {
  const long long chunk = norm_chunk(sizes, count);
  long long blocks = 0;
  for (int32_t i = 0; i < count; ++i) blocks += (sizes[i] + chunk - 1) / chunk;
  return blocks;
}

extern "C" size_t acdc_grad_norm_workspace_size(const int64_t* sizes, int32_t count) {
  if (count < 0 || (count > 0 && sizes == nullptr)) return 0;
  for (int32_t i = 0; i < count; ++i)
    if (sizes[i] < 0 || sizes[i] > kMaxElements) return 0;
  return size_t(norm_blocks(sizes, count)) * sizeof(double);
}

extern "C" int acdc_grad_norm(const void* const* grads, const int64_t* sizes, const int32_t* types, int32_t count,
                              float max_norm, float* out, void* workspace, size_t workspace_bytes,
                              acdc_stream_t stream) {
  if (count < 0 || (count > 0 && (grads == nullptr || sizes == nullptr || types == nullptr))) return ACDC_ERR_INVALID_ARG;
  if (out == nullptr || !aligned_to(out, 4) || !aligned_to(workspace, 8) || max_norm != max_norm) return ACDC_ERR_INVALID_ARG;
  for (int32_t i = 0; i < count; ++i) {
    const size_t eb = dtype_bytes(types[i]);
    if (eb == 0 || sizes[i] < 0 || sizes[i] > kMaxElements) return ACDC_ERR_INVALID_ARG;
    if (sizes[i] > 0 && (grads[i] == nullptr || !aligned_to(grads[i], eb))) return ACDC_ERR_INVALID_ARG;
  }
  const long long total = norm_blocks(sizes, count), chunk = norm_chunk(sizes, count);
  if (total > 0 && (workspace == nullptr || workspace_bytes < size_t(total) * sizeof(double))) return ACDC_ERR_WORKSPACE;
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  double* sums = static_cast<double*>(workspace);
  NormBatch b;
  int used = 0;
  long long blocks = 0, at = 0;
  auto flush = [&]() -> int {
    if (used == 0) return ACDC_OK;
    hipLaunchKernelGGL(k_square_sums, dim3(static_cast<unsigned>(blocks)), dim3(kThreads), 0, st, b, used, int(chunk),
                       sums + at);
    at += blocks;
    used = 0;
    blocks = 0;
    return done();
  };
  for (int32_t i = 0; i < count; ++i) {
    if (sizes[i] == 0) continue;
    const long long need = (sizes[i] + chunk - 1) / chunk;
    if (used == kNormBatch || blocks + need > kMaxBlocks) {
      const int rc = flush();
      if (rc != ACDC_OK) return rc;
    }
    b.first[used] = int(blocks);
    b.t[used] = NormTensor{grads[i], (unsigned long long)sizes[i] << 1 | (types[i] == ACDC_BF16 ? 1u : 0u)};
    ++used;
    blocks += need;
  }
  int rc = flush();
  if (rc != ACDC_OK) return rc;
  hipLaunchKernelGGL(k_norm, dim3(1), dim3(kWide), 0, st, sums, total, max_norm, out);
  return done();
}
