// The global norm of many gradients, and their clipping by it.  Contract:
// include/slim_lm.h.
//
//   norm = sqrt(sum g^2),  out = min(1, max_norm / norm) * g
//
// Two launches: one reads every gradient and leaves one partial sum per block,
// one adds the partial sums (every block all of them, in the same order),
// scales and writes.  HBM bounds both; a set that fits L2 is read from HBM once,
// and of a larger set the second launch starts with the end, which L2 still
// holds.  The tensors' addresses travel as kernel parameters: no copy and no
// device table.  279 M fp32 gradients into a second list: 505-516 us, of which
// the norm 165 (6.8 TB/s) and the scaling 340 (6.5 TB/s read and written).
//
// Range: a thread adds the squares of 64 to 128 elements in fp32 and moves the
// sum to fp64.  Squares leave fp32's range long before the gradients do, so a
// thread whose sum overflowed, or is so small that it may have lost squares to
// underflow, takes its elements again scaled by a power of two, which fits
// every value of the types.
#include <float.h>
#include <stdint.h>

#include <type_traits>

#include "../../include/slim_lm.h"
#include "common.cuh"
#include "launch.h"
#include "profiler.h"
#include "tc_common.cuh"

namespace slim {
namespace lm {
namespace {

constexpr int kThreads = 256;
// Blocks of either launch.  1.1 GB of fp32, eight 16-byte loads in flight a
// thread: the norm reads 6.75 TB/s with four blocks an SM and 6.5 with eight, the
// scaling moves 6.1 and 6.5 (with four loads in flight 6.2 and 6.3 at eight).
constexpr int kGridNorm = 152 * 4, kGridClip = 152 * 8;
// Bytes of one tensor that a block takes at a time: large enough to keep every
// thread's loads going (16 KB: 3 % slower at 1.1 GB), smaller where the whole list
// would leave blocks idle (26 gradients of 4.3 MB in all: 16.2 -> 14.5 us).
constexpr int kChunkMost = 65536, kChunkLeast = 4096;

// A launch's tensors.  Tensor t's chunks are numbered [start[t], start[t+1]); they
// begin at its first 128-byte boundary (of the source for the norm, of the target
// for the scaling), and the first one also takes the elements before that: a
// warp's 512 bytes then cover whole lines, and no chunk but a tensor's last leaves
// a few threads with loads of their own.
template <int CAP>
struct Table {
  const void* src[CAP];
  void* dst[CAP];
  unsigned long long numel[CAP];  // bit 63: bf16
  unsigned start[CAP + 1];
  int n;
  int chunk;  // bytes
};
constexpr unsigned long long kBf16Bit = 1ull << 63;

template <int CAP>
__device__ __forceinline__ int find_tensor(const Table<CAP>& tb, unsigned chunk) {
  int lo = 0, hi = tb.n;  // start[lo] <= chunk < start[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (tb.start[mid] <= chunk)
      lo = mid;
    else
      hi = mid;
  }
  return lo;
}

// 16 bytes of T as fp32 values.
template <typename T> struct Pack;
template <> struct Pack<float> {
  static constexpr int n = 4;
  static __device__ __forceinline__ void get(const uint4& u, float* f) {
    f[0] = __uint_as_float(u.x);
    f[1] = __uint_as_float(u.y);
    f[2] = __uint_as_float(u.z);
    f[3] = __uint_as_float(u.w);
  }
  static __device__ __forceinline__ uint4 put(const float* f) {
    return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]),
                      __float_as_uint(f[3]));
  }
};
template <> struct Pack<__nv_bfloat16> {
  static constexpr int n = 8;
  static __device__ __forceinline__ void get(const uint4& u, float* f) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = __uint_as_float(w[i] << 16);
      f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ uint4 put(const float* f) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
};

// Elements of 2^ls bytes from address p to its next 128-byte boundary, at most n.
__host__ __device__ __forceinline__ long long to_line(const void* p, long long n, int ls) {
  const long long lead = (long long)(-(intptr_t)p & 127) >> ls;
  return lead < n ? lead : n;
}

// A chunk: elements [at, at + m) of the tensor, and [0, lead) beside them.
struct Chunk {
  long long at, m, lead;
};
template <int CAP>
__device__ __forceinline__ Chunk find_chunk(const Table<CAP>& tb, int t, unsigned chunk,
                                            const void* p, long long n, int ls) {
  const long long per = tb.chunk >> ls, lead = to_line(p, n, ls);
  const long long x = chunk - tb.start[t], a = x * per;
  const long long left = n - lead - a;
  return Chunk{lead + a, left < per ? left : per, x == 0 ? lead : 0};
}

// ------------------------------------------------------------------ norm
// Thresholds of a thread's fp32 sum of squares.  Above kTiny, squares lost to
// underflow (each below 2^-126) are below its rounding; at or under it every
// element is below 2^-40, and 2^96 lifts the smallest subnormal's square into
// the normal range without overflow.
constexpr float kTiny = 0x1p-80f;

template <typename T>
__device__ __forceinline__ float square_sum(const T* p, const Chunk& c, float scale,
                                            unsigned& any) {
  constexpr int W = Pack<T>::n;
  float s = 0.0f;
  const uint4* v = reinterpret_cast<const uint4*>(p + c.at);
  const long long nvec = c.m / W;
  long long i = threadIdx.x;
  auto take = [&](const uint4& u) {
    any |= (u.x | u.y | u.z | u.w);
    float f[W];
    Pack<T>::get(u, f);
#pragma unroll
    for (int e = 0; e < W; ++e) {
      const float x = f[e] * scale;
      s = fmaf(x, x, s);
    }
  };
  for (; i + 7 * kThreads < nvec; i += 8 * kThreads) {
    uint4 u[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) u[j] = v[i + j * kThreads];
#pragma unroll
    for (int j = 0; j < 8; ++j) take(u[j]);
  }
  for (; i < nvec; i += kThreads) take(v[i]);
  // the elements before the first line and after the last 16 bytes
  auto one = [&](long long k) {
    const float x = Io<T>::load(p, k) * scale;
    any |= x != 0.0f;
    s = fmaf(x, x, s);
  };
  if (threadIdx.x < c.lead) one(threadIdx.x);
  if (nvec * W + threadIdx.x < c.m) one(c.at + nvec * W + threadIdx.x);
  return s;
}

// Once more, scaled; out of line, as it hardly ever runs.
template <typename T>
__device__ __noinline__ double scaled_squares(const T* p, long long at, long long m,
                                              long long lead, bool up) {
  unsigned any = 0;
  const double s = (double)square_sum<T>(p, Chunk{at, m, lead}, up ? 0x1p96f : 0x1p-96f, any);
  return s * (up ? 0x1p-192 : 0x1p192);
}
template <typename T>
__device__ __forceinline__ double chunk_squares(const T* p, const Chunk& c) {
  unsigned any = 0;
  const float s = square_sum<T>(p, c, 1.0f, any);
  if (s >= kTiny && s <= FLT_MAX) return (double)s;
  const bool up = s < kTiny;  // else an overflow, an infinity or NaN
  if (up && (any << 1) == 0) return 0.0;  // nothing but zeros
  return scaled_squares<T>(p, c.at, c.m, c.lead, up);
}

// Sum of x over the block, in a fixed order, for thread 0.  By one warp: fp64
// runs at two lanes a clock, and every thread adding up cost more than the loads.
__device__ __forceinline__ double block_sum(double x, double* sh) {
  sh[threadIdx.x] = x;
  __syncthreads();
  double t = 0.0;
  if (threadIdx.x < 32) {
#pragma unroll
    for (int i = 0; i < kThreads / 32; ++i) t += sh[threadIdx.x + 32 * i];
    for (int o = 16; o; o >>= 1) t += __shfl_xor_sync(0xffffffffu, t, o);
  }
  return t;
}

template <int CAP>
__global__ void __launch_bounds__(kThreads) k_norm(const __grid_constant__ Table<CAP> tb,
                                                   double* part, int* header) {
  __shared__ double sh[kThreads];
  tc::grid_dependency_wait();
  if (header && blockIdx.x == 0 && threadIdx.x < 4) header[threadIdx.x] = 0;
  double acc = 0.0;
  const unsigned total = tb.start[tb.n];
  for (unsigned c = blockIdx.x; c < total; c += gridDim.x) {
    const int t = find_tensor(tb, c);
    const bool half = tb.numel[t] & kBf16Bit;
    const long long n = (long long)(tb.numel[t] & ~kBf16Bit);
    const Chunk ch = find_chunk(tb, t, c, tb.src[t], n, half ? 1 : 2);
    if (half)
      acc += chunk_squares(static_cast<const __nv_bfloat16*>(tb.src[t]), ch);
    else
      acc += chunk_squares(static_cast<const float*>(tb.src[t]), ch);
  }
  const double s = block_sum(acc, sh);
  if (threadIdx.x == 0) part[blockIdx.x] = s;
}

// ------------------------------------------------------------------ clip
// Bytes k .. k+15 of the 32 bytes (a, b), k = 4 W + r / 8.
template <int W>
__device__ __forceinline__ uint4 shifted(const uint4& a, const uint4& b, unsigned r) {
  const uint32_t c[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
  return make_uint4(__funnelshift_r(c[W], c[W + 1], r), __funnelshift_r(c[W + 1], c[W + 2], r),
                    __funnelshift_r(c[W + 2], c[W + 3], r), __funnelshift_r(c[W + 3], c[W + 4], r));
}

// max_norm / norm as the product of two, a step each: below fp32's normal range
// it would lose its digits (1e38 clipped to 1e-3: 13 bits of them left).
struct Factor {
  float a, b;
  __device__ __forceinline__ float operator()(float x) const { return x * a * b; }
};
__device__ __forceinline__ Factor make_factor(double f) {
  if (f >= 0x1p-126) return Factor{(float)f, 1.0f};
  return Factor{(float)(f * 0x1p126), 0x1p-126f};
}

template <typename T>
__device__ __forceinline__ void scale_chunk(const T* p, T* q, const Chunk& ch, const Factor& c) {
  constexpr int W = Pack<T>::n;
  const long long nvec = ch.m / W;
  uint4* o = reinterpret_cast<uint4*>(q + ch.at);
  auto put = [&](const uint4& u) {
    float f[W];
    Pack<T>::get(u, f);
#pragma unroll
    for (int e = 0; e < W; ++e) f[e] = c(f[e]);
    return Pack<T>::put(f);
  };
  // the source may lie otherwise: then every 16 bytes come from the two aligned
  // pieces that hold them (each holds some, so neither leaves the buffer)
  const uintptr_t src = reinterpret_cast<uintptr_t>(p + ch.at);
  const unsigned k = (unsigned)(src & 15u);
  const uint4* v = reinterpret_cast<const uint4*>(src - k);
  long long i = threadIdx.x;
  if (k == 0) {
    for (; i + 7 * kThreads < nvec; i += 8 * kThreads) {
      uint4 u[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) u[j] = v[i + j * kThreads];
#pragma unroll
      for (int j = 0; j < 8; ++j) o[i + j * kThreads] = put(u[j]);
    }
    for (; i < nvec; i += kThreads) o[i] = put(v[i]);
  } else {
    const unsigned r = (k & 3u) * 8;
    auto all = [&](auto word) {
      constexpr int w = decltype(word)::value;
      for (; i + 3 * kThreads < nvec; i += 4 * kThreads) {
        uint4 a[4], b[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          a[j] = v[i + j * kThreads];
          b[j] = v[i + j * kThreads + 1];
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) o[i + j * kThreads] = put(shifted<w>(a[j], b[j], r));
      }
      for (; i < nvec; i += kThreads) o[i] = put(shifted<w>(v[i], v[i + 1], r));
    };
    switch (k >> 2) {
      case 0: all(std::integral_constant<int, 0>()); break;
      case 1: all(std::integral_constant<int, 1>()); break;
      case 2: all(std::integral_constant<int, 2>()); break;
      default: all(std::integral_constant<int, 3>()); break;
    }
  }
  if (threadIdx.x < ch.lead) Io<T>::store(q, threadIdx.x, c(Io<T>::load(p, threadIdx.x)));
  if (nvec * W + threadIdx.x < ch.m) {
    const long long k = ch.at + nvec * W + threadIdx.x;
    Io<T>::store(q, k, c(Io<T>::load(p, k)));
  }
}

template <int CAP>
__global__ void __launch_bounds__(kThreads) k_clip(const __grid_constant__ Table<CAP> tb,
                                                   const double* part, int parts, float max_norm,
                                                   int in_place, float* norm_out) {
  __shared__ Factor factor;
  tc::grid_dependency_wait();
  if (threadIdx.x < 32) {
    double acc = 0.0;
    for (int i = threadIdx.x; i < parts; i += 32) acc += part[i];
    for (int o = 16; o; o >>= 1) acc += __shfl_xor_sync(0xffffffffu, acc, o);
    if (threadIdx.x == 0) {
      const double norm = sqrt(acc);
      const float told = (float)norm;
      if (norm_out && blockIdx.x == 0) *norm_out = told;
      // a norm that is not finite scales nothing: the one that the caller reads,
      // which overflows before the sum in fp64 does
      factor = make_factor(norm > (double)max_norm && told <= FLT_MAX ? (double)max_norm / norm : 1.0);
    }
  }
  __syncthreads();
  const Factor c = factor;
  if (c.a * c.b == 1.0f && in_place) return;
  const unsigned total = tb.start[tb.n];
  for (unsigned x = blockIdx.x; x < total; x += gridDim.x) {
    const unsigned chunk = total - 1 - x;  // the end first: L2 holds what was read last
    const int t = find_tensor(tb, chunk);
    const bool half = tb.numel[t] & kBf16Bit;
    const long long n = (long long)(tb.numel[t] & ~kBf16Bit);
    const Chunk ch = find_chunk(tb, t, chunk, tb.dst[t], n, half ? 1 : 2);
    if (half)
      scale_chunk(static_cast<const __nv_bfloat16*>(tb.src[t]),
                  static_cast<__nv_bfloat16*>(tb.dst[t]), ch, c);
    else
      scale_chunk(static_cast<const float*>(tb.src[t]), static_cast<float*>(tb.dst[t]), ch, c);
  }
}

// ------------------------------------------------------------------ host
// Kernel parameters hold at most 4 KB on the short path and 32,764 bytes on
// the long one; longer lists take several launches of the latter.
constexpr int kSmall = 128, kLarge = 1024;
static_assert(sizeof(Table<kSmall>) <= 3900 && sizeof(Table<kLarge>) <= 32000, "parameters");

struct List {
  const void* const* src;
  void* const* dst;
  const long long* numel;
  const slim_dtype* dtypes;
  int n;
};

// Tensors [a, ..) of the list, as many as fit; returns the next one that is not
// empty (or n): only a list without elements makes a launch without tensors, and
// the launches that leave partial sums are those that the workspace counts.  The
// chunks begin where `by_dst` says.
template <int CAP>
int fill(const List& l, int a, bool by_dst, Table<CAP>* tb, bool* in_place, double* bytes) {
  tb->n = 0;
  unsigned long long chunks = 0;
  *in_place = true;
  *bytes = 0.0;
  int t = a;
  for (; t < l.n && tb->n < CAP; ++t) {
    if (l.numel[t] == 0) continue;
    const bool half = l.dtypes[t] == SLIM_BF16;
    const int ls = half ? 1 : 2;
    const long long per = tb->chunk >> ls;
    const long long body = l.numel[t] - to_line(by_dst ? l.dst[t] : l.src[t], l.numel[t], ls);
    const int i = tb->n++;
    tb->src[i] = l.src[t];
    tb->dst[i] = l.dst[t];
    tb->numel[i] = (unsigned long long)l.numel[t] | (half ? kBf16Bit : 0);
    tb->start[i] = (unsigned)chunks;
    chunks += body > 0 ? (unsigned long long)((body + per - 1) / per) : 1;
    if (l.src[t] != l.dst[t]) *in_place = false;
    *bytes += (double)l.numel[t] * (half ? 2 : 4);
  }
  while (t < l.n && l.numel[t] == 0) ++t;
  tb->start[tb->n] = (unsigned)chunks;
  return t;
}

template <int CAP>
slim_status run(const List& l, float max_norm, float* norm, int* header, double* part,
                cudaStream_t s) {
  static_assert(sizeof(Table<CAP>) < 32764, "kernel parameters");
  Table<CAP> tb;
  tb.n = 0;
  tb.start[0] = 0;
  double all = 0.0;
  for (int t = 0; t < l.n; ++t) all += (double)l.numel[t] * (l.dtypes[t] == SLIM_BF16 ? 2 : 4);
  tb.chunk = kChunkMost;
  while (tb.chunk > kChunkLeast && all / tb.chunk < 2 * kGridClip) tb.chunk >>= 1;
  bool in_place;
  double bytes;
  int parts = 0;
  auto grid = [&](unsigned most) {
    const unsigned c = tb.start[tb.n];
    return c < 1 ? 1u : c < most ? c : most;
  };
  int a = 0;
  do {
    a = fill(l, a, false, &tb, &in_place, &bytes);
    prof::Scope ps(prof::K_CLIP, s, 0.0, bytes);
    if (!launch_on<Table<CAP>, double*, int*>(k_norm<CAP>, grid(kGridNorm), kThreads, 0, 1, parts > 0, s, tb,
                                              part + parts, parts == 0 ? header : nullptr))
      return SLIM_ERR_CUDA;
    parts += (int)grid(kGridNorm);
  } while (a < l.n);
  a = 0;
  bool first = true;
  do {
    a = fill(l, a, true, &tb, &in_place, &bytes);
    prof::Scope ps(prof::K_CLIP, s, 0.0, bytes);
    if (!launch_on<Table<CAP>, const double*, int, float, int, float*>(
            k_clip<CAP>, grid(kGridClip), kThreads, 0, 1, true, s, tb, part, parts, max_norm, in_place,
            first ? norm : nullptr))
      return SLIM_ERR_CUDA;
    first = false;
  } while (a < l.n);
  return SLIM_OK;
}

}  // namespace
}  // namespace lm
}  // namespace slim

extern "C" slim_status slim_clip_workspace_size(int n, size_t* bytes) {
  if (!bytes || n < 0) return SLIM_ERR_INVALID_ARG;
  slim::Carver cv(nullptr);
  cv.take<int>(4);
  const size_t groups = n == 0 ? 1 : ((size_t)n + slim::lm::kLarge - 1) / slim::lm::kLarge;
  cv.take<double>(groups * slim::lm::kGridNorm);
  *bytes = cv.bytes();
  return SLIM_OK;
}

extern "C" slim_status slim_clip_grads(const void* const* src, void* const* dst,
                                       const long long* numel, const slim_dtype* dtypes, int n,
                                       float max_norm, float* norm, void* workspace,
                                       size_t workspace_bytes, void* stream) {
  using namespace slim::lm;
  if (n < 0 || !(max_norm > 0.0f) || !norm || (reinterpret_cast<uintptr_t>(norm) & 3u))
    return SLIM_ERR_INVALID_ARG;
  if (n > 0 && (!src || !dst || !numel || !dtypes)) return SLIM_ERR_INVALID_ARG;
  long long total = 0;
  int live = 0;
  for (int t = 0; t < n; ++t) {
    if (dtypes[t] != SLIM_F32 && dtypes[t] != SLIM_BF16) return SLIM_ERR_INVALID_ARG;
    if (numel[t] < 0 || numel[t] > (1LL << 40)) return SLIM_ERR_INVALID_ARG;
    if (numel[t] == 0) continue;
    const uintptr_t mask = dtypes[t] == SLIM_BF16 ? 1 : 3;
    if (!src[t] || !dst[t] || (reinterpret_cast<uintptr_t>(src[t]) & mask) ||
        (reinterpret_cast<uintptr_t>(dst[t]) & mask))
      return SLIM_ERR_INVALID_ARG;
    total += numel[t];
    ++live;
    if (total > (1LL << 42)) return SLIM_ERR_INVALID_ARG;  // chunk numbers fit 32 bits
  }
  size_t need = 0;
  slim_clip_workspace_size(n, &need);
  if (workspace == nullptr || workspace_bytes < need) return SLIM_ERR_WORKSPACE;
  if (reinterpret_cast<uintptr_t>(workspace) & 255u) return SLIM_ERR_INVALID_ARG;
  slim::Carver cv(workspace);
  int* header = cv.take<int>(4);  // the call's error word (no kernel here waits)
  double* part = cv.take<double>(0);
  const List l{src, dst, numel, dtypes, n};
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (live <= kSmall) return run<kSmall>(l, max_norm, norm, header, part, s);
  return run<kLarge>(l, max_norm, norm, header, part, s);
}
