// The gated feed-forward of a few rows (one decoding step of a handful of
// requests).  Contract: include/slim_layer.h.
//
// h = act(x w_gate^T) * (x w_up^T): w is read once, and the products are far below
// its traffic, in fp32 FMA for either type.  A warp takes one feature at a time, its
// lanes along D: both words and the rows of x arrive in 16-byte pieces that do not
// depend on each other, so a feature costs one trip to memory.  Its 2 N partial sums
// are added over the lanes by halving, which leaves each lane one of them.
#include <stdint.h>

#include <type_traits>

#include "common.cuh"
#include "launch.h"
#include "layer_ff.h"
#include "profiler.h"
#include "tc_common.cuh"

namespace slim {
namespace layer {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kMaxRows = 8;

// n elements of T at p as fp32; VEC: one 16-byte load.
template <typename T, bool VEC> struct Piece {
  static constexpr int n = VEC ? 16 / sizeof(T) : 1;
  static __device__ __forceinline__ void load(const T* p, bool on, float* f) {
    if constexpr (!VEC) {
      f[0] = on ? Io<T>::load(p, 0) : 0.0f;
    } else {
      const uint4 u = on ? *reinterpret_cast<const uint4*>(p) : make_uint4(0, 0, 0, 0);
      const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 4)
          f[i] = __uint_as_float(w[i]);
        else
          tc::unpack_bf16(w[i], f[2 * i], f[2 * i + 1]);
      }
    }
  }
};

template <typename T, bool VEC, int NT>
__global__ void __launch_bounds__(kThreads) k_ff_rows(const T* x, const T* w, int N, int D, int F,
                                                      int act, T* h) {
  using P = Piece<T, VEC>;
  constexpr int C = 2 * NT;
  const int lane = threadIdx.x & 31;
  const int warps = gridDim.x * kWarps;
  for (int f = blockIdx.x * kWarps + (threadIdx.x >> 5); f < F; f += warps) {
    float a[C];
#pragma unroll
    for (int i = 0; i < C; ++i) a[i] = 0.0f;
    const T* gate = w + (size_t)f * D;
    const T* up = w + ((size_t)F + f) * D;
#pragma unroll (NT <= 2 ? 4 : 2)
    for (long long d = (long long)lane * P::n; d < D; d += 32 * P::n) {
      float g[P::n], u[P::n], v[NT][P::n];
      P::load(gate + d, true, g);
      P::load(up + d, true, u);
#pragma unroll
      for (int r = 0; r < NT; ++r) P::load(x + (size_t)r * D + d, r < N, v[r]);
#pragma unroll
      for (int r = 0; r < NT; ++r)
#pragma unroll
        for (int e = 0; e < P::n; ++e) {
          a[r] = fmaf(g[e], v[r][e], a[r]);
          a[NT + r] = fmaf(u[e], v[r][e], a[NT + r]);
        }
    }
    int mask = 16;
#pragma unroll
    for (int k = C / 2; k >= 1; k >>= 1, mask >>= 1) {
      const bool high = lane & mask;
#pragma unroll
      for (int i = 0; i < k; ++i) {
        const float keep = high ? a[i + k] : a[i], give = high ? a[i] : a[i + k];
        a[i] = keep + __shfl_xor_sync(0xffffffffu, give, mask);
      }
    }
    for (; mask >= 1; mask >>= 1) a[0] += __shfl_xor_sync(0xffffffffu, a[0], mask);
    // the upper half of the lanes has the up sums, of the same rows in the same order
    const float other = __shfl_xor_sync(0xffffffffu, a[0], 16);
    constexpr int per = 32 / C;  // lanes of a row, in the lower half
    const int row = lane / per;
    if (lane < 16 && lane % per == 0 && row < N) {
      float v = 0.0f, none;
      with_act(act, [&](auto c) { activate<decltype(c)::value, false, false>(a[0], v, none); });
      Io<T>::store(h, (size_t)row * F + f, v * other);
    }
  }
}

template <typename T, bool VEC, int NT>
bool run(const void* x, const void* w, int N, int D, int F, int act, void* h, cudaStream_t s) {
  const int want = (F + kWarps - 1) / kWarps, most = 152 * 8;
  prof::Scope ps(prof::K_FF_ROWS, s, 4.0 * N * D * F, 2.0 * F * D * sizeof(T));
  k_ff_rows<T, VEC, NT><<<want < most ? want : most, kThreads, 0, s>>>(
      static_cast<const T*>(x), static_cast<const T*>(w), N, D, F, act, static_cast<T*>(h));
  return cudaGetLastError() == cudaSuccess;
}
template <typename T, bool VEC>
bool by_rows(const void* x, const void* w, int N, int D, int F, int act, void* h, cudaStream_t s) {
  if (N == 1) return run<T, VEC, 1>(x, w, N, D, F, act, h, s);
  if (N == 2) return run<T, VEC, 2>(x, w, N, D, F, act, h, s);
  if (N <= 4) return run<T, VEC, 4>(x, w, N, D, F, act, h, s);
  return run<T, VEC, 8>(x, w, N, D, F, act, h, s);
}

}  // namespace

// fp32, up to eight rows: 512 x 2048, 8 rows 16 us (tiles 24), 2048 x 8192 79 (134).  bf16,
// where the FMAs stay below the tiles' time: 512 x 2048, 8 rows 11 us (tiles 14), 2048 x
// 8192, 4 rows 34 and 8 rows 57 (tiles 30).
bool ff_rows_fit(long long N, int D, int F, slim_dtype dtype) {
  if (N < 1 || N > kMaxRows) return false;
  return dtype == SLIM_F32 || N == 1 || (double)N * D * F <= 0x1p25;
}

slim_status ff_rows_fwd(const void* x, const void* w, int N, int D, int F, slim_dtype dtype,
                        slim_act act, void* h, cudaStream_t s) {
  using B = __nv_bfloat16;
  const bool ok = dtype == SLIM_F32
                      ? (D % 4 == 0 ? by_rows<float, true>(x, w, N, D, F, act, h, s)
                                    : by_rows<float, false>(x, w, N, D, F, act, h, s))
                      : (D % 8 == 0 ? by_rows<B, true>(x, w, N, D, F, act, h, s)
                                    : by_rows<B, false>(x, w, N, D, F, act, h, s));
  return ok ? SLIM_OK : SLIM_ERR_CUDA;
}

}  // namespace layer
}  // namespace slim
