// The vocabulary loss of a few rows (one drafted token, a handful of requests),
// forward and backward.  Contract: include/slim_lm.h.
//
// With N <= 8 (fp32) or 4 (bf16) the products are far below the memory traffic: w is read once and,
// backward, dw written once.  So the rows of x sit on the chip in fp32, w
// streams past them in 16-byte loads, and the products are fp32 FMA in either
// type: no staging, no split, g never rounded.
//
// A warp takes four words at a time, lanes across the features; its 4 N partial
// dot products are summed over the lanes by halving (31 shuffles for 32 of
// them), which leaves each lane with one logit.  One row of 512 against 32768
// words, bf16: 15 us forward (5 of them HBM's), 21 us backward (10); latency of
// the launches and of two rounds of words a warp bounds the rest.
#include <type_traits>

#include "lm_loss_rows.h"

#include "common.cuh"
#include "lm_loss_dev.cuh"
#include "profiler.h"

namespace slim {
namespace lm {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kWords = 4;            // of a warp at a time
constexpr int kTile = kWarps * kWords;
constexpr int kMaxRows = 8, kMaxElems = 16384;
constexpr int kFwdBlocks = 152 * 4, kBwdBlocks = 152 * 2;

struct Job {
  const void *x, *w, *targets;
  int i64, N, D, V;
  long long ignore;
  // forward
  float2* part;  // [blocks][kMaxRows]
  float* zt;     // [kMaxRows]
  unsigned* done;
  float *loss, *lse_out, *total;
  // backward
  const float *lse, *dloss, *count;
  int dstride;
  void *dw, *dx;
  float* dx_part;  // [blocks][N][D]
  int words;       // of a block
  int* header;     // the call's error word (nothing here waits)
};

// VB bytes of T as fp32.
template <typename T, int VB> struct Load;
template <> struct Load<float, 16> {
  static constexpr int n = 4;
  using raw = float4;
  static __device__ __forceinline__ void get(const float4& r, float* f) {
    f[0] = r.x;
    f[1] = r.y;
    f[2] = r.z;
    f[3] = r.w;
  }
  static __device__ __forceinline__ float4 put(const float* f) {
    return make_float4(f[0], f[1], f[2], f[3]);
  }
  static __device__ __forceinline__ float4 zero() { return make_float4(0.f, 0.f, 0.f, 0.f); }
};
template <> struct Load<float, 4> {
  static constexpr int n = 1;
  using raw = float;
  static __device__ __forceinline__ void get(float r, float* f) { f[0] = r; }
  static __device__ __forceinline__ float put(const float* f) { return f[0]; }
  static __device__ __forceinline__ float zero() { return 0.0f; }
};
template <> struct Load<__nv_bfloat16, 16> {
  static constexpr int n = 8;
  using raw = uint4;
  static __device__ __forceinline__ void get(const uint4& r, float* f) {
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
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
  static __device__ __forceinline__ uint4 zero() { return make_uint4(0, 0, 0, 0); }
};
template <> struct Load<__nv_bfloat16, 2> {
  static constexpr int n = 1;
  using raw = __nv_bfloat16;
  static __device__ __forceinline__ void get(__nv_bfloat16 r, float* f) {
    f[0] = __bfloat162float(r);
  }
  static __device__ __forceinline__ __nv_bfloat16 put(const float* f) {
    return __float2bfloat16_rn(f[0]);
  }
  static __device__ __forceinline__ __nv_bfloat16 zero() { return __float2bfloat16_rn(0.0f); }
};

// Features of a row in shared memory: whole warp steps of vectors, zero beyond D.
__host__ __device__ constexpr int padded(int D, int n) { return (D + 32 * n - 1) / (32 * n) * (32 * n); }

// The rows of x into shared memory as fp32; an ignored row (where targets say
// so) and rows past N as zero.
template <typename T, int n, int NT>
__device__ void load_rows(const Job& j, float* xs, bool drop_ignored) {
  const int P = padded(j.D, n);
  const T* x = static_cast<const T*>(j.x);
  for (int e = threadIdx.x; e < NT * P; e += kThreads) {
    const int r = e / P, d = e - r * P;
    bool on = r < j.N && d < j.D;
    if (on && drop_ignored) on = load_target(j.targets, j.i64, r) != j.ignore;
    xs[e] = on ? Io<T>::load(x, (size_t)r * j.D + d) : 0.0f;
  }
}

// Logits of words v0 .. v0+3 against all rows: the lane's is that of word
// (lane >> shift) / NT and row (lane >> shift) % NT, shift = 5 - log2(4 NT).
template <typename T, int VB, int NT>
__device__ __forceinline__ float dot_words(const Job& j, const float* xs, int v0) {
  using L = Load<T, VB>;
  constexpr int n = L::n, C = kWords * NT;
  const int lane = threadIdx.x & 31, U = j.D / n, P = padded(j.D, n);
  const T* w = static_cast<const T*>(j.w);
  float a[C];
#pragma unroll
  for (int i = 0; i < C; ++i) a[i] = 0.0f;
#pragma unroll 2
  for (int u0 = 0; u0 < U; u0 += 32) {
    const int u = u0 + lane;
    typename L::raw r[kWords];
#pragma unroll
    for (int k = 0; k < kWords; ++k)
      r[k] = u < U && v0 + k < j.V
                 ? *reinterpret_cast<const typename L::raw*>(w + (size_t)(v0 + k) * j.D + (size_t)u * n)
                 : L::zero();
    float f[kWords][n];
#pragma unroll
    for (int k = 0; k < kWords; ++k) L::get(r[k], f[k]);
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      float xv[n];
      const float* xp = xs + i * P + u * n;
      if constexpr (n % 4 == 0) {
#pragma unroll
        for (int e = 0; e < n; e += 4) Load<float, 16>::get(*reinterpret_cast<const float4*>(xp + e), xv + e);
      } else {
        xv[0] = xp[0];
      }
#pragma unroll
      for (int k = 0; k < kWords; ++k)
#pragma unroll
        for (int e = 0; e < n; ++e) a[k * NT + i] = fmaf(f[k][e], xv[e], a[k * NT + i]);
    }
  }
  int mask = 16;
#pragma unroll
  for (int h = C / 2; h >= 1; h >>= 1, mask >>= 1) {
    const bool up = lane & mask;
#pragma unroll
    for (int i = 0; i < h; ++i) {
      const float keep = up ? a[i + h] : a[i], give = up ? a[i] : a[i + h];
      a[i] = keep + __shfl_xor_sync(0xffffffffu, give, mask);
    }
  }
  for (; mask >= 1; mask >>= 1) a[0] += __shfl_xor_sync(0xffffffffu, a[0], mask);
  return a[0];
}

template <int NT> struct Shift {  // 5 - log2(4 NT)
  static constexpr int value = NT == 1 ? 3 : NT == 2 ? 2 : NT == 4 ? 1 : 0;
};

// ------------------------------------------------------------------ forward
template <typename T, int VB, int NT>
__global__ void __launch_bounds__(kThreads) k_rows_fwd(Job j) {
  constexpr int n = Load<T, VB>::n, shift = Shift<NT>::value;
  extern __shared__ float4 smem4[];
  float* xs = reinterpret_cast<float*>(smem4);
  __shared__ float2 st[kWarps][NT];
  __shared__ bool last;
  load_rows<T, n, NT>(j, xs, false);
  __syncthreads();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int slot = lane >> shift, row = slot % NT, word = slot / NT;
  int target = -1;
  if (row < j.N) {
    const long long t = load_target(j.targets, j.i64, row);
    if (t != j.ignore && t >= 0 && t < j.V) target = (int)t;
  }
  const bool owner = (lane & ((1 << shift) - 1)) == 0 && row < j.N;
  LogSum a;
  for (long long v = ((long long)blockIdx.x * kWarps + warp) * kWords; v < j.V;
       v += (long long)gridDim.x * kTile) {
    const float z = dot_words<T, VB, NT>(j, xs, (int)v);
    const int me = (int)v + word;
    if (owner && me < j.V) {
      if (me == target)
        j.zt[row] = z;
      else
        a.add(z * kLog2e, z == z ? 1.0f : z);  // a NaN stays one
    }
  }
  // lanes of the same row, then warps, then (by the block done last) blocks
#pragma unroll
  for (int o = 16; o >= NT << shift; o >>= 1)
    a.add(__shfl_xor_sync(0xffffffffu, a.base, o), __shfl_xor_sync(0xffffffffu, a.sum, o));
  if (owner && word == 0) st[warp][row] = make_float2(a.base, a.sum);
  __syncthreads();
  if (threadIdx.x < j.N) {
    LogSum b;
    for (int w = 0; w < kWarps; ++w) b.add(st[w][threadIdx.x].x, st[w][threadIdx.x].y);
    j.part[blockIdx.x * kMaxRows + threadIdx.x] = make_float2(b.base, b.sum);
  }
  __threadfence();
  __syncthreads();
  if (threadIdx.x == 0) last = atomicAdd(j.done, 1u) == gridDim.x - 1;
  __syncthreads();
  if (!last) return;
  __threadfence();
  __shared__ float2 res[kMaxRows];
  if (warp < j.N) {
    LogSum b;
    for (unsigned i = lane; i < gridDim.x; i += 32) {
      const float2 p = __ldcg(j.part + i * kMaxRows + warp);
      b.add(p.x, p.y);
    }
    for (int o = 16; o; o >>= 1)
      b.add(__shfl_xor_sync(0xffffffffu, b.base, o), __shfl_xor_sync(0xffffffffu, b.sum, o));
    if (lane == 0) {
      const long long t = load_target(j.targets, j.i64, warp);
      const float z = t >= 0 && t < j.V ? __ldcg(j.zt + warp) : 0.0f;
      float loss, lse;
      const bool counts = finish_loss(b, t, j.ignore, j.V, &z, loss, lse);
      j.loss[warp] = loss;
      j.lse_out[warp] = lse;
      res[warp] = make_float2(loss, counts ? 1.0f : 0.0f);
    }
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    float s = 0.0f, c = 0.0f;
    for (int i = 0; i < j.N; ++i) {
      s += res[i].x;
      c += res[i].y;
    }
    j.total[0] = s;
    j.total[1] = c;
  }
}

// ------------------------------------------------------------------ backward
// A block takes a run of words, kTile at a time: first the warps compute the
// tile's g (kept in shared memory, fp32), then every thread, which owns vectors
// of the features, adds g w to its part of dx (registers) and writes its part of
// dw = g^T x.  w's second read finds the tile in L1.
template <typename T, int VB, int NT>
__global__ void __launch_bounds__(kThreads) k_rows_bwd(Job j) {
  using L = Load<T, VB>;
  constexpr int n = L::n, shift = Shift<NT>::value;
  constexpr int CB = kMaxElems / kThreads / NT / n > 0 ? kMaxElems / kThreads / NT / n : 1;
  extern __shared__ float4 smem4[];
  float* xs = reinterpret_cast<float*>(smem4);
  __shared__ float gs[kTile][NT];
  if (blockIdx.x == 0 && threadIdx.x < 4) j.header[threadIdx.x] = 0;
  load_rows<T, n, NT>(j, xs, true);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int U = j.D / n, P = padded(j.D, n);
  const int slot = lane >> shift, row = slot % NT, word = slot / NT;
  // the lane's row
  int target = -1;
  float coef = 0.0f, lse = 0.0f;
  bool live = false;
  if (row < j.N) {
    const long long t = load_target(j.targets, j.i64, row);
    if (t != j.ignore) {
      live = true;
      lse = j.lse[row];
      coef = j.dloss[(size_t)row * j.dstride];
      if (j.count) coef = *j.count == 0.0f ? 0.0f : coef / *j.count;
      if (t >= 0 && t < j.V)
        target = (int)t;
      else
        coef = __int_as_float(0x7fffffff);
    }
  }
  // this thread's columns: vectors u, u + gw, ... of every word first, first + lanes, ...
  int gl = 0;
  while (gl < 8 && (1 << gl) < U) ++gl;
  const int gw = 1 << gl, wl = kThreads >> gl, u_me = threadIdx.x & (gw - 1),
            first = threadIdx.x >> gl;
  float dx[CB][NT][n];
#pragma unroll
  for (int c = 0; c < CB; ++c)
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
      for (int e = 0; e < n; ++e) dx[c][i][e] = 0.0f;
  const T* w = static_cast<const T*>(j.w);
  T* dw = static_cast<T*>(j.dw);
  const long long a = (long long)blockIdx.x * j.words;
  const int end = (int)(a + j.words < j.V ? a + j.words : j.V);
  for (int v0 = (int)a; v0 < end; v0 += kTile) {
    __syncthreads();
    const int mine = v0 + warp * kWords;
    if (mine < end) {
      const float z = dot_words<T, VB, NT>(j, xs, mine);
      if ((lane & ((1 << shift) - 1)) == 0) {
        float g = 0.0f;
        if (live) g = coef * (expf(z - lse) - (mine + word == target ? 1.0f : 0.0f));
        gs[warp * kWords + word][row] = g;
      }
    }
    __syncthreads();
    const int words = end - v0 < kTile ? end - v0 : kTile;
#pragma unroll
    for (int c = 0; c < CB; ++c) {
      const int u = u_me + c * gw;
      if (u >= U || (c > 0 && gw < kThreads)) break;
      float xv[NT][n];
#pragma unroll
      for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int e = 0; e < n; ++e) xv[i][e] = xs[i * P + u * n + e];
#pragma unroll 2
      for (int k = first; k < words; k += wl) {
        const size_t at = (size_t)(v0 + k) * j.D + (size_t)u * n;
        float f[n], o[n];
        L::get(*reinterpret_cast<const typename L::raw*>(w + at), f);
#pragma unroll
        for (int e = 0; e < n; ++e) o[e] = 0.0f;
#pragma unroll
        for (int i = 0; i < NT; ++i) {
          const float g = gs[k][i];
#pragma unroll
          for (int e = 0; e < n; ++e) {
            dx[c][i][e] = fmaf(g, f[e], dx[c][i][e]);
            o[e] = fmaf(g, xv[i][e], o[e]);
          }
        }
        *reinterpret_cast<typename L::raw*>(dw + at) = L::put(o);
      }
    }
  }
  // the block's dx: over the threads that share columns, in order
  __syncthreads();
#pragma unroll
  for (int c = 0; c < CB; ++c) {
    const int u = u_me + c * gw;
    if (c > 0 && gw < kThreads) break;
#pragma unroll
    for (int i = 0; i < NT; ++i) {
#pragma unroll
      for (int e = 0; e < n; ++e) {
        float s = dx[c][i][e];
        if (wl > 1) {
          xs[threadIdx.x] = s;
          __syncthreads();
          if (first == 0)
            for (int q = 1; q < wl; ++q) s += xs[q * gw + u_me];
          __syncthreads();
        }
        if (first == 0 && u < U && i < j.N)
          j.dx_part[((size_t)blockIdx.x * j.N + i) * j.D + (size_t)u * n + e] = s;
      }
    }
  }
}

// dx from the blocks' parts: 32 elements a block, eight threads each.
template <typename T>
__global__ void __launch_bounds__(kThreads) k_rows_dx(Job j, int blocks) {
  __shared__ float sh[8][32];
  const int col = threadIdx.x & 31, q = threadIdx.x >> 5;
  const long long e = (long long)blockIdx.x * 32 + col, total = (long long)j.N * j.D;
  float s = 0.0f;
  const int per = (blocks + 7) / 8, b1 = min((q + 1) * per, blocks);
  if (e < total) {
#pragma unroll 8
    for (int b = q * per; b < b1; ++b) s += j.dx_part[b * total + e];
  }
  sh[q][col] = s;
  __syncthreads();
  if (q == 0 && e < total) {
    for (int i = 1; i < 8; ++i) s += sh[i][col];
    const bool live = load_target(j.targets, j.i64, e / j.D) != j.ignore;
    Io<T>::store(static_cast<T*>(j.dx), e, live ? s : 0.0f);
  }
}

// ------------------------------------------------------------------ host
struct Ws {
  int* header;
  float2* part;
  float *zt, *dx_part;
};
int bwd_words(int V) {  // of a block: whole tiles
  const int tiles = (V + kTile - 1) / kTile;
  return (tiles + kBwdBlocks - 1) / kBwdBlocks * kTile;
}
int bwd_blocks(int V) { return (V + bwd_words(V) - 1) / bwd_words(V); }

Ws carve(Carver& cv, int N, int D, int V, bool bwd) {
  Ws w{};
  w.header = cv.take<int>(32);
  if (bwd) {
    w.dx_part = cv.take<float>((size_t)bwd_blocks(V) * N * D);
  } else {
    w.part = cv.take<float2>((size_t)kFwdBlocks * kMaxRows);
    w.zt = cv.take<float>(kMaxRows);
  }
  return w;
}

// Once per kernel and device (`flags` are the kernel's own): rows of up to
// kMaxElems floats, padded to a warp step each, fit this.
bool allow_smem(void (*kernel)(Job), bool (&flags)[kMaxDevices]) {
  bool* f = device_flag(flags);
  if (f && *f) return true;
  if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 96 * 1024) !=
      cudaSuccess)
    return false;
  if (f) *f = true;
  return true;
}

template <typename T, int VB, int NT>
slim_status run(const Job& j, bool bwd, cudaStream_t s) {
  constexpr int n = Load<T, VB>::n;
  size_t smem = (size_t)NT * padded(j.D, n) * sizeof(float);
  if (smem < kThreads * sizeof(float)) smem = kThreads * sizeof(float);
  const double bytes = (double)j.V * j.D * sizeof(T);
  if (!bwd) {
    static bool flags[kMaxDevices];
    if (!allow_smem(k_rows_fwd<T, VB, NT>, flags)) return SLIM_ERR_CUDA;
    // every block reads the rows of x again: no more blocks than are resident
    const int most = kFwdBlocks / (NT == 1 ? 1 : NT <= 4 ? 2 : 4);
    const int want = (j.V + kTile - 1) / kTile;
    prof::Scope ps(prof::K_LOSS_ROWS, s, 2.0 * j.N * j.D * j.V, bytes);
    k_rows_fwd<T, VB, NT><<<want < most ? want : most, kThreads, smem, s>>>(j);
    return cudaGetLastError() == cudaSuccess ? SLIM_OK : SLIM_ERR_CUDA;
  }
  static bool flags[kMaxDevices];
  if (!allow_smem(k_rows_bwd<T, VB, NT>, flags)) return SLIM_ERR_CUDA;
  const int blocks = bwd_blocks(j.V);
  {
    prof::Scope ps(prof::K_LOSS_ROWS, s, 6.0 * j.N * j.D * j.V, 2 * bytes);
    k_rows_bwd<T, VB, NT><<<blocks, kThreads, smem, s>>>(j);
    if (cudaGetLastError() != cudaSuccess) return SLIM_ERR_CUDA;
  }
  prof::Scope ps(prof::K_LOSS_ROWS, s);
  k_rows_dx<T><<<(unsigned)(((long long)j.N * j.D + 31) / 32), kThreads, 0, s>>>(j, blocks);
  return cudaGetLastError() == cudaSuccess ? SLIM_OK : SLIM_ERR_CUDA;
}

template <typename T, int VB>
slim_status by_rows(const Job& j, bool bwd, cudaStream_t s) {
  if (j.N == 1) return run<T, VB, 1>(j, bwd, s);
  if (j.N == 2) return run<T, VB, 2>(j, bwd, s);
  if constexpr (sizeof(T) == 4) {
    if (j.N > 4) return run<T, VB, 8>(j, bwd, s);
  }
  return run<T, VB, 4>(j, bwd, s);
}

slim_status dispatch(const Job& j, slim_dtype dtype, bool bwd, cudaStream_t s) {
  if (dtype == SLIM_F32)
    return j.D % 4 == 0 ? by_rows<float, 16>(j, bwd, s) : by_rows<float, 4>(j, bwd, s);
  return j.D % 8 == 0 ? by_rows<__nv_bfloat16, 16>(j, bwd, s)
                      : by_rows<__nv_bfloat16, 2>(j, bwd, s);
}

}  // namespace

// Measured against the tile kernels at nine rows (forward / backward, us): bf16,
// 512 x 32768, 3 rows 16.7/43 and 8 rows 20.7/86 here, 23.8/53 there; 1024 x
// 50000, 33/110 and 54/212 against 41/118.  fp32, which the tile kernels have to
// split first: 512 x 32768, 8 rows 24.7/82 here, 73.9/159 there.
bool rows_fit(long long N, int D, slim_dtype dtype) {
  if (N < 1 || N > (dtype == SLIM_BF16 ? kMaxRows / 2 : kMaxRows)) return false;
  const int nt = N == 1 ? 1 : N == 2 ? 2 : N <= 4 ? 4 : 8;
  return (long long)nt * D <= kMaxElems;
}

size_t rows_workspace(int N, int D, int V, bool bwd) {
  Carver cv(nullptr);
  carve(cv, N, D, V, bwd);
  return cv.bytes();
}

slim_status rows_fwd(const void* x, const void* w, const void* targets, slim_index it, int N, int D,
                     int V, slim_dtype dtype, long long ignore, float* loss, float* lse,
                     float* total, void* workspace, cudaStream_t s) {
  Carver cv(workspace);
  const Ws ws = carve(cv, N, D, V, false);
  if (cudaMemsetAsync(ws.header, 0, 32 * sizeof(int), s) != cudaSuccess) return SLIM_ERR_CUDA;
  Job j{};
  j.x = x;
  j.w = w;
  j.targets = targets;
  j.i64 = it == SLIM_I64;
  j.N = N;
  j.D = D;
  j.V = V;
  j.ignore = ignore;
  j.part = ws.part;
  j.zt = ws.zt;
  j.done = reinterpret_cast<unsigned*>(ws.header + 4);
  j.loss = loss;
  j.lse_out = lse;
  j.total = total;
  return dispatch(j, dtype, false, s);
}

slim_status rows_bwd(const void* x, const void* w, const void* targets, slim_index it,
                     const float* lse, const float* dloss, int dstride, const float* count, int N,
                     int D, int V, slim_dtype dtype, long long ignore, void* dx, void* dw,
                     void* workspace, cudaStream_t s) {
  Carver cv(workspace);
  const Ws ws = carve(cv, N, D, V, true);
  Job j{};
  j.x = x;
  j.w = w;
  j.targets = targets;
  j.i64 = it == SLIM_I64;
  j.N = N;
  j.D = D;
  j.V = V;
  j.ignore = ignore;
  j.lse = lse;
  j.dloss = dloss;
  j.count = count;
  j.dstride = dstride;
  j.dw = dw;
  j.dx = dx;
  j.dx_part = ws.dx_part;
  j.words = bwd_words(V);
  j.header = ws.header;
  return dispatch(j, dtype, true, s);
}

}  // namespace lm
}  // namespace slim
