// Gated linear recurrence over long sequences, and its gradients.  Contract:
// include/slim_layer.h.
//
//     h_t = a_t h_(t-1) + u_t            per channel
//     r_t = a_t g_t,  g_t = dh_t + r_(t+1)    backward: the same from the other end
//
// A chunk of kChunk steps takes a state to A state + H.  First every chunk's (A, H)
// is computed on its own, then the states between chunks by one pass over those, and
// then each chunk runs from its state.  The order of every sum is fixed by the sizes.
//
// Backward, dgate needs h_(t-1): the forward keeps the states between chunks in fp32
// (1 / 16 the values of h), and a chunk's states are computed again from there.
#include <math.h>
#include <stdint.h>

#include "../../include/slim_layer.h"
#include "common.cuh"
#include "launch.h"
#include "profiler.h"
#include "tc_common.cuh"

namespace slim {
namespace layer {
namespace {

constexpr int kChunk = SLIM_SCAN_CHUNK;
constexpr int kThreads = 128;
constexpr int kSub = 8;  // steps held in registers at a time

struct Job {
  const void *gate, *x, *dh;
  long long gate_pitch, x_pitch;
  const float* enter;  // forward: h0, backward: dlast; or null (zero)
  const float* kept;   // backward: states before each chunk
  void *h, *dgate, *dx;
  long long dgate_pitch, dx_pitch;
  float* leave;        // forward: last state, backward: dh0; or null
  float* states;       // [B][chunks][D]: what enters each chunk (from its running end)
  float2* sums;        // [B][chunks][D]: the chunks' (A, H)
  int B, L, D, chunks;
};

// a and u of a step, from the gate and x; and the gate's gradient.
template <int KIND> struct Gate {
  static __device__ __forceinline__ void split(float g, float& a, float& b) {
    if (KIND == SLIM_GATE_SIGMOID) {
      // sigmoid(g) and sigmoid(-g), each to its own digits
      const float e = expf(-fabsf(g)), big = 1.0f / (1.0f + e), small = e * big;
      a = g >= 0.0f ? big : small;
      b = g >= 0.0f ? small : big;
      if (g != g) a = b = g;
    } else {
      a = KIND == SLIM_GATE_LOG ? expf(g) : g;
      b = 1.0f;
    }
  }
  static __device__ __forceinline__ float u(float b, float x) {
    return KIND == SLIM_GATE_SIGMOID ? b * x : x;
  }
  // d loss / d gate from g = d loss / d h_t and the state before the step
  static __device__ __forceinline__ float grad(float g, float a, float b, float before, float x) {
    if (KIND == SLIM_GATE_VALUE) return g * before;
    if (a == 0.0f) return 0.0f;  // whatever the state that it forgot
    return KIND == SLIM_GATE_LOG ? g * before * a : g * (before - x) * (a * b);
  }
};

// a s + u; a gate of zero forgets a state that is not finite, too.
__device__ __forceinline__ float step(float a, float s, float u) { return a == 0.0f ? u : fmaf(a, s, u); }

template <typename T, int V> struct Vec {
  static __device__ __forceinline__ void load(const T* p, float* v) {
    if constexpr (V == 1) {
      v[0] = Io<T>::load(p, 0);
    } else if constexpr (sizeof(T) == 4) {
      const float4 u = *reinterpret_cast<const float4*>(p);
      v[0] = u.x;
      v[1] = u.y;
      v[2] = u.z;
      v[3] = u.w;
    } else {
      const uint2 u = *reinterpret_cast<const uint2*>(p);
      tc::unpack_bf16(u.x, v[0], v[1]);
      tc::unpack_bf16(u.y, v[2], v[3]);
    }
  }
  static __device__ __forceinline__ void store(T* p, const float* v) {
    if constexpr (V == 1)
      Io<T>::store(p, 0, v[0]);
    else if constexpr (sizeof(T) == 4)
      *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
    else
      *reinterpret_cast<uint2*>(p) =
          make_uint2(tc::pack_bf16(v[0], v[1]), tc::pack_bf16(v[2], v[3]));
  }
};

// A thread has V channels of one chunk of one sequence.
struct Place {
  int c, chunk, b, t0, n;
  bool on;
};
template <int V>
__device__ __forceinline__ Place place(const Job& j) {
  Place p;
  const long long per = (j.D + V - 1) / V, i = (long long)blockIdx.x * kThreads + threadIdx.x;
  const long long row = i / per;
  p.c = (int)(i - row * per) * V;
  p.on = row < (long long)j.B * j.chunks;
  p.b = (int)(row / j.chunks);
  p.chunk = (int)(row - (long long)p.b * j.chunks);
  p.t0 = p.chunk * kChunk;
  p.n = min(kChunk, j.L - p.t0);
  return p;
}
__device__ __forceinline__ size_t at_row(const Job& j, const Place& p, int t) {
  return (size_t)p.b * j.L + p.t0 + t;
}

// ------------------------------------------------------------------ chunks' sums
template <typename T, int V, int KIND, bool BWD>
__global__ void __launch_bounds__(kThreads) k_scan_sums(const __grid_constant__ Job j) {
  const Place p = place<V>(j);
  if (!p.on) return;
  using W = Vec<T, V>;
  float A[V], H[V];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    A[v] = 1.0f;
    H[v] = 0.0f;
  }
  auto one = [&](const float* g, const float* x) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      float a, b;
      Gate<KIND>::split(g[v], a, b);
      // backward x is dh, which enters ahead of the gate
      H[v] = BWD ? (a == 0.0f ? 0.0f : a * (x[v] + H[v])) : step(a, H[v], Gate<KIND>::u(b, x[v]));
      A[v] *= a;
    }
  };
  const T* gate = static_cast<const T*>(j.gate) + p.c;
  const T* x = static_cast<const T*>(BWD ? j.dh : j.x) + p.c;
  const long long xp = BWD ? j.D : j.x_pitch;
  for (int s = 0; s < p.n; s += kSub) {
    float g[kSub][V], y[kSub][V];
#pragma unroll
    for (int k = 0; k < kSub; ++k) {
      const int t = BWD ? p.n - 1 - (s + k) : s + k;
      if (s + k < p.n) {
        W::load(gate + at_row(j, p, t) * j.gate_pitch, g[k]);
        W::load(x + at_row(j, p, t) * xp, y[k]);
      }
    }
#pragma unroll
    for (int k = 0; k < kSub; ++k)
      if (s + k < p.n) one(g[k], y[k]);
  }
  float2* to = j.sums + ((size_t)p.b * j.chunks + p.chunk) * j.D + p.c;
#pragma unroll
  for (int v = 0; v < V; ++v) to[v] = make_float2(A[v], H[v]);
}

// ------------------------------------------------------------------ states between chunks
// 32 channels a block, kSegs threads each: a thread takes its chunks' sums together,
// the threads' are joined in order, and each writes the states of its own.
constexpr int kSegs = 16;
__global__ void __launch_bounds__(32 * kSegs) k_scan_states(const __grid_constant__ Job j, int back) {
  tc::grid_dependency_wait();
  __shared__ float2 part[kSegs][32];
  const int lane = threadIdx.x & 31, seg = threadIdx.x >> 5;
  const int c = blockIdx.x * 32 + lane, b = blockIdx.y;
  const int per = (j.chunks + kSegs - 1) / kSegs, i0 = seg * per, i1 = min(i0 + per, j.chunks);
  const size_t base = (size_t)b * j.chunks * j.D + c;
  auto at = [&](int i) { return base + (size_t)(back ? j.chunks - 1 - i : i) * j.D; };
  float A = 1.0f, H = 0.0f;
  if (c < j.D) {
#pragma unroll 8
    for (int i = i0; i < i1; ++i) {
      const float2 s = j.sums[at(i)];
      H = step(s.x, H, s.y);
      A *= s.x;
    }
  }
  part[seg][lane] = make_float2(A, H);
  __syncthreads();
  if (c >= j.D) return;
  float s = j.enter ? j.enter[(size_t)b * j.D + c] : 0.0f;
  for (int k = 0; k < seg; ++k) s = step(part[k][lane].x, s, part[k][lane].y);
#pragma unroll 8
  for (int i = i0; i < i1; ++i) {
    const float2 f = j.sums[at(i)];
    j.states[at(i)] = s;
    s = step(f.x, s, f.y);
  }
}

// ------------------------------------------------------------------ the chunks themselves
template <int V>
__device__ __forceinline__ void enter(const Job& j, const Place& p, float* s) {
  const float* from = j.chunks > 1 ? j.states + ((size_t)p.b * j.chunks + p.chunk) * j.D + p.c
                      : j.enter    ? j.enter + (size_t)p.b * j.D + p.c
                                   : nullptr;
#pragma unroll
  for (int v = 0; v < V; ++v) s[v] = from ? from[v] : 0.0f;
}

template <typename T, int V, int KIND>
__global__ void __launch_bounds__(kThreads) k_scan_fwd(const __grid_constant__ Job j) {
  tc::grid_dependency_wait();
  const Place p = place<V>(j);
  if (!p.on) return;
  using W = Vec<T, V>;
  float h[V];
  enter<V>(j, p, h);
  if (j.chunks == 1 && j.states)
#pragma unroll
    for (int v = 0; v < V; ++v) j.states[(size_t)p.b * j.D + p.c + v] = h[v];
  const T* gate = static_cast<const T*>(j.gate) + p.c;
  const T* x = static_cast<const T*>(j.x) + p.c;
  T* out = static_cast<T*>(j.h) + p.c;
  for (int s = 0; s < p.n; s += kSub) {
    float g[kSub][V], y[kSub][V];
#pragma unroll
    for (int k = 0; k < kSub; ++k) {
      if (s + k < p.n) {
        W::load(gate + at_row(j, p, s + k) * j.gate_pitch, g[k]);
        W::load(x + at_row(j, p, s + k) * j.x_pitch, y[k]);
      }
    }
#pragma unroll
    for (int k = 0; k < kSub; ++k) {
      if (s + k < p.n) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
          float a, b;
          Gate<KIND>::split(g[k][v], a, b);
          h[v] = step(a, h[v], Gate<KIND>::u(b, y[k][v]));
        }
        W::store(out + at_row(j, p, s + k) * j.D, h);
      }
    }
  }
  if (j.leave && p.chunk == j.chunks - 1)
#pragma unroll
    for (int v = 0; v < V; ++v) j.leave[(size_t)p.b * j.D + p.c + v] = h[v];
}

template <typename T, int V, int KIND>
__global__ void __launch_bounds__(kThreads) k_scan_bwd(const __grid_constant__ Job j) {
  tc::grid_dependency_wait();
  const Place p = place<V>(j);
  if (!p.on) return;
  using W = Vec<T, V>;
  constexpr int kSubs = kChunk / kSub;
  const T* gate = static_cast<const T*>(j.gate) + p.c;
  const T* x = static_cast<const T*>(j.x) + p.c;
  const T* dh = static_cast<const T*>(j.dh) + p.c;
  T* dgate = static_cast<T*>(j.dgate) + p.c;
  T* dx = static_cast<T*>(j.dx) + p.c;
  // the states before each group of kSub steps
  float group[kSubs][V], h[V];
#pragma unroll
  for (int v = 0; v < V; ++v) h[v] = j.kept[((size_t)p.b * j.chunks + p.chunk) * j.D + p.c + v];
#pragma unroll
  for (int q = 0; q < kSubs; ++q) {
#pragma unroll
    for (int v = 0; v < V; ++v) group[q][v] = h[v];
#pragma unroll
    for (int k = 0; k < kSub; ++k) {
      const int t = q * kSub + k;
      if (t >= p.n) break;
      float g[V], y[V];
      W::load(gate + at_row(j, p, t) * j.gate_pitch, g);
      W::load(x + at_row(j, p, t) * j.x_pitch, y);
#pragma unroll
      for (int v = 0; v < V; ++v) {
        float a, b;
        Gate<KIND>::split(g[v], a, b);
        h[v] = step(a, h[v], Gate<KIND>::u(b, y[v]));
      }
    }
  }
  float r[V];
  enter<V>(j, p, r);
#pragma unroll
  for (int q = kSubs - 1; q >= 0; --q) {
    if (q * kSub >= p.n) continue;
    float a[kSub][V], b[kSub][V], y[kSub][V], before[kSub][V];
#pragma unroll
    for (int k = 0; k < kSub; ++k) {
      const int t = q * kSub + k;
      if (t >= p.n) break;
      float g[V];
      W::load(gate + at_row(j, p, t) * j.gate_pitch, g);
      W::load(x + at_row(j, p, t) * j.x_pitch, y[k]);
#pragma unroll
      for (int v = 0; v < V; ++v) {
        Gate<KIND>::split(g[v], a[k][v], b[k][v]);
        before[k][v] = k == 0 ? group[q][v]
                              : step(a[k - 1][v], before[k - 1][v], Gate<KIND>::u(b[k - 1][v], y[k - 1][v]));
      }
    }
#pragma unroll
    for (int k = kSub - 1; k >= 0; --k) {
      const int t = q * kSub + k;
      if (t >= p.n) continue;
      float up[V], dg[V], du[V];
      W::load(dh + at_row(j, p, t) * j.D, up);
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const float g = up[v] + r[v];
        dg[v] = Gate<KIND>::grad(g, a[k][v], b[k][v], before[k][v], y[k][v]);
        du[v] = Gate<KIND>::u(b[k][v], g);
        r[v] = a[k][v] == 0.0f ? 0.0f : a[k][v] * g;
      }
      W::store(dgate + at_row(j, p, t) * j.dgate_pitch, dg);
      W::store(dx + at_row(j, p, t) * j.dx_pitch, du);
    }
  }
  if (j.leave && p.chunk == 0)
#pragma unroll
    for (int v = 0; v < V; ++v) j.leave[(size_t)p.b * j.D + p.c + v] = r[v];
}

// ------------------------------------------------------------------ host
bool sizes_ok(int B, int L, int D, slim_dtype dtype, slim_gate kind) {
  if (B < 0 || L < 0 || D < 1 || D > (1 << 30) || L > (1 << 30)) return false;
  if (dtype != SLIM_F32 && dtype != SLIM_BF16) return false;
  if (kind != SLIM_GATE_VALUE && kind != SLIM_GATE_LOG && kind != SLIM_GATE_SIGMOID) return false;
  return (double)B * L * D <= 0x1p40 && (double)B * D <= 0x1p36 && B <= 65535;
}

int chunks_of(int L) { return (L + kChunk - 1) / kChunk; }

struct Ws {
  float2* sums;
  float* states;
};
Ws carve(Carver& cv, int B, int L, int D, bool bwd, bool kept) {
  Ws w{};
  const size_t n = (size_t)B * chunks_of(L) * D;
  if (chunks_of(L) > 1) {
    w.sums = cv.take<float2>(n);
    if (bwd || !kept) w.states = cv.take<float>(n);
  }
  return w;
}

template <typename T, int V, int KIND>
bool run_as(const Job& j, bool bwd, cudaStream_t s) {
  const long long n = (long long)j.B * j.chunks * ((j.D + V - 1) / V);
  const dim3 blocks((unsigned)((n + kThreads - 1) / kThreads));
  const double e = (double)j.B * j.L * j.D;
  if (j.chunks > 1) {
    {
      prof::Scope ps(prof::K_SCAN_SUMS, s, 2 * e, 2 * e * sizeof(T));
      if (bwd)
        k_scan_sums<T, V, KIND, true><<<blocks, kThreads, 0, s>>>(j);
      else
        k_scan_sums<T, V, KIND, false><<<blocks, kThreads, 0, s>>>(j);
      if (cudaGetLastError() != cudaSuccess) return false;
    }
    prof::Scope ps(prof::K_SCAN_STATES, s);
    if (!launch_on(k_scan_states, dim3((j.D + 31) / 32, j.B), 32 * kSegs, 0, 1, true, s, j, (int)bwd))
      return false;
  }
  prof::Scope ps(bwd ? prof::K_SCAN_BWD : prof::K_SCAN_FWD, s, e * (bwd ? 10 : 4),
                 e * sizeof(T) * (bwd ? 5 : 3));
  return launch_on(bwd ? k_scan_bwd<T, V, KIND> : k_scan_fwd<T, V, KIND>, blocks, kThreads, 0, 1,
                   j.chunks > 1, s, j);
}

template <typename T, int V>
bool run_v(const Job& j, slim_gate kind, bool bwd, cudaStream_t s) {
  if (kind == SLIM_GATE_VALUE) return run_as<T, V, SLIM_GATE_VALUE>(j, bwd, s);
  if (kind == SLIM_GATE_LOG) return run_as<T, V, SLIM_GATE_LOG>(j, bwd, s);
  return run_as<T, V, SLIM_GATE_SIGMOID>(j, bwd, s);
}

bool run(const Job& j, slim_dtype dtype, slim_gate kind, bool bwd, bool fours, cudaStream_t s) {
  if (dtype == SLIM_F32) return fours ? run_v<float, 4>(j, kind, bwd, s) : run_v<float, 1>(j, kind, bwd, s);
  return fours ? run_v<__nv_bfloat16, 4>(j, kind, bwd, s) : run_v<__nv_bfloat16, 1>(j, kind, bwd, s);
}

// A tensor of rows: pointer and pitch.
struct Rows {
  const void* p;
  long long pitch;
  bool written;
};
constexpr long long kMaxPitch = 1LL << 40;
bool rows_ok(const Rows& r, int B, int L, int D, int es, bool* fours) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(r.p);
  if (!r.p || (a & (es - 1)) || r.pitch < (r.written ? D : 0) || r.pitch > kMaxPitch) return false;
  if ((double)r.pitch * B * L >= 0x1p60) return false;
  *fours = *fours && (a & (4 * es - 1)) == 0 && (r.pitch & 3) == 0;
  return true;
}
bool fp32_ok(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3) == 0; }

// A state to another place, or zero.
slim_status pass_on(const float* from, float* to, size_t n, cudaStream_t s) {
  if (!to || n == 0 || to == from) return SLIM_OK;
  const cudaError_t e = from ? cudaMemcpyAsync(to, from, n * sizeof(float), cudaMemcpyDeviceToDevice, s)
                             : cudaMemsetAsync(to, 0, n * sizeof(float), s);
  return e == cudaSuccess ? SLIM_OK : SLIM_ERR_CUDA;
}

slim_status workspace_ok(const void* ws, size_t have, size_t need) {
  if (need == 0) return SLIM_OK;
  if (!ws || have < need) return SLIM_ERR_WORKSPACE;
  return reinterpret_cast<uintptr_t>(ws) & 255 ? SLIM_ERR_INVALID_ARG : SLIM_OK;
}

}  // namespace
}  // namespace layer
}  // namespace slim

extern "C" slim_status slim_gated_scan_workspace_size(int B, int L, int D, int backward, size_t* bytes) {
  using namespace slim::layer;
  if (!bytes || !sizes_ok(B, L, D, SLIM_F32, SLIM_GATE_VALUE) || (backward & ~1)) return SLIM_ERR_INVALID_ARG;
  slim::Carver cv(nullptr);
  carve(cv, B, L, D, backward != 0, false);
  *bytes = cv.bytes();
  return SLIM_OK;
}

extern "C" slim_status slim_gated_scan_fwd(const void* gate, long long gate_pitch, const void* x,
                                           long long x_pitch, const float* h0, int B, int L, int D,
                                           slim_dtype dtype, slim_gate kind, void* h, float* last,
                                           float* kept, void* workspace, size_t workspace_bytes,
                                           void* stream) {
  using namespace slim::layer;
  if (!sizes_ok(B, L, D, dtype, kind)) return SLIM_ERR_INVALID_ARG;
  if (!fp32_ok(h0) || !fp32_ok(last) || !fp32_ok(kept)) return SLIM_ERR_INVALID_ARG;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (B == 0 || L == 0) return pass_on(h0, last, (size_t)B * D, s);
  const int es = dtype == SLIM_F32 ? 4 : 2;
  bool fours = D % 4 == 0;
  for (const Rows& r : {Rows{gate, gate_pitch, false}, Rows{x, x_pitch, false}, Rows{h, D, true}})
    if (!rows_ok(r, B, L, D, es, &fours)) return SLIM_ERR_INVALID_ARG;
  size_t need = 0;
  slim_gated_scan_workspace_size(B, L, D, 0, &need);
  const slim_status st = workspace_ok(workspace, workspace_bytes, need);
  if (st != SLIM_OK) return st;
  slim::Carver cv(workspace);
  const Ws w = carve(cv, B, L, D, false, false);
  Job j{};
  j.gate = gate;
  j.gate_pitch = gate_pitch;
  j.x = x;
  j.x_pitch = x_pitch;
  j.enter = h0;
  j.h = h;
  j.leave = last;
  j.states = kept ? kept : w.states;
  j.sums = w.sums;
  j.B = B;
  j.L = L;
  j.D = D;
  j.chunks = chunks_of(L);
  return run(j, dtype, kind, false, fours, s) ? SLIM_OK : SLIM_ERR_CUDA;
}

extern "C" slim_status slim_gated_scan_bwd(const void* gate, long long gate_pitch, const void* x,
                                           long long x_pitch, const float* kept, const void* dh,
                                           const float* dlast, int B, int L, int D, slim_dtype dtype,
                                           slim_gate kind, void* dgate, long long dgate_pitch,
                                           void* dx, long long dx_pitch, float* dh0, void* workspace,
                                           size_t workspace_bytes, void* stream) {
  using namespace slim::layer;
  if (!sizes_ok(B, L, D, dtype, kind)) return SLIM_ERR_INVALID_ARG;
  if (!fp32_ok(dlast) || !fp32_ok(dh0) || !fp32_ok(kept)) return SLIM_ERR_INVALID_ARG;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (B == 0 || L == 0) return pass_on(dlast, dh0, (size_t)B * D, s);
  const int es = dtype == SLIM_F32 ? 4 : 2;
  bool fours = D % 4 == 0;
  for (const Rows& r : {Rows{gate, gate_pitch, false}, Rows{x, x_pitch, false}, Rows{dh, D, false},
                        Rows{dgate, dgate_pitch, true}, Rows{dx, dx_pitch, true}})
    if (!rows_ok(r, B, L, D, es, &fours)) return SLIM_ERR_INVALID_ARG;
  if (!kept) return SLIM_ERR_INVALID_ARG;
  size_t need = 0;
  slim_gated_scan_workspace_size(B, L, D, 1, &need);
  const slim_status st = workspace_ok(workspace, workspace_bytes, need);
  if (st != SLIM_OK) return st;
  slim::Carver cv(workspace);
  const Ws w = carve(cv, B, L, D, true, true);
  Job j{};
  j.gate = gate;
  j.gate_pitch = gate_pitch;
  j.x = x;
  j.x_pitch = x_pitch;
  j.dh = dh;
  j.enter = dlast;
  j.kept = kept;
  j.dgate = dgate;
  j.dgate_pitch = dgate_pitch;
  j.dx = dx;
  j.dx_pitch = dx_pitch;
  j.leave = dh0;
  j.states = w.states;
  j.sums = w.sums;
  j.B = B;
  j.L = L;
  j.D = D;
  j.chunks = chunks_of(L);
  return run(j, dtype, kind, true, fours, s) ? SLIM_OK : SLIM_ERR_CUDA;
}
