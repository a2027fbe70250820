// Gated linear recurrence over long sequences, and its gradients.  Contract:
// include/slim_layer.h.
//
//     h_t = a_t h_(t-1) + u_t            per channel
//     r_t = a_t g_t,  g_t = dh_t + r_(t+1)    backward: the same from the other end
//
// Some steps together take a state to A state + H.  A thread has four steps of V
// neighbouring channels in registers, sixteen half warps of them one behind the other
// are a block's tile of 64 steps, and the blocks of a cluster have tiles one behind
// the other (a round).  Every thread computes its (A, H); two warps that do nothing
// else scan the tile's, read those of the cluster's other blocks from their shared
// memory and fold them onto the state that all blocks carry from round to round; then
// each thread runs from its own state and writes.  The folding warps have no stores to
// global memory on their way: the cluster barrier's release, which waits for its
// thread's earlier stores (5 us a round when the writing warps took part in it), finds
// none, and the other warps arrive without one.
//
// A thread's inputs come by asynchronous copies into slots of shared memory of its own,
// those of the next round while this one is computed.  The order of every sum is fixed
// by the sizes: tiles are folded one by one, however many a cluster has.
//
// Backward, dgate needs h_(t-1): the forward keeps the states between tiles in fp32
// (1 / 64 the bytes of an fp32 h), and a tile's states are computed again from there,
// so that h itself is not read.
#include <math.h>
#include <stdint.h>

#include <type_traits>

#include "../../include/slim_layer.h"
#include "common.cuh"
#include "launch.h"
#include "profiler.h"
#include "tc_common.cuh"

namespace slim {
namespace layer {
namespace {

constexpr int kChunk = SLIM_SCAN_CHUNK;  // steps of a tile
constexpr int kSteps = 4;                // of a thread
constexpr int kWarps = 8, kRun = 32 * kWarps, kThreads = kRun + 64;  // two folding warps
constexpr int kLanes = 16;               // across the channels
constexpr int kMaxCluster = 16;
constexpr int kShort = 8;  // sequences up to here need no neighbours: a thread has all steps
static_assert(2 * kWarps * kSteps == kChunk, "the states kept are those between tiles");

struct Job {
  const void *gate, *x, *dh;
  long long gate_pitch, x_pitch;
  const float* enter;  // forward: h0, backward: dlast; or null (zero)
  const float* start;  // backward: the states before each chunk
  void *h, *dgate, *dx;
  long long dgate_pitch, dx_pitch;
  float* leave;        // forward: last state, backward: dh0; or null
  float* kept;         // forward: the states before each chunk, or null
  int B, L, D, chunks;
  int groups;          // of channels
  int tiles, rounds;
};

// V channels of a step as they lie in memory.
template <typename T, int V> struct Raw;
template <> struct Raw<float, 1> { using type = float; };
template <> struct Raw<float, 2> { using type = float2; };
template <> struct Raw<float, 4> { using type = float4; };
template <> struct Raw<__nv_bfloat16, 1> { using type = __nv_bfloat16; };
template <> struct Raw<__nv_bfloat16, 2> { using type = uint32_t; };
template <> struct Raw<__nv_bfloat16, 4> { using type = uint2; };
__device__ __forceinline__ void unpack(float r, float* v) { v[0] = r; }
__device__ __forceinline__ void unpack(float2 r, float* v) {
  v[0] = r.x;
  v[1] = r.y;
}
__device__ __forceinline__ void unpack(float4 r, float* v) {
  v[0] = r.x;
  v[1] = r.y;
  v[2] = r.z;
  v[3] = r.w;
}
__device__ __forceinline__ void unpack(__nv_bfloat16 r, float* v) { v[0] = __bfloat162float(r); }
__device__ __forceinline__ void unpack(uint32_t r, float* v) {
  v[0] = __uint_as_float(r << 16);
  v[1] = __uint_as_float(r & 0xffff0000u);
}
__device__ __forceinline__ void unpack(uint2 r, float* v) {
  unpack(r.x, v);
  unpack(r.y, v + 2);
}
__device__ __forceinline__ void pack(const float* v, float& r) { r = v[0]; }
__device__ __forceinline__ void pack(const float* v, float2& r) { r = make_float2(v[0], v[1]); }
__device__ __forceinline__ void pack(const float* v, float4& r) { r = make_float4(v[0], v[1], v[2], v[3]); }
__device__ __forceinline__ void pack(const float* v, __nv_bfloat16& r) { r = __float2bfloat16_rn(v[0]); }
__device__ __forceinline__ void pack(const float* v, uint32_t& r) { r = tc::pack_bf16(v[0], v[1]); }
__device__ __forceinline__ void pack(const float* v, uint2& r) {
  r = make_uint2(tc::pack_bf16(v[0], v[1]), tc::pack_bf16(v[2], v[3]));
}

// One step's V channels to a slot in shared memory.  Odd bf16 channels are too small for
// an asynchronous copy.
template <typename R>
__device__ __forceinline__ void fetch_to(R* slot, const R* from) {
  if constexpr (sizeof(R) == 2)
    *slot = *from;
  else
    asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(tc::smem_u32(slot)), "l"(from), "n"(sizeof(R))
                 : "memory");
}

// 1 / x to a unit in the last place, for x in [1, 2].
__device__ __forceinline__ float reciprocal(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

template <int KIND> struct Gate {
  // a, and b with u = b x.  The exponential is 2^(g log2 e): off by 2^-22, and by
  // 1.25 |g| 2^-24 from its argument's rounding.
  static __device__ __forceinline__ void split(float g, float& a, float& b) {
    constexpr float log2e = 1.44269504f;
    if (KIND == SLIM_GATE_SIGMOID) {
      // sigmoid(g) and sigmoid(-g), each to its own digits
      const float e = tc::ex2_approx(-log2e * fabsf(g)), big = reciprocal(1.0f + e), small = e * big;
      a = g < 0.0f ? small : big;
      b = g < 0.0f ? big : small;
    } else {
      a = KIND == SLIM_GATE_LOG ? tc::ex2_approx(log2e * g) : g;
      b = 1.0f;
    }
  }
  static __device__ __forceinline__ float u(float b, float x) {
    return KIND == SLIM_GATE_SIGMOID ? b * x : x;
  }
  // d loss / d gate from g = d loss / d h_t and the state before the step
  template <bool SAFE>
  static __device__ __forceinline__ float grad(float g, float a, float b, float before, float x) {
    if (KIND == SLIM_GATE_VALUE) return g * before;
    // a step that starts anew: nothing, whatever the state that it forgot
    if (SAFE && a == 0.0f) return 0.0f;
    return KIND == SLIM_GATE_LOG ? g * before * a : g * (before - x) * (a * b);
  }
};

// a s + u; a of zero forgets a state that is not finite, too.
__device__ __forceinline__ float step(float a, float s, float u) { return a == 0.0f ? u : fmaf(a, s, u); }
// The same where `safe`, else the plain sum.  The plain sum of a state that is not
// finite stays so to the end of a thread's steps, which then takes them again.
template <bool SAFE>
__device__ __forceinline__ float next(float a, float s, float u) {
  return SAFE ? step(a, s, u) : fmaf(a, s, u);
}
// What of g passes to the step before a's.
template <bool SAFE>
__device__ __forceinline__ float back(float a, float g) {
  return SAFE && a == 0.0f ? 0.0f : __fmul_rn(a, g);
}
template <int V>
__device__ __forceinline__ bool finite(const float* s) {
  bool ok = true;
#pragma unroll
  for (int v = 0; v < V; ++v) ok = ok && fabsf(s[v]) < INFINITY;
  return ok;
}
// (A, H) of two runs of steps, one behind the other.
__device__ __forceinline__ float2 join(float2 first, float2 then) {
  return make_float2(first.x * then.x, step(then.x, first.y, then.y));
}

// A thread's S steps of V channels.  Those from n on do not exist: a = 1, u = 0 (FULL:
// all do).
template <typename T, int V, int S> struct Steps {
  using R = typename Raw<T, V>::type;
  static __device__ __forceinline__ void load(const T* p, long long pitch, int n, R* r) {
#pragma unroll
    for (int i = 0; i < S; ++i) {
      if (i < n) r[i] = *reinterpret_cast<const R*>(p);
      p += pitch;
    }
  }
  // The slots of a tensor: step i's is kRun on from step i - 1's.
  static __device__ __forceinline__ void fetch(const T* p, long long pitch, int n, R* slot) {
#pragma unroll
    for (int i = 0; i < S; ++i) {
      if (i < n) fetch_to(slot + i * kRun, reinterpret_cast<const R*>(p));
      p += pitch;
    }
  }
  static __device__ __forceinline__ void take(const R* slot, R* r) {
#pragma unroll
    for (int i = 0; i < S; ++i) r[i] = slot[i * kRun];
  }
  static __device__ __forceinline__ void store(T* p, const float* v) {
    R r;
    pack(v, r);
    *reinterpret_cast<R*>(p) = r;
  }
  template <int KIND, bool FULL>
  static __device__ __forceinline__ void gates(const R* g, int n, float (*a)[V], float (*b)[V]) {
#pragma unroll
    for (int i = 0; i < S; ++i) {
      float f[V];
      unpack(g[i], f);
#pragma unroll
      for (int v = 0; v < V; ++v) {
        Gate<KIND>::split(f[v], a[i][v], b[i][v]);
        if (!FULL && i >= n) {
          a[i][v] = 1.0f;
          b[i][v] = 0.0f;
        }
      }
    }
  }
  template <bool FULL>
  static __device__ __forceinline__ void values(const R* g, int n, float (*x)[V]) {
#pragma unroll
    for (int i = 0; i < S; ++i) {
      unpack(g[i], x[i]);
#pragma unroll
      for (int v = 0; v < V; ++v)
        if (!FULL && i >= n) x[i][v] = 0.0f;
    }
  }
  static __device__ __forceinline__ void product(const float (*a)[V], float* A) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      A[v] = a[0][v];
#pragma unroll
      for (int i = 1; i < S; ++i) A[v] *= a[i][v];
    }
  }
  template <bool SAFE>
  static __device__ __forceinline__ void forward(const float (*a)[V], const float (*u)[V], float* s) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      s[v] = u[0][v];
#pragma unroll
      for (int i = 1; i < S; ++i) s[v] = next<SAFE>(a[i][v], s[v], u[i][v]);
    }
  }
  // r = a_0 g_0 of these steps alone
  template <bool SAFE>
  static __device__ __forceinline__ void backward(const float (*a)[V], const float (*dh)[V], float* r) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      float g = dh[S - 1][v];
#pragma unroll
      for (int i = S - 2; i >= 0; --i) g = next<SAFE>(a[i + 1][v], g, dh[i][v]);
      r[v] = back<SAFE>(a[0][v], g);
    }
  }
  // runs from s and writes h
  template <bool SAFE>
  static __device__ __forceinline__ void write(T* p, long long pitch, int n, const float (*a)[V],
                                               const float (*u)[V], float* s) {
#pragma unroll
    for (int i = 0; i < S; ++i) {
#pragma unroll
      for (int v = 0; v < V; ++v) s[v] = next<SAFE>(a[i][v], s[v], u[i][v]);
      if (i < n) store(p, s);
      p += pitch;
    }
  }
  static __device__ __forceinline__ void run(T* p, long long pitch, int n, const float (*a)[V],
                                             const float (*u)[V], float* s) {
    float from[V];
#pragma unroll
    for (int v = 0; v < V; ++v) from[v] = s[v];
    write<false>(p, pitch, n, a, u, s);
    if (!finite<V>(s)) {
#pragma unroll
      for (int v = 0; v < V; ++v) s[v] = from[v];
      write<true>(p, pitch, n, a, u, s);
    }
  }
  // the states before each step, from s
  template <bool SAFE, int KIND>
  static __device__ __forceinline__ void states(const float (*a)[V], const float (*b)[V], const float (*x)[V],
                                                float* s, float (*before)[V]) {
#pragma unroll
    for (int i = 0; i < S; ++i)
#pragma unroll
      for (int v = 0; v < V; ++v) {
        before[i][v] = s[v];
        s[v] = next<SAFE>(a[i][v], s[v], Gate<KIND>::u(b[i][v], x[i][v]));
      }
  }
  // the gradients, from r = a_(t+1) g_(t+1) of the step behind the last
  template <bool SAFE, int KIND>
  static __device__ __forceinline__ void grads(T* pg, long long g_pitch, T* px, long long x_pitch, int n,
                                               const float (*a)[V], const float (*b)[V], const float (*x)[V],
                                               const float (*dh)[V], const float (*before)[V], float* r) {
    float g[V];
#pragma unroll
    for (int i = S - 1; i >= 0; --i) {
      float dg[V], dx[V];
#pragma unroll
      for (int v = 0; v < V; ++v) {
        g[v] = i == S - 1 ? __fadd_rn(dh[i][v], r[v]) : next<SAFE>(a[i + 1][v], g[v], dh[i][v]);
        dg[v] = Gate<KIND>::template grad<SAFE>(g[v], a[i][v], b[i][v], before[i][v], x[i][v]);
        dx[v] = Gate<KIND>::u(b[i][v], g[v]);
      }
      if (i < n) {
        store(pg + i * g_pitch, dg);
        store(px + i * x_pitch, dx);
      }
    }
#pragma unroll
    for (int v = 0; v < V; ++v) r[v] = back<SAFE>(a[0][v], g[v]);
  }
  template <int KIND>
  static __device__ __forceinline__ void run_back(T* pg, long long g_pitch, T* px, long long x_pitch, int n,
                                                  const float (*a)[V], const float (*b)[V], const float (*x)[V],
                                                  const float (*dh)[V], float* s, float* r) {
    float before[S][V], from[V], into[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      from[v] = s[v];
      into[v] = r[v];
    }
    states<false, KIND>(a, b, x, s, before);
    const bool plain = finite<V>(s);
    grads<false, KIND>(pg, g_pitch, px, x_pitch, n, a, b, x, dh, before, r);
    if (!plain || !finite<V>(r)) {
      states<true, KIND>(a, b, x, from, before);
#pragma unroll
      for (int v = 0; v < V; ++v) r[v] = into[v];
      grads<true, KIND>(pg, g_pitch, px, x_pitch, n, a, b, x, dh, before, r);
    }
  }
};

// ------------------------------------------------------------------ barriers
__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ uint32_t cluster_blocks() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
  return r;
}
// Every warp of the cluster meets; what a RELEASE warp wrote before it is seen behind it.
template <bool RELEASE>
__device__ __forceinline__ void cluster_meet() {
  __syncwarp();
  if (RELEASE)
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  else
    asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// The running warps' sums are there (0); what enters their steps is (1).
enum { SUMS = 1, ENTER = 2 };
template <int ID>
__device__ __forceinline__ void hand_over() {
  __syncwarp();
  asm volatile("bar.arrive %0, %1;" ::"n"(ID), "n"(kThreads) : "memory");
}
template <int ID>
__device__ __forceinline__ void take_over() {
  __syncwarp();
  asm volatile("bar.sync %0, %1;" ::"n"(ID), "n"(kThreads) : "memory");
}
// p of this block's shared memory, read from block `rank`'s.
__device__ __forceinline__ float2 load_of(const float2* p, uint32_t rank) {
  uint32_t at;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(tc::smem_u32(p)), "r"(rank));
  float2 v;
  asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(at) : "memory");
  return v;
}

// The folding warps' round, one thread a channel: from the warps' sums (BACK: the
// tile's last first) what precedes each, `s` the state that enters the round, and
// `enter` the one that enters this block's tile.
template <int CH, bool BACK>
__device__ __forceinline__ void fold_tile(const float2 (*sum)[CH], float2 (*before)[CH], float2* whole, int ch) {
  float2 f[kWarps], e = make_float2(1.0f, 0.0f);
#pragma unroll
  for (int w = 0; w < kWarps; ++w) f[w] = sum[w][ch];
#pragma unroll
  for (int i = 0; i < kWarps; ++i) {
    const int w = BACK ? kWarps - 1 - i : i;
    before[w][ch] = e;
    e = i ? join(e, f[w]) : f[w];
  }
  if (whole) whole[ch] = e;
}
__device__ __forceinline__ void fold_round(const float2* mine, uint32_t rank, uint32_t blocks, float* enter,
                                           float& s) {
  if (blocks == 1) {
    const float2 f = *mine;
    *enter = s;
    s = step(f.x, s, f.y);
    return;
  }
  float2 f[kMaxCluster];
#pragma unroll
  for (int z = 0; z < kMaxCluster; ++z)
    if (z < blocks) f[z] = load_of(mine, z);
#pragma unroll
  for (int z = 0; z < kMaxCluster; ++z)
    if (z < blocks) {
      if (z == rank) *enter = s;
      s = step(f[z].x, s, f[z].y);
    }
}

// A warp's two halves joined: the sum of both goes to shared memory, and what the later
// half has ahead of it stays (the identity in the earlier one).
template <int V, bool BACK>
__device__ __forceinline__ void join_halves(const float* A, const float* H, int lane, float2* to, float2* ahead) {
  const bool later = (lane >= kLanes) != BACK;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const float2 own = make_float2(A[v], H[v]);
    const float2 other = make_float2(__shfl_xor_sync(0xffffffffu, own.x, kLanes),
                                     __shfl_xor_sync(0xffffffffu, own.y, kLanes));
    ahead[v] = later ? other : make_float2(1.0f, 0.0f);
    if (later) to[v] = join(other, own);
  }
}

// ------------------------------------------------------------------ kernels
// Places in shared memory are written again only behind two hand-overs; a block's
// sums, which its neighbours read, have a second copy: whoever writes the next but one
// round's has met all readers in the round between.
template <typename T, int V, int KIND>
__global__ void __launch_bounds__(kThreads, 2) k_scan_fwd(const __grid_constant__ Job j) {
  constexpr int S = kSteps, CH = kLanes * V;
  using P = Steps<T, V, S>;
  using R = typename P::R;
  __shared__ float2 sum[kWarps][CH], before[kWarps][CH], whole[2][CH];
  __shared__ float enter[CH];
  extern __shared__ uint4 slots[];
  const uint32_t rank = cluster_rank(), blocks = cluster_blocks();
  const int stream = blockIdx.x / blocks, b = stream / j.groups, c0 = (stream - b * j.groups) * CH;
  if (threadIdx.x >= kRun) {
    const int ch = threadIdx.x - kRun;
    const bool on = ch < CH && c0 + ch < j.D;
    float s = on && j.enter ? j.enter[(size_t)b * j.D + c0 + ch] : 0.0f;
    for (int r = 0; r < j.rounds; ++r) {
      take_over<SUMS>();
      if (ch < CH) fold_tile<CH, false>(sum, before, whole[r & 1], ch);
      if (blocks > 1) cluster_meet<true>();
      if (ch < CH) fold_round(&whole[r & 1][ch], rank, blocks, &enter[ch], s);
      hand_over<ENTER>();
    }
    if (blocks > 1) cluster_meet<true>();
    return;
  }
  R* mine = reinterpret_cast<R*>(slots) + threadIdx.x;  // [2][gate, x][S][kRun]
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, at = lane % kLanes * V;
  const int c = c0 + at, first = (2 * warp + lane / kLanes) * S;  // of the tile's steps
  const bool on = c < j.D;
  int t0 = rank * kChunk + first;
  const long long row = (long long)b * j.L + t0;
  const T* gate = static_cast<const T*>(j.gate) + row * j.gate_pitch + c;
  const T* x = static_cast<const T*>(j.x) + row * j.x_pitch + c;
  T* h_out = static_cast<T*>(j.h) + row * j.D + c;
  const int round = blocks * kChunk;
  auto steps_at = [&](int t) { return on ? min(max(j.L - t, 0), S) : 0; };
  auto fetch = [&](int n, int stage) {
    P::fetch(gate, j.gate_pitch, n, mine + (2 * stage) * S * kRun);
    P::fetch(x, j.x_pitch, n, mine + (2 * stage + 1) * S * kRun);
  };
  int n = steps_at(t0);
  fetch(n, 0);
  for (int r = 0; r < j.rounds; ++r) {
    tc::cp_async_wait_all();
    gate += round * j.gate_pitch;
    x += round * j.x_pitch;
    const int later = r + 1 < j.rounds ? steps_at(t0 + round) : 0;
    fetch(later, (r + 1) & 1);
    float a[S][V], u[S][V];
    auto inputs = [&](auto full) {
      constexpr bool FULL = decltype(full)::value;
      float bb[S][V];
      R in[S];
      P::take(mine + (2 * (r & 1)) * S * kRun, in);
      P::template gates<KIND, FULL>(in, n, a, bb);
      P::take(mine + (2 * (r & 1) + 1) * S * kRun, in);
      P::template values<FULL>(in, n, u);
#pragma unroll
      for (int i = 0; i < S; ++i)
#pragma unroll
        for (int v = 0; v < V; ++v) u[i][v] = Gate<KIND>::u(bb[i][v], u[i][v]);
    };
    if (__all_sync(0xffffffffu, n == S))
      inputs(std::true_type());
    else
      inputs(std::false_type());
    float A[V], H[V];
    P::product(a, A);
    P::template forward<false>(a, u, H);
    if (!finite<V>(H)) P::template forward<true>(a, u, H);
    float2 ahead[V];
    join_halves<V, false>(A, H, lane, &sum[warp][at], ahead);
    hand_over<SUMS>();
    if (blocks > 1) cluster_meet<false>();
    take_over<ENTER>();
    if (n > 0) {
      float h[V];
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const float2 k = before[warp][at + v];
        h[v] = step(k.x, enter[at + v], k.y);
        h[v] = step(ahead[v].x, h[v], ahead[v].y);
      }
      if (j.kept && first == 0)
#pragma unroll
        for (int v = 0; v < V; ++v) j.kept[((size_t)b * j.chunks + t0 / kChunk) * j.D + c + v] = h[v];
      P::run(h_out, j.D, n, a, u, h);
      if (j.leave && t0 + n == j.L)
#pragma unroll
        for (int v = 0; v < V; ++v) j.leave[(size_t)b * j.D + c + v] = h[v];
    }
    h_out += (long long)round * j.D;
    t0 += round;
    n = later;
  }
  if (blocks > 1) cluster_meet<false>();  // no block leaves while another reads its sums
}

template <typename T, int V, int KIND>
__global__ void __launch_bounds__(kThreads, 2) k_scan_bwd(const __grid_constant__ Job j) {
  constexpr int S = kSteps, CH = kLanes * V;
  using P = Steps<T, V, S>;
  using R = typename P::R;
  __shared__ float2 sum[kWarps][CH], before[kWarps][CH], whole[2][CH];  // backward (A, G)
  __shared__ float2 run[kWarps][CH], run_before[kWarps][CH];            // the forward's (A, H)
  __shared__ float enter[CH];
  extern __shared__ uint4 slots[];
  const uint32_t rank = cluster_rank(), blocks = cluster_blocks();
  const int stream = blockIdx.x / blocks, b = stream / j.groups, c0 = (stream - b * j.groups) * CH;
  if (threadIdx.x >= kRun) {
    const int ch = threadIdx.x - kRun;
    const bool on = ch < CH && c0 + ch < j.D;
    float s = on && j.enter ? j.enter[(size_t)b * j.D + c0 + ch] : 0.0f;
    for (int r = 0; r < j.rounds; ++r) {
      take_over<SUMS>();
      if (ch < CH) {
        fold_tile<CH, true>(sum, before, whole[r & 1], ch);
        if (blocks == 1) fold_tile<CH, false>(run, run_before, nullptr, ch);
      }
      if (blocks > 1) {
        __syncwarp();
        asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
        if (ch < CH) fold_tile<CH, false>(run, run_before, nullptr, ch);  // the cluster's meeting meanwhile
        __syncwarp();
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
      }
      if (ch < CH) fold_round(&whole[r & 1][ch], rank, blocks, &enter[ch], s);
      hand_over<ENTER>();
    }
    if (blocks > 1) cluster_meet<true>();
    return;
  }
  R* mine = reinterpret_cast<R*>(slots) + threadIdx.x;  // [2][gate, x, dh][S][kRun]
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, at = lane % kLanes * V;
  const int c = c0 + at, first = (2 * warp + lane / kLanes) * S;
  const bool on = c < j.D;
  int tile = j.tiles - 1 - (int)rank;  // tiles come from the last
  const long long row = (long long)b * j.L + (long long)tile * kChunk + first;
  const T* gate = static_cast<const T*>(j.gate) + row * j.gate_pitch + c;
  const T* x = static_cast<const T*>(j.x) + row * j.x_pitch + c;
  const T* dh_in = static_cast<const T*>(j.dh) + row * j.D + c;
  T* dgate = static_cast<T*>(j.dgate) + row * j.dgate_pitch + c;
  T* dx = static_cast<T*>(j.dx) + row * j.dx_pitch + c;
  const long long round = (long long)blocks * kChunk;
  auto steps_of = [&](int q) { return on && q >= 0 ? min(max(j.L - (q * kChunk + first), 0), S) : 0; };
  auto fetch = [&](int n, int stage) {
    P::fetch(gate, j.gate_pitch, n, mine + (3 * stage) * S * kRun);
    P::fetch(x, j.x_pitch, n, mine + (3 * stage + 1) * S * kRun);
    P::fetch(dh_in, j.D, n, mine + (3 * stage + 2) * S * kRun);
  };
  int n = steps_of(tile);
  fetch(n, 0);
  for (int r = 0; r < j.rounds; ++r) {
    tc::cp_async_wait_all();
    gate -= round * j.gate_pitch;
    x -= round * j.x_pitch;
    dh_in -= round * j.D;
    const int later = r + 1 < j.rounds ? steps_of(tile - (int)blocks) : 0;
    fetch(later, (r + 1) & 1);
    float h[V];
#pragma unroll
    for (int v = 0; v < V; ++v) h[v] = n > 0 ? j.start[((size_t)b * j.chunks + tile) * j.D + c + v] : 0.0f;
    const R* now = mine + 3 * (r & 1) * S * kRun;
    float a[S][V], bb[S][V], y[S][V], dh[S][V];
    auto inputs = [&](auto full) {
      constexpr bool FULL = decltype(full)::value;
      R in[S];
      P::take(now, in);
      P::template gates<KIND, FULL>(in, n, a, bb);
      P::take(now + S * kRun, in);
      P::template values<FULL>(in, n, y);
      P::take(now + 2 * S * kRun, in);
      P::template values<FULL>(in, n, dh);
    };
    if (__all_sync(0xffffffffu, n == S))
      inputs(std::true_type());
    else
      inputs(std::false_type());
    float A[V], H[V], G[V];
    auto sums_of = [&](auto safe) {
      float u[S][V];
#pragma unroll
      for (int i = 0; i < S; ++i)
#pragma unroll
        for (int v = 0; v < V; ++v) u[i][v] = Gate<KIND>::u(bb[i][v], y[i][v]);
      P::template forward<decltype(safe)::value>(a, u, H);
      P::template backward<decltype(safe)::value>(a, dh, G);
    };
    P::product(a, A);
    sums_of(std::false_type());
    if (!finite<V>(H) || !finite<V>(G)) sums_of(std::true_type());
    float2 ahead[V], run_ahead[V];
    join_halves<V, true>(A, G, lane, &sum[warp][at], ahead);
    join_halves<V, false>(A, H, lane, &run[warp][at], run_ahead);
    hand_over<SUMS>();
    if (blocks > 1) cluster_meet<false>();
    take_over<ENTER>();
    if (n > 0) {
      float e[V];
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const float2 k = before[warp][at + v], f = run_before[warp][at + v];
        e[v] = step(k.x, enter[at + v], k.y);
        e[v] = step(ahead[v].x, e[v], ahead[v].y);
        h[v] = step(f.x, h[v], f.y);
        h[v] = step(run_ahead[v].x, h[v], run_ahead[v].y);
      }
      P::template run_back<KIND>(dgate, j.dgate_pitch, dx, j.dx_pitch, n, a, bb, y, dh, h, e);
      if (j.leave && tile == 0 && first == 0)
#pragma unroll
        for (int v = 0; v < V; ++v) j.leave[(size_t)b * j.D + c + v] = e[v];
    }
    dgate -= round * j.dgate_pitch;
    dx -= round * j.dx_pitch;
    tile -= (int)blocks;
    n = later;
  }
  if (blocks > 1) cluster_meet<false>();
}

// Up to kShort steps (a decoding step): a thread has V channels of a sequence.
template <typename T, int V, int KIND, bool BWD>
__global__ void __launch_bounds__(128) k_scan_short(const __grid_constant__ Job j) {
  constexpr int S = kShort;
  using P = Steps<T, V, S>;
  const long long i = (long long)blockIdx.x * 128 + threadIdx.x;
  const int per = j.D / V;
  const long long b = i / per;
  if (b >= j.B) return;
  const int c = (int)(i - b * per) * V, n = j.L;
  const long long row = b * j.L;
  typename P::R g[S], x[S], up[S];
  P::load(static_cast<const T*>(j.gate) + row * j.gate_pitch + c, j.gate_pitch, n, g);
  P::load(static_cast<const T*>(j.x) + row * j.x_pitch + c, j.x_pitch, n, x);
  if (BWD) P::load(static_cast<const T*>(j.dh) + row * j.D + c, j.D, n, up);
  float s[V];
#pragma unroll
  for (int v = 0; v < V; ++v) s[v] = j.enter ? j.enter[b * j.D + c + v] : 0.0f;
  float a[S][V], bb[S][V], y[S][V];
  P::template gates<KIND, false>(g, n, a, bb);
  P::template values<false>(x, n, y);
  if (BWD) {
    float dh[S][V], h[V];
    P::template values<false>(up, n, dh);
#pragma unroll
    for (int v = 0; v < V; ++v) h[v] = j.start[b * j.D + c + v];
    P::template run_back<KIND>(static_cast<T*>(j.dgate) + row * j.dgate_pitch + c, j.dgate_pitch,
                               static_cast<T*>(j.dx) + row * j.dx_pitch + c, j.dx_pitch, n, a, bb, y, dh, h, s);
  } else {
#pragma unroll
    for (int k = 0; k < S; ++k)
#pragma unroll
      for (int v = 0; v < V; ++v) y[k][v] = Gate<KIND>::u(bb[k][v], y[k][v]);
    if (j.kept)
#pragma unroll
      for (int v = 0; v < V; ++v) j.kept[b * j.D + c + v] = s[v];
    P::run(static_cast<T*>(j.h) + row * j.D + c, j.D, n, a, y, s);
  }
  if (j.leave)
#pragma unroll
    for (int v = 0; v < V; ++v) j.leave[b * j.D + c + v] = s[v];
}

// ------------------------------------------------------------------ host
bool sizes_ok(int B, int L, int D, slim_dtype dtype, slim_gate kind) {
  if (B < 0 || L < 0 || D < 1 || D > (1 << 30) || L > (1 << 30)) return false;
  if (dtype != SLIM_F32 && dtype != SLIM_BF16) return false;
  if (kind != SLIM_GATE_VALUE && kind != SLIM_GATE_LOG && kind != SLIM_GATE_SIGMOID) return false;
  return (double)B * L * D <= 0x1p40 && (double)B * D <= 0x1p32;
}

int cdiv(long long a, long long b) { return (int)((a + b - 1) / b); }

// Blocks of a cluster: as many as are resident together (two an SM), as far as there
// are tiles.
int cluster_of(long long streams, int tiles) {
  const long long room = 152 * 2;
  long long z = room / streams;
  if (z > kMaxCluster) z = kMaxCluster;
  if (z > 8 && z < 16) z = 8;
  if (z > tiles) z = tiles;
  return z < 1 ? 1 : (int)z;
}

template <typename T, int V, int KIND>
bool run_as(Job j, bool bwd, cudaStream_t s) {
  const double e = (double)j.B * j.L * j.D;
  prof::Scope ps(bwd ? prof::K_SCAN_BWD : prof::K_SCAN_FWD, s, e * (bwd ? 10 : 4), e * sizeof(T) * (bwd ? 5 : 3));
  if (j.L <= kShort) {
    const long long n = (long long)j.B * (j.D / V);
    auto k = bwd ? k_scan_short<T, V, KIND, true> : k_scan_short<T, V, KIND, false>;
    k<<<(unsigned)((n + 127) / 128), 128, 0, s>>>(j);
    return cudaGetLastError() == cudaSuccess;
  }
  j.groups = cdiv(j.D, kLanes * V);
  j.tiles = cdiv(j.L, kChunk);
  const long long streams = (long long)j.B * j.groups;
  const int z = cluster_of(streams, j.tiles);
  j.rounds = cdiv(j.tiles, z);
  auto k = bwd ? k_scan_bwd<T, V, KIND> : k_scan_fwd<T, V, KIND>;
  const size_t smem = (size_t)2 * (bwd ? 3 : 2) * kSteps * V * kRun * sizeof(T);  // slots
  static bool flags[2][kMaxDevices];
  bool* ready = device_flag(flags[bwd]);
  if (!ready || !*ready) {
    if (cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess ||
        cudaFuncSetAttribute(k, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess)
      return false;
    if (ready) *ready = true;
  }
  return launch_on(k, dim3((unsigned)(streams * z)), kThreads, smem, z, false, s, j);
}

template <typename T, int V>
bool run_v(const Job& j, slim_gate kind, bool bwd, cudaStream_t s) {
  if (kind == SLIM_GATE_VALUE) return run_as<T, V, SLIM_GATE_VALUE>(j, bwd, s);
  if (kind == SLIM_GATE_LOG) return run_as<T, V, SLIM_GATE_LOG>(j, bwd, s);
  return run_as<T, V, SLIM_GATE_SIGMOID>(j, bwd, s);
}
template <typename T>
bool run_t(const Job& j, slim_gate kind, bool bwd, int together, cudaStream_t s) {
  if (together == 4) return run_v<T, 4>(j, kind, bwd, s);
  return together == 2 ? run_v<T, 2>(j, kind, bwd, s) : run_v<T, 1>(j, kind, bwd, s);
}
bool run(const Job& j, slim_dtype dtype, slim_gate kind, bool bwd, int together, cudaStream_t s) {
  return dtype == SLIM_F32 ? run_t<float>(j, kind, bwd, together, s)
                           : run_t<__nv_bfloat16>(j, kind, bwd, together, s);
}

// A tensor of rows: pointer and pitch.
struct Rows {
  const void* p;
  long long pitch;
  bool written;
};
constexpr long long kMaxPitch = 1LL << 40;
// `together`: channels that every tensor so far can move in one piece.
bool rows_ok(const Rows& r, int B, int L, int D, int es, int* together) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(r.p);
  if (!r.p || (a & (es - 1)) || r.pitch < (r.written ? D : 0) || r.pitch > kMaxPitch) return false;
  if ((double)r.pitch * B * L >= 0x1p60) return false;
  while (*together > 1 && ((a & (*together * es - 1)) || (r.pitch & (*together - 1)))) *together /= 2;
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

}  // namespace
}  // namespace layer
}  // namespace slim

extern "C" slim_status slim_gated_scan_fwd(const void* gate, long long gate_pitch, const void* x,
                                           long long x_pitch, const float* h0, int B, int L, int D,
                                           slim_dtype dtype, slim_gate kind, void* h, float* last,
                                           float* kept, void* stream) {
  using namespace slim::layer;
  if (!sizes_ok(B, L, D, dtype, kind)) return SLIM_ERR_INVALID_ARG;
  if (!fp32_ok(h0) || !fp32_ok(last) || !fp32_ok(kept)) return SLIM_ERR_INVALID_ARG;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (B == 0 || L == 0) return pass_on(h0, last, (size_t)B * D, s);
  const int es = dtype == SLIM_F32 ? 4 : 2;
  int together = D % 4 == 0 ? 4 : D % 2 == 0 ? 2 : 1;
  for (const Rows& r : {Rows{gate, gate_pitch, false}, Rows{x, x_pitch, false}, Rows{h, D, true}})
    if (!rows_ok(r, B, L, D, es, &together)) return SLIM_ERR_INVALID_ARG;
  Job j{};
  j.gate = gate;
  j.gate_pitch = gate_pitch;
  j.x = x;
  j.x_pitch = x_pitch;
  j.enter = h0;
  j.h = h;
  j.leave = last;
  j.kept = kept;
  j.B = B;
  j.L = L;
  j.D = D;
  j.chunks = cdiv(L, kChunk);
  return run(j, dtype, kind, false, together, s) ? SLIM_OK : SLIM_ERR_CUDA;
}

extern "C" slim_status slim_gated_scan_bwd(const void* gate, long long gate_pitch, const void* x,
                                           long long x_pitch, const float* kept, const void* dh,
                                           const float* dlast, int B, int L, int D, slim_dtype dtype,
                                           slim_gate kind, void* dgate, long long dgate_pitch,
                                           void* dx, long long dx_pitch, float* dh0, void* stream) {
  using namespace slim::layer;
  if (!sizes_ok(B, L, D, dtype, kind)) return SLIM_ERR_INVALID_ARG;
  if (!fp32_ok(dlast) || !fp32_ok(dh0) || !fp32_ok(kept)) return SLIM_ERR_INVALID_ARG;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (B == 0 || L == 0) return pass_on(dlast, dh0, (size_t)B * D, s);
  const int es = dtype == SLIM_F32 ? 4 : 2;
  int together = D % 4 == 0 ? 4 : D % 2 == 0 ? 2 : 1;
  for (const Rows& r : {Rows{gate, gate_pitch, false}, Rows{x, x_pitch, false}, Rows{dh, D, false},
                        Rows{dgate, dgate_pitch, true}, Rows{dx, dx_pitch, true}})
    if (!rows_ok(r, B, L, D, es, &together)) return SLIM_ERR_INVALID_ARG;
  if (!kept) return SLIM_ERR_INVALID_ARG;
  Job j{};
  j.gate = gate;
  j.gate_pitch = gate_pitch;
  j.x = x;
  j.x_pitch = x_pitch;
  j.dh = dh;
  j.enter = dlast;
  j.start = kept;
  j.dgate = dgate;
  j.dgate_pitch = dgate_pitch;
  j.dx = dx;
  j.dx_pitch = dx_pitch;
  j.leave = dh0;
  j.B = B;
  j.L = L;
  j.D = D;
  j.chunks = cdiv(L, kChunk);
  return run(j, dtype, kind, true, together, s) ? SLIM_OK : SLIM_ERR_CUDA;
}
