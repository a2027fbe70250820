// Gated linear recurrence over long sequences, and its gradients.  Contract:
// include/slim_layer.h.
//
//     h_t = a_t h_(t-1) + u_t            per channel
//     r_t = a_t g_t,  g_t = dh_t + r_(t+1)    backward: the same from the other end
//
// Some steps together take a state to A state + H.  A tile is eight parts of S steps, a
// line of 128 bytes of channels wide; a running warp has a part.  It computes the part's
// (A, H); the tile's sum is joined from them and given away; then the warp runs from the
// state that enters its part and writes.  What enters a tile is its predecessors' work:
//
//   * a sequence of a few tiles is a cluster, whose blocks read each other's sums from
//     shared memory and fold them one by one;
//   * else blocks take tiles in order and look back in global memory: from the nearest
//     earlier tile behind which the state is known, over the sums of those between.
//
// Either way the state is folded tile by tile from the start, so that the bits do not
// depend on which tiles were ready.  The look back is a warp's of its own, and the next
// tile's sums are given away before this one's state is waited for: its wait lies under
// the running warps' work (1 x 65536 x 512 fp32 forward: 120 us with the next tile's
// sums behind it, 87 before it).  Inputs come by asynchronous copies two tiles ahead, and
// their gates are computed again for the second pass, from shared memory (fp32: left there by
// the first): registers for two tiles would leave room for one block an SM.
//
// Measured: 1 x 65536 x 512 fp32 forward 84 us (4.8 TB/s of inputs and outputs; 190 us
// with all of a sequence's tiles in one cluster's rounds), 8 x 4096 x 512 bf16 step with
// sigmoid gates 109 us (forward kernel 40, backward 68).  bf16 has 51 instructions an
// element forward and 79 backward, both passes, at 0.6 a cycle and scheduler, and 73 and
// 136 MB of DRAM traffic: neither is full, and the backward's registers spill.  fp32 waits
// for the exchange and HBM.
//
// Backward, dgate needs h_(t-1): the forward keeps the states every 64 steps in fp32
// (1 / 64 the bytes of an fp32 h), and a tile's states are computed again from there,
// so that h itself is not read.
#include <math.h>
#include <stdint.h>

#include <type_traits>

#include "../../include/slim_layer.h"
#include "common.cuh"
#include "launch.h"
#include "profiler.h"
#include "report.h"
#include "tc_common.cuh"

namespace slim {
namespace layer {
namespace {

constexpr int kChunk = SLIM_SCAN_CHUNK;  // steps between the states that are kept
constexpr int kRun = 256, kParts = kRun / 32;  // running threads, and the parts of a tile's steps
// Of an SM: 96 registers a thread, at which the backward of two bf16 channels a thread
// spills 108 to 144 bytes, and other backward kernels up to 96; three leave 64.
constexpr int kBlocks = 2;
constexpr int kMaxCluster = 16;
constexpr int kStages = 3;  // tiles of a block whose inputs have slots
constexpr int kShort = 8;  // sequences up to here need no neighbours: a thread has all steps
constexpr int kHeader = 64;              // ints: error word, report address, tickets

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
  int groups, tiles;   // of a sequence
  bool wide;           // inputs' rows come in 16-byte pieces
  long long streams;   // B groups
  int* err;            // the header of a workspace, where there is one
  // LOOK (else null)
  unsigned long long* tickets;
  unsigned long long* sum;  // [streams][tiles][CH]
  unsigned* state;
};

// V channels of a step as they lie in memory.
template <typename T, int V> struct Raw;
template <> struct Raw<float, 1> { using type = float; };
template <> struct Raw<float, 2> { using type = float2; };
template <> struct Raw<__nv_bfloat16, 1> { using type = __nv_bfloat16; };
template <> struct Raw<__nv_bfloat16, 2> { using type = uint32_t; };
template <> struct Raw<__nv_bfloat16, 4> { using type = uint2; };
__device__ __forceinline__ void unpack(float r, float* v) { v[0] = r; }
__device__ __forceinline__ void unpack(float2 r, float* v) {
  v[0] = r.x;
  v[1] = r.y;
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

// A gate multiplies the state at every step, and a state that lasts m steps has its error
// m times over.  So a gate near 1 is rounded once: LOG gates by the exponential's series,
// the larger of sigmoid(g) and sigmoid(-g) as 1 less the smaller.  (2^x of the MUFU unit is
// off by up to 2 units of 2^-24, low by 0.1 to 0.5 on average.)
template <typename T, int KIND> struct Gate {
  static constexpr bool WIDE = sizeof(T) == 4;
  // e^g as 2^(g log2 e), zero below 2^-126.  bf16 inputs: off by 2^-22, and by 1.25 |g|
  // 2^-24 from its argument's rounding, which fp32 inputs have back.
  static __device__ __forceinline__ float exponential(float g) {
    constexpr float log2e = 1.44269504f, ln2 = 0.69314718f;
    if (!WIDE) return tc::ex2_approx(log2e * g);
    asm("max.NaN.f32 %0, %0, 0fC3480000;" : "+f"(g));  // -200: an infinity has no remainder
    const float t = log2e * g, e = tc::ex2_approx(t);
    return fmaf(e, fmaf(-t, ln2, g), e);
  }
  // a, or of a sigmoid the smaller of a and b.
  static __device__ __forceinline__ float first(float g) {
    if (KIND == SLIM_GATE_SIGMOID) {
      const float e = exponential(-fabsf(g));
      return e * reciprocal(1.0f + e);
    }
    if (KIND == SLIM_GATE_LOG) {
      // up to g^5 / 5! for |g| < 2^-3, the rest below 2^-27; bf16: up to g^3 / 3! for
      // |g| < 2^-6, the rest below 2^-28
      constexpr float near = WIDE ? 0x1p-3f : 0x1p-6f;
      float p = WIDE ? fmaf(g, fmaf(g, 1.0f / 120.0f, 1.0f / 24.0f), 1.0f / 6.0f) : 1.0f / 6.0f;
      p = fmaf(g, fmaf(g, p, 0.5f), 1.0f);
      return fabsf(g) < near ? fmaf(g, p, 1.0f) : exponential(g);
    }
    return g;
  }
  // a, and b with u = b x.
  static __device__ __forceinline__ void both(float v, bool low, float& a, float& b) {
    const float large = 1.0f - v;
    a = KIND != SLIM_GATE_SIGMOID || low ? v : large;
    b = KIND != SLIM_GATE_SIGMOID ? 1.0f : low ? large : v;
  }
  static __device__ __forceinline__ void split(float g, float& a, float& b) { both(first(g), g < 0.0f, a, b); }
  // fp32: what is held of a gate for the second pass, in its own room, and from there: a,
  // or the smaller sigmoid with the sign of -g.
  static __device__ __forceinline__ float hold(float g) {
    return KIND == SLIM_GATE_SIGMOID ? copysignf(first(g), -g) : first(g);
  }
  static __device__ __forceinline__ void open(float held, float& a, float& b) {
    if (KIND == SLIM_GATE_SIGMOID)
      both(fabsf(held), __float_as_int(held) >= 0, a, b);
    else
      both(held, true, a, b);
  }
  static __device__ __forceinline__ float u(float b, float x) {
    return KIND == SLIM_GATE_SIGMOID ? b * x : x;
  }
  // d h_t / d gate, from the state before the step
  static __device__ __forceinline__ float factor(float a, float b, float before, float x) {
    if (KIND == SLIM_GATE_VALUE) return before;
    return KIND == SLIM_GATE_LOG ? before * a : (before - x) * (a * b);
  }
  // d loss / d gate from g = d loss / d h_t
  template <bool SAFE>
  static __device__ __forceinline__ float grad(float g, float a, float factor) {
    // a step that starts anew: nothing, whatever the state that it forgot
    if (KIND != SLIM_GATE_VALUE && SAFE && a == 0.0f) return 0.0f;
    return g * factor;
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
// A s + H over the steps that (A, H) stand for.  Where their gates' product is past fp32's
// range, a state of zero stays zero, as it does step by step.
__device__ __forceinline__ float over(float A, float s, float H) {
  return A == 0.0f || s == 0.0f ? H : fmaf(A, s, H);
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
// A gate that is not a number leaves no state one, zero included.
template <int V>
__device__ __forceinline__ void poison(const float* A, float* H) {
#pragma unroll
  for (int v = 0; v < V; ++v)
    if (A[v] != A[v]) H[v] = A[v];
}
// (A, H) of two runs of steps, one behind the other.  A product past fp32's range is not
// carried over a new start, on either side of it.
__device__ __forceinline__ float2 join(float2 first, float2 then) {
  return make_float2(then.x == 0.0f || first.x == 0.0f ? 0.0f : first.x * then.x, over(then.x, first.y, then.y));
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
  static __device__ __forceinline__ void take(const R* slot, R* r) {
#pragma unroll
    for (int i = 0; i < S; ++i) r[i] = slot[i * 32];
  }
  // Gates: the first pass leaves the second what is held of them.
  template <int KIND, bool FIRST>
  static __device__ __forceinline__ void take_gates(R* slot, R* r) {
    take(slot, r);
    if constexpr (FIRST && sizeof(T) == 4 && KIND != SLIM_GATE_VALUE) {
#pragma unroll
      for (int i = 0; i < S; ++i) slot[i * 32] = r[i] = Gate<T, KIND>::hold(r[i]);
    }
  }
  static __device__ __forceinline__ void store(T* p, const float* v) {
    R r;
    pack(v, r);
    *reinterpret_cast<R*>(p) = r;
  }
  // HELD: of what take_gates left
  template <int KIND, bool FULL, bool HELD>
  static __device__ __forceinline__ void gates(const R* g, int n, float (*a)[V], float (*b)[V]) {
#pragma unroll
    for (int i = 0; i < S; ++i) {
      float f[V];
      unpack(g[i], f);
#pragma unroll
      for (int v = 0; v < V; ++v) {
        if (HELD && sizeof(T) == 4)
          Gate<T, KIND>::open(f[v], a[i][v], b[i][v]);
        else
          Gate<T, KIND>::split(f[v], a[i][v], b[i][v]);
        if (!FULL && i >= n) {
          a[i][v] = 1.0f;
          b[i][v] = 0.0f;
        }
      }
    }
  }
  // one path for whole parts, which all but the last of a sequence are
  template <int KIND>
  static __device__ __forceinline__ void gates_of(const R* g, int n, float (*a)[V], float (*b)[V]) {
    if (n == S)
      gates<KIND, true, true>(g, n, a, b);
    else
      gates<KIND, false, true>(g, n, a, b);
  }
  static __device__ __forceinline__ void values_of(const R* g, int n, float (*x)[V]) {
    if (n == S)
      values<true>(g, n, x);
    else
      values<false>(g, n, x);
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
  // SAFE: past fp32's range it may go, but not over a new start
  template <bool SAFE>
  static __device__ __forceinline__ void product(const float (*a)[V], float* A) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      A[v] = a[0][v];
#pragma unroll
      for (int i = 1; i < S; ++i) A[v] = SAFE && a[i][v] == 0.0f ? 0.0f : A[v] * a[i][v];
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
  template <bool SAFE, bool FULL>
  static __device__ __forceinline__ void write(T* p, long long pitch, int n, const float (*a)[V],
                                               const float (*u)[V], float* s) {
#pragma unroll
    for (int i = 0; i < S; ++i) {
#pragma unroll
      for (int v = 0; v < V; ++v) s[v] = next<SAFE>(a[i][v], s[v], u[i][v]);
      if (FULL || i < n) store(p, s);
      p += pitch;
    }
  }
  static __device__ __forceinline__ void run(T* p, long long pitch, int n, const float (*a)[V],
                                             const float (*u)[V], float* s) {
    float from[V];
#pragma unroll
    for (int v = 0; v < V; ++v) from[v] = s[v];
    if (n == S)
      write<false, true>(p, pitch, n, a, u, s);
    else
      write<false, false>(p, pitch, n, a, u, s);
    if (!finite<V>(s)) {
#pragma unroll
      for (int v = 0; v < V; ++v) s[v] = from[v];
      write<true, false>(p, pitch, n, a, u, s);
    }
  }
  // The state behind the steps, from s (`zero`: from zero).
  template <bool SAFE, int KIND>
  static __device__ __forceinline__ void run_over(const float (*a)[V], const float (*b)[V], const float (*x)[V],
                                                  float* s, bool zero) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      float t = zero ? Gate<T, KIND>::u(b[0][v], x[0][v]) : next<SAFE>(a[0][v], s[v], Gate<T, KIND>::u(b[0][v], x[0][v]));
#pragma unroll
      for (int i = 1; i < S; ++i) t = next<SAFE>(a[i][v], t, Gate<T, KIND>::u(b[i][v], x[i][v]));
      s[v] = t;
    }
  }
  // x becomes what dgate is of g, d h_t / d gate: from the state s before the first step
  template <bool SAFE, int KIND>
  static __device__ __forceinline__ void factors(const float (*a)[V], const float (*b)[V], float (*x)[V],
                                                 const float* s) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      float t = s[v];
#pragma unroll
      for (int i = 0; i < S; ++i) {
        const float before = t;
        if (i + 1 < S) t = next<SAFE>(a[i][v], t, Gate<T, KIND>::u(b[i][v], x[i][v]));
        x[i][v] = Gate<T, KIND>::factor(a[i][v], b[i][v], before, x[i][v]);
      }
    }
  }
  // the gradients, from r = a_(t+1) g_(t+1) of the step behind the last
  template <bool SAFE, bool FULL, int KIND>
  static __device__ __forceinline__ void grads(T* pg, long long g_pitch, T* px, long long x_pitch, int n,
                                               const float (*a)[V], const float (*b)[V], const float (*factor)[V],
                                               const float (*dh)[V], float* r) {
    float g[V];
#pragma unroll
    for (int i = S - 1; i >= 0; --i) {
      float dg[V], dx[V];
#pragma unroll
      for (int v = 0; v < V; ++v) {
        g[v] = i == S - 1 ? __fadd_rn(dh[i][v], r[v]) : next<SAFE>(a[i + 1][v], g[v], dh[i][v]);
        dg[v] = Gate<T, KIND>::template grad<SAFE>(g[v], a[i][v], factor[i][v]);
        dx[v] = Gate<T, KIND>::u(b[i][v], g[v]);
      }
      if (FULL || i < n) {
        store(pg + i * g_pitch, dg);
        store(px + i * x_pitch, dx);
      }
    }
#pragma unroll
    for (int v = 0; v < V; ++v) r[v] = back<SAFE>(a[0][v], g[v]);
  }
  // From the state s before the steps and r, which becomes what the step before them
  // gets; x is used up, above(dh) reads the last input.
  template <int KIND, typename Above>
  static __device__ __forceinline__ void run_back(T* pg, long long g_pitch, T* px, long long x_pitch, int n,
                                                  const float (*a)[V], const float (*b)[V], float (*x)[V],
                                                  const float* s, float* r, const Above& above) {
    float end[V], from[V], dh[S][V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      end[v] = s[v];
      from[v] = r[v];
    }
    run_over<false, KIND>(a, b, x, end, false);
    const bool plain = finite<V>(end);
    if (plain)
      factors<false, KIND>(a, b, x, s);
    else
      factors<true, KIND>(a, b, x, s);
    above(dh);
    if (n == S)
      grads<false, true, KIND>(pg, g_pitch, px, x_pitch, n, a, b, x, dh, r);
    else
      grads<false, false, KIND>(pg, g_pitch, px, x_pitch, n, a, b, x, dh, r);
    if (!plain || !finite<V>(r)) {
#pragma unroll
      for (int v = 0; v < V; ++v) r[v] = from[v];
      grads<true, false, KIND>(pg, g_pitch, px, x_pitch, n, a, b, x, dh, r);
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
// All threads of the cluster meet.
__device__ __forceinline__ void cluster_meet() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// p of this block's shared memory, read from block `rank`'s.
__device__ __forceinline__ float2 load_of(const float2* p, uint32_t rank) {
  uint32_t at;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(tc::smem_u32(p)), "r"(rank));
  float2 v;
  asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(at) : "memory");
  return v;
}

// ------------------------------------------------------------------ between the tiles
// LOOK, tiles that do not fit one cluster or two waves of blocks: for each tile and
// channel, the tile's sum (A, H) and the state behind it, as soon as they are known.  A
// word is its own flag: it starts as kNone, a NaN that arithmetic does not make, and is
// written once and whole.  So no fence is needed, which would wait for its warp's copies
// and stores as well (with flags and fences 8 x 4096 x 512 bf16 took 73 instead of 57 us).
constexpr unsigned kNone = 0xffffffffu;
constexpr unsigned long long kNone2 = 0xffffffffffffffffull;
// V neighbouring channels' words.
template <int V>
__device__ __forceinline__ void look_at(const unsigned long long* p, unsigned long long* v) {
  if constexpr (V == 2)
    asm volatile("ld.relaxed.gpu.global.v2.b64 {%0, %1}, [%2];" : "=l"(v[0]), "=l"(v[1]) : "l"(p) : "memory");
  else
    asm volatile("ld.relaxed.gpu.global.b64 %0, [%1];" : "=l"(v[0]) : "l"(p) : "memory");
}
template <int V>
__device__ __forceinline__ void look_at(const unsigned* p, unsigned* v) {
  if constexpr (V == 2)
    asm volatile("ld.relaxed.gpu.global.v2.b32 {%0, %1}, [%2];" : "=r"(v[0]), "=r"(v[1]) : "l"(p) : "memory");
  else
    asm volatile("ld.relaxed.gpu.global.b32 %0, [%1];" : "=r"(v[0]) : "l"(p) : "memory");
}
template <int V, typename W>
__device__ __forceinline__ bool there(const W* v) {
  return v[0] != (W)kNone2 && v[V - 1] != (W)kNone2;
}
__device__ __forceinline__ void show(unsigned long long* p, float2 f) {
  unsigned long long v = (unsigned long long)__float_as_uint(f.y) << 32 | __float_as_uint(f.x);
  if (v == kNone2) v = 0x7fffffff7fffffffull;
  asm volatile("st.relaxed.gpu.global.b64 [%0], %1;" ::"l"(p), "l"(v) : "memory");
}
__device__ __forceinline__ void show(unsigned* p, float f) {
  unsigned v = __float_as_uint(f);
  if (v == kNone) v = 0x7fffffffu;
  asm volatile("st.relaxed.gpu.global.b32 [%0], %1;" ::"l"(p), "r"(v) : "memory");
}
__device__ __forceinline__ float fold(unsigned long long f, float s) {
  return over(__uint_as_float((unsigned)f), s, __uint_as_float((unsigned)(f >> 32)));
}

// A wait's polls (see tc_common.cuh): false once it has to give up.
struct Patience {
  uint32_t i = 0;
  uint64_t t0 = 0;
  __device__ __forceinline__ bool operator()(int* err) {
    if ((i & 63) == 63) {
      if (*reinterpret_cast<volatile int*>(err) != 0) return false;
      const uint64_t now = tc::globaltimer_ns();
      if (i == 63) t0 = now;
      if (now - t0 > tc::kWaitLimitNs || i >= tc::kWaitMaxPolls) {
        tc::give_up(err);
        return false;
      }
    }
    ++i;
    __nanosleep(64);
    return true;
  }
};

// The state that enters tile q > 0 of V channels (tiles counted in the order they are
// run): from an earlier tile behind which it is known, over the sums of those between
// one by one -- the same operations whichever tile that is.  sum and state are the first
// tile's, CH words from a tile to the next; the first tile has no sum.
template <int V>
__device__ __forceinline__ void look_back(const unsigned long long* sum, const unsigned* state, int q, int* err,
                                          float* s) {
  constexpr int N = 8, CH = 32 * V;
  Patience more;
#pragma unroll
  for (int v = 0; v < V; ++v) s[v] = 0.0f;
  int m = -1;  // s enters tile m
  for (int low = q; m < 0; low -= N) {
    if (low <= 0) {
      if (!more(err)) return;
      low = q;
    }
    unsigned st[N][V];
#pragma unroll
    for (int k = 0; k < N; ++k) {
      st[k][0] = kNone;
      if (low - 1 - k >= 0) look_at<V>(state + (size_t)(low - 1 - k) * CH, st[k]);
    }
#pragma unroll
    for (int k = N - 1; k >= 0; --k)
      if (there<V>(st[k])) {
#pragma unroll
        for (int v = 0; v < V; ++v) s[v] = __uint_as_float(st[k][v]);
        m = low - k;
      }
  }
  while (m < q) {
    unsigned long long f[N][V];
#pragma unroll
    for (int k = 0; k < N; ++k) {
      f[k][0] = kNone2;
      if (m + k < q) look_at<V>(sum + (size_t)(m + k) * CH, f[k]);
    }
    int n = 0;
#pragma unroll
    for (int k = 0; k < N; ++k)
      if (n == k && there<V>(f[k])) {
#pragma unroll
        for (int v = 0; v < V; ++v) s[v] = fold(f[k][v], s[v]);
        n = k + 1;
      }
    m += n;
    if (n == 0) {
      do {
        if (!more(err)) return;
        look_at<V>(sum + (size_t)m * CH, f[0]);
      } while (!there<V>(f[0]));
    }
  }
}

// Where a block is: tile q (in the order they are run; < 0: none) of a stream, channels
// c0 ..
struct Place {
  int b, c0, q;
  long long stream;
};
template <int CH>
__device__ __forceinline__ Place place_of(const Job& j, long long stream, int q) {
  Place p;
  p.stream = stream;
  p.q = q;
  p.b = (int)(stream / j.groups);
  p.c0 = (int)(stream - (long long)p.b * j.groups) * CH;
  return p;
}
// LOOK: the tile of the next ticket.  Tickets go in order, so that whatever a tile waits
// for has been taken by a running block, which ends its tiles in order.
template <int CH>
__device__ __forceinline__ Place next_place(const Job& j) {
  const unsigned long long t = atomicAdd(j.tickets, 1ull), q = t / (unsigned long long)j.streams;
  if (q >= j.tiles) return Place{0, 0, -1, 0};
  return place_of<CH>(j, (long long)(t - q * j.streams), (int)q);
}

// What a block's warps hand each other.  The running ones (a part of the tile's steps
// each) put their sums; the first of them put the tile's and what stands before each
// part; the folding one puts the state that enters the tile.  What is there twice goes in
// turn: whoever writes the next but one tile's has met all readers of the first.
template <int CH> struct Exchange {
  float2 sum[kParts][CH];        // (A, H); backward (A, G)
  float2 before[2][kParts][CH];  // of the parts run before
  float2 whole[2][CH];
  float enter[2][CH];
  Place start[3], place[2];      // the first tiles; the third behind the one that runs
};
// Barriers: the running warps among each other; the entering state is there; the tile's
// sum is.  (Two each of the last, in turn.)
enum { SUMS = 1, ENTER = 2, WHOLE = 4 };
__device__ __forceinline__ void arrive(int id, int threads) {
  __syncwarp();
  asm volatile("bar.arrive %0, %1;" ::"r"(id), "r"(threads) : "memory");
}
__device__ __forceinline__ void meet(int id, int threads) {
  __syncwarp();
  asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory");
}

// The folding warp, V channels a lane: it runs ahead of the others, so that what enters
// a tile is there soon after its sums are.
template <int V>
__device__ __forceinline__ void fold_tiles(const Job& j, Exchange<32 * V>& ex, Place at) {
  constexpr int CH = 32 * V;
  const int ch = (threadIdx.x - kRun) * V;
  auto enters = [&](const Place& p, float* s) {
#pragma unroll
    for (int v = 0; v < V; ++v)
      s[v] = j.enter && p.c0 + ch + v < j.D ? j.enter[(size_t)p.b * j.D + p.c0 + ch + v] : 0.0f;
  };
  float s[V];
  if (!j.tickets) {  // the block's tile in a cluster of the sequence's
    const uint32_t blocks = cluster_blocks();
    enters(at, s);
    if (blocks > 1) {
      cluster_meet();
      for (int z0 = 0; z0 < at.q; z0 += 8) {
        float2 f[8][V];
#pragma unroll
        for (int z = 0; z < 8; ++z)
#pragma unroll
          for (int v = 0; v < V; ++v)
            if (z0 + z < at.q) f[z][v] = load_of(&ex.whole[0][ch + v], z0 + z);
#pragma unroll
        for (int z = 0; z < 8; ++z)
#pragma unroll
          for (int v = 0; v < V; ++v)
            if (z0 + z < at.q) s[v] = over(f[z][v].x, s[v], f[z][v].y);
      }
    }
#pragma unroll
    for (int v = 0; v < V; ++v) ex.enter[0][ch + v] = s[v];
    arrive(ENTER, kRun + 32);
    if (blocks > 1) cluster_meet();  // no block leaves while another reads its sums
    return;
  }
  Place then = ex.start[1], later = ex.start[2];
  for (int k = 0; at.q >= 0; k ^= 1) {
    Place last = later;
    if (threadIdx.x == kRun && later.q >= 0) last = next_place<CH>(j);
    const size_t tile0 = (size_t)at.stream * j.tiles * CH + ch;
    if (at.q == 0)
      enters(at, s);
    else
      look_back<V>(j.sum + tile0, j.state + tile0, at.q, j.err, s);
    meet(WHOLE + k, 32 + CH);  // and every running warp has left the tile before the last
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const float2 f = ex.whole[k][ch + v];
      if (at.q + 1 < j.tiles) show(j.state + tile0 + (size_t)at.q * CH + v, over(f.x, s[v], f.y));
      ex.enter[k][ch + v] = s[v];
    }
    if (threadIdx.x == kRun) ex.place[k] = last;
    arrive(ENTER + k, kRun + 32);
    at = then;
    then = later;
    later = ex.place[k];
  }
}

// A running warp, its sums put: the first CH threads join a channel's.
template <int CH, bool BACK>
__device__ __forceinline__ void join_parts(const Job& j, Exchange<CH>& ex, const Place& at, int k) {
  const int ch = threadIdx.x;
  if (ch < CH) {
    float2 f = make_float2(1.0f, 0.0f);
#pragma unroll
    for (int i = 0; i < kParts; ++i) {
      const int p = BACK ? kParts - 1 - i : i;
      ex.before[k][p][ch] = f;
      f = i ? join(f, ex.sum[p][ch]) : ex.sum[p][ch];
    }
    ex.whole[k][ch] = f;
    if (j.tickets) {
      if (at.q > 0 && at.q + 1 < j.tiles) show(j.sum + ((size_t)at.stream * j.tiles + at.q) * CH + ch, f);
      arrive(WHOLE + k, 32 + CH);
    }
  }
  if (!j.tickets && cluster_blocks() > 1) cluster_meet();
}
// What enters the warp's part.
template <int V>
__device__ __forceinline__ void enter_part(const Exchange<32 * V>& ex, int k, int part, int at, float* s) {
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const float2 f = ex.before[k][part][at + v];
    s[v] = over(f.x, ex.enter[k][at + v], f.y);
  }
}

// ------------------------------------------------------------------ kernels
// LOOK: clears the words that the scan's blocks wait for, and its header; tickets begin
// with `ticket`.
__global__ void __launch_bounds__(256) k_scan_clear(int* header, uint4* words, long long n, unsigned* rep,
                                                    unsigned long long ticket) {
  tc::grid_dependency_wait();
  const uint4 none = make_uint4(kNone, kNone, kNone, kNone);
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < n; i += (long long)gridDim.x * 256) words[i] = none;
  if (blockIdx.x == 0 && threadIdx.x < kHeader && (threadIdx.x < 2 || threadIdx.x > 5)) header[threadIdx.x] = 0;
  if (blockIdx.x == 0 && threadIdx.x == 4) *reinterpret_cast<unsigned long long*>(header + 4) = ticket;
  if (blockIdx.x == 0 && threadIdx.x == 0) tc::set_report(header, rep);
}

// The block's first tile, to all its threads.
template <int CH>
__device__ __forceinline__ Place begin(const Job& j, Exchange<CH>& ex) {
  tc::grid_dependency_wait();
  if (threadIdx.x == kRun) {
    if (j.tickets) {
      for (int i = 0; i < 3; ++i) ex.start[i] = next_place<CH>(j);
    } else {
      if (j.err && blockIdx.x == 0) *j.err = 0;
      ex.start[0] = place_of<CH>(j, blockIdx.x / cluster_blocks(), (int)cluster_rank());
      ex.start[1] = ex.start[2] = ex.place[0] = Place{0, 0, -1, 0};
    }
  }
  __syncthreads();
  return ex.start[0];
}

// A warp's rows of a tensor to its slots, [S][32 lanes]: `wide`, in 16-byte pieces, else
// each lane its own channels.  The first n steps, channels of c0 .. up to D.
template <typename T, int V, int S>
__device__ __forceinline__ void fetch_rows(const T* rows, long long pitch, int n, int c0, int D, bool wide,
                                           typename Raw<T, V>::type* slots) {
  const int lane = threadIdx.x & 31;
  if (wide) {
    constexpr int E = 16 / sizeof(T), per = 32 * V / E;  // elements of a piece, pieces of a row
    const int c = lane % per * E;
    if (c0 + c >= D) return;
    rows += lane / per * pitch + c0 + c;
    uint32_t to = tc::smem_u32(slots) + lane * 16;
#pragma unroll
    for (int i = 0; i < S; i += 32 / per) {
      if (i + lane / per < n) tc::cp_async16(to, rows, 16);
      rows += 32 / per * pitch;
      to += 512;
    }
  } else if (c0 + lane * V < D) {
    rows += c0 + lane * V;
#pragma unroll
    for (int i = 0; i < S; ++i) {
      if (i < n) fetch_to(slots + i * 32 + lane, reinterpret_cast<const typename Raw<T, V>::type*>(rows));
      rows += pitch;
    }
  }
}
__device__ __forceinline__ void fetched() { asm volatile("cp.async.commit_group;" ::: "memory"); }
// All but the last group are there.
__device__ __forceinline__ void fetch_wait() {
  asm volatile("cp.async.wait_group 1;" ::: "memory");
  __syncwarp();
}

template <typename T, int V, int S, int KIND>
__global__ void __launch_bounds__(kRun + 32, kBlocks) k_scan_fwd(const __grid_constant__ Job j) {
  constexpr int CH = 32 * V, kTile = kParts * S;
  using P = Steps<T, V, S>;
  using R = typename P::R;
  __shared__ __align__(16) Exchange<CH> ex;
  extern __shared__ uint4 slots[];
  Place at = begin<CH>(j, ex);
  if (threadIdx.x >= kRun) {
    fold_tiles<V>(j, ex, at);
    return;
  }
  const int part = threadIdx.x / 32, lane = threadIdx.x & 31;
  R* mine = reinterpret_cast<R*>(slots) + part * (kStages * 2 * S * 32);  // [kStages][gate, x][S][32]
  auto steps_of = [&](const Place& p) { return p.q >= 0 ? min(max(j.L - (p.q * kTile + part * S), 0), S) : 0; };
  auto fetch = [&](const Place& p, int k) {
    const long long row = (long long)p.b * j.L + p.q * kTile + part * S;
    const int n = steps_of(p);
    fetch_rows<T, V, S>(static_cast<const T*>(j.gate) + row * j.gate_pitch, j.gate_pitch, n, p.c0, j.D, j.wide,
                        mine + 2 * k * S * 32);
    fetch_rows<T, V, S>(static_cast<const T*>(j.x) + row * j.x_pitch, j.x_pitch, n, p.c0, j.D, j.wide,
                        mine + (2 * k + 1) * S * 32);
    fetched();
  };
  auto inputs = [&](auto first, int n, int k, float (*a)[V], float (*u)[V]) {
    float bb[S][V];
    R in[S];
    P::template take_gates<KIND, decltype(first)::value>(mine + 2 * k * S * 32 + lane, in);
    P::template gates_of<KIND>(in, n, a, bb);
    P::take(mine + (2 * k + 1) * S * 32 + lane, in);
    P::values_of(in, n, u);
#pragma unroll
    for (int i = 0; i < S; ++i)
#pragma unroll
      for (int v = 0; v < V; ++v) u[i][v] = Gate<T, KIND>::u(bb[i][v], u[i][v]);
  };
  auto sums = [&](const Place& p, int slot, int k) {
    float a[S][V], u[S][V], A[V], H[V];
    inputs(std::true_type(), steps_of(p), slot, a, u);
    P::template product<false>(a, A);
    P::template forward<false>(a, u, H);
    if (!finite<V>(H) || !finite<V>(A)) {
      P::template product<true>(a, A);
      P::template forward<true>(a, u, H);
      poison<V>(A, H);
    }
#pragma unroll
    for (int v = 0; v < V; ++v) ex.sum[part][lane * V + v] = make_float2(A[v], H[v]);
    meet(SUMS, kRun);
    join_parts<CH, false>(j, ex, p, k);
  };
  Place then = ex.start[1], later = ex.start[2];
  fetch(at, 0);
  fetch(then, 1);
  fetch_wait();
  sums(at, 0, 0);
  meet(SUMS, kRun);  // the sums are read: no state is waited for between these and the next
  int slot = 0;
  for (int k = 0; at.q >= 0; k ^= 1) {
    const int slot1 = slot == 2 ? 0 : slot + 1;
    if (then.q >= 0) {
      fetch(later, slot1 == 2 ? 0 : slot1 + 1);
      fetch_wait();
      sums(then, slot1, k ^ 1);
    }
    meet(ENTER + k, kRun + 32);
    const Place last = ex.place[k];
    const int n = steps_of(at), c = at.c0 + lane * V;
    if (n > 0 && c < j.D) {
      float a[S][V], u[S][V], h[V];
      inputs(std::false_type(), n, slot, a, u);
      enter_part<V>(ex, k, part, lane * V, h);
      const int t0 = at.q * kTile + part * S;
      if (j.kept && t0 % kChunk == 0)
#pragma unroll
        for (int v = 0; v < V; ++v) j.kept[((size_t)at.b * j.chunks + t0 / kChunk) * j.D + c + v] = h[v];
      P::run(static_cast<T*>(j.h) + ((long long)at.b * j.L + t0) * j.D + c, j.D, n, a, u, h);
      if (j.leave && t0 + n == j.L)
#pragma unroll
        for (int v = 0; v < V; ++v) j.leave[(size_t)at.b * j.D + c + v] = h[v];
    }
    __syncwarp();  // the slots are read
    at = then;
    then = later;
    later = last;
    slot = slot1;
  }
  if (!j.tickets && cluster_blocks() > 1) cluster_meet();
}

template <typename T, int V, int S, int KIND>
__global__ void __launch_bounds__(kRun + 32, kBlocks) k_scan_bwd(const __grid_constant__ Job j) {
  constexpr int CH = 32 * V, kTile = kParts * S;
  using P = Steps<T, V, S>;
  using R = typename P::R;
  __shared__ __align__(16) Exchange<CH> ex;
  __shared__ float run[kParts][CH], run_enter[2][kParts][CH];  // the forward's H, and its states
  extern __shared__ uint4 slots[];
  Place at = begin<CH>(j, ex);
  if (threadIdx.x >= kRun) {
    fold_tiles<V>(j, ex, at);
    return;
  }
  const int part = threadIdx.x / 32, lane = threadIdx.x & 31;
  R* mine = reinterpret_cast<R*>(slots) + part * (kStages * 3 * S * 32);  // [kStages][gate, x, dh][S][32]
  // The last warps run the forward's states over a chunk's parts, from p0: a thread a channel.
  constexpr int per = kChunk / S, runners = kParts / per * CH;
  static_assert(runners <= kRun, "a thread for each chunk and channel");
  const int runner = kRun - 1 - (int)threadIdx.x, p0 = runner / CH * per, own = runner < runners ? runner % CH : CH;
  auto first_of = [&](const Place& p) { return (j.tiles - 1 - p.q) * kTile + part * S; };  // tiles come from the last
  auto steps_of = [&](const Place& p) {
    return p.q >= 0 && p.q < j.tiles ? min(max(j.L - first_of(p), 0), S) : 0;
  };
  auto fetch = [&](const Place& p, int k) {
    const long long row = (long long)p.b * j.L + first_of(p);
    const int n = steps_of(p);
    fetch_rows<T, V, S>(static_cast<const T*>(j.gate) + row * j.gate_pitch, j.gate_pitch, n, p.c0, j.D, j.wide,
                        mine + 3 * k * S * 32);
    fetch_rows<T, V, S>(static_cast<const T*>(j.x) + row * j.x_pitch, j.x_pitch, n, p.c0, j.D, j.wide,
                        mine + (3 * k + 1) * S * 32);
    fetch_rows<T, V, S>(static_cast<const T*>(j.dh) + row * j.D, j.D, n, p.c0, j.D, j.wide,
                        mine + (3 * k + 2) * S * 32);
    fetched();
  };
  auto front = [&](auto first, int n, int k, float (*a)[V], float (*bb)[V], float (*y)[V]) {
    R in[S];
    P::template take_gates<KIND, decltype(first)::value>(mine + 3 * k * S * 32 + lane, in);
    P::template gates_of<KIND>(in, n, a, bb);
    P::take(mine + (3 * k + 1) * S * 32 + lane, in);
    P::values_of(in, n, y);
  };
  auto above = [&](int n, int k, float (*dh)[V]) {
    R in[S];
    P::take(mine + (3 * k + 2) * S * 32 + lane, in);
    P::values_of(in, n, dh);
  };
  auto start_of = [&](const Place& p) {
    const int t = (j.tiles - 1 - p.q) * kTile + p0 * S;
    return own < CH && p.q >= 0 && p.c0 + own < j.D && t >= 0 && t < j.L
               ? j.start[((size_t)p.b * j.chunks + t / kChunk) * j.D + p.c0 + own]
               : 0.0f;
  };
  auto sums = [&](const Place& p, int slot, int k) {
    float before = start_of(p);
    const int n = steps_of(p);
    float a[S][V], bb[S][V], y[S][V], dh[S][V], A[V], H[V], G[V];
    front(std::true_type(), n, slot, a, bb, y);
    P::template product<false>(a, A);
    P::template run_over<false, KIND>(a, bb, y, H, true);
    if (!finite<V>(H) || !finite<V>(A)) {
      P::template product<true>(a, A);
      P::template run_over<true, KIND>(a, bb, y, H, true);
      poison<V>(A, H);
    }
    above(n, slot, dh);
    P::template backward<false>(a, dh, G);
    if (!finite<V>(G) || !finite<V>(A)) {
      P::template backward<true>(a, dh, G);
      poison<V>(A, G);
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
      ex.sum[part][lane * V + v] = make_float2(A[v], G[v]);
      run[part][lane * V + v] = H[v];
    }
    meet(SUMS, kRun);
    join_parts<CH, true>(j, ex, p, k);
    if (own < CH) {
#pragma unroll
      for (int i = 0; i < per; ++i) {
        run_enter[k][p0 + i][own] = before;
        before = over(ex.sum[p0 + i][own].x, before, run[p0 + i][own]);
      }
    }
  };
  Place then = ex.start[1], later = ex.start[2];
  fetch(at, 0);
  fetch(then, 1);
  fetch_wait();
  sums(at, 0, 0);
  meet(SUMS, kRun);  // the sums are read: no state is waited for between these and the next
  int slot = 0;
  for (int k = 0; at.q >= 0; k ^= 1) {
    const int slot1 = slot == 2 ? 0 : slot + 1;
    if (then.q >= 0) {
      fetch(later, slot1 == 2 ? 0 : slot1 + 1);
      fetch_wait();
      sums(then, slot1, k ^ 1);
    }
    meet(ENTER + k, kRun + 32);
    const Place last = ex.place[k];
    const int n = steps_of(at), c = at.c0 + lane * V, t0 = first_of(at);
    if (n > 0 && c < j.D) {
      float a[S][V], bb[S][V], y[S][V], e[V], h[V];
      front(std::false_type(), n, slot, a, bb, y);
      enter_part<V>(ex, k, part, lane * V, e);
#pragma unroll
      for (int v = 0; v < V; ++v) h[v] = run_enter[k][part][lane * V + v];
      const long long row = (long long)at.b * j.L + t0;
      P::template run_back<KIND>(static_cast<T*>(j.dgate) + row * j.dgate_pitch + c, j.dgate_pitch,
                                 static_cast<T*>(j.dx) + row * j.dx_pitch + c, j.dx_pitch, n, a, bb, y, h, e,
                                 [&](float (*dh)[V]) { above(n, slot, dh); });
      if (j.leave && t0 == 0)
#pragma unroll
        for (int v = 0; v < V; ++v) j.leave[(size_t)at.b * j.D + c + v] = e[v];
    }
    __syncwarp();  // the slots are read
    at = then;
    then = later;
    later = last;
    slot = slot1;
  }
  if (!j.tickets && cluster_blocks() > 1) cluster_meet();
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
  if (BWD) {
    float h[V];
#pragma unroll
    for (int v = 0; v < V; ++v) h[v] = j.start[b * j.D + c + v];
    float a[S][V], bb[S][V], y[S][V];
    P::template gates<KIND, false, false>(g, n, a, bb);
    P::template values<false>(x, n, y);
    P::template run_back<KIND>(static_cast<T*>(j.dgate) + row * j.dgate_pitch + c, j.dgate_pitch,
                               static_cast<T*>(j.dx) + row * j.dx_pitch + c, j.dx_pitch, n, a, bb, y, h, s,
                               [&](float (*dh)[V]) { P::template values<false>(up, n, dh); });
  } else {
    float a[S][V], bb[S][V], y[S][V];
    P::template gates<KIND, false, false>(g, n, a, bb);
    P::template values<false>(x, n, y);
#pragma unroll
    for (int k = 0; k < S; ++k)
#pragma unroll
      for (int v = 0; v < V; ++v) y[k][v] = Gate<T, KIND>::u(bb[k][v], y[k][v]);
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

// A thread's channels: a row of a tile is a line of 128 bytes.  A tile is kParts parts
// of S steps.
template <typename T> constexpr int kWidest = 4 / sizeof(T);
// (16 steps: fewer tiles to look back over, where a thread's registers hold them.)
constexpr int part_steps(int es, bool bwd) { return es == 4 && !bwd ? 16 : 8; }
int element(slim_dtype dtype) { return dtype == SLIM_F32 ? 4 : 2; }

// Whether the tiles look back through the workspace: else a sequence's tiles are a
// cluster (of 2 .. 8 or 16 blocks), which needs neither it nor a launch before (3 x 1021
// x 201 fp32: 8 us a direction; the launch that clears the words is 4).  Clusters of
// more than two waves of blocks, whose blocks all wait for room together, fall behind.
bool looks(int B, int L, int D, slim_dtype dtype, bool bwd) {
  const int tiles = cdiv(L, kParts * part_steps(element(dtype), bwd));
  const double groups = cdiv(D, 32 * (dtype == SLIM_F32 ? kWidest<float> : kWidest<__nv_bfloat16>));
  return L > kShort && tiles > 1 && (tiles > kMaxCluster || B * groups * tiles > 152.0 * kBlocks * 2);
}

struct ScanWs {
  int* header;
  unsigned long long* sum;
  unsigned* state;  // directly behind the sums
  long long uint4s; // of both
};
ScanWs carve(Carver& cv, int B, int L, int D, slim_dtype dtype, bool bwd) {
  // room for groups of any width
  const size_t words = (size_t)B * cdiv(L, kParts * part_steps(element(dtype), bwd)) * cdiv(D, 64) * 64;
  ScanWs w;
  w.header = cv.take<int>(kHeader);
  w.sum = cv.take<unsigned long long>(words);
  w.state = cv.take<unsigned>(words);
  w.uint4s = (long long)words * 12 / 16;
  return w;
}

struct Call {
  bool bwd;
  void* workspace;
  unsigned* rep;
  cudaStream_t s;
  bool lost;  // diagnostic: nobody runs the sequences' first tiles
};

template <typename T, int V, int KIND, bool BWD>
bool run_tiles(Job j, const Call& call) {
  constexpr int S = part_steps(sizeof(T), BWD), CH = 32 * V, threads = kRun + 32;
  j.groups = cdiv(j.D, CH);
  j.tiles = cdiv(j.L, kParts * S);
  j.streams = (long long)j.B * j.groups;
  int z = 1;
  long long blocks = j.streams;
  const cudaStream_t s = call.s;
  const double e = (double)j.B * j.L * j.D;
  const slim_dtype dtype = sizeof(T) == 4 ? SLIM_F32 : SLIM_BF16;
  const bool look = looks(j.B, j.L, j.D, dtype, BWD);
  if (look) {
    Carver cv(call.workspace);
    const ScanWs w = carve(cv, j.B, j.L, j.D, dtype, BWD);
    j.err = w.header;
    j.tickets = reinterpret_cast<unsigned long long*>(w.header + 4);
    j.sum = w.sum;
    j.state = w.state;
    const long long most = 152 * kBlocks;
    blocks = j.streams * j.tiles < most ? j.streams * j.tiles : most;
    prof::Scope ps(prof::K_SCAN_CLEAR, s);
    const long long n = (w.uint4s + 255) / 256;
    k_scan_clear<<<(unsigned)(n < 152 * 8 ? n : 152 * 8), 256, 0, s>>>(w.header, reinterpret_cast<uint4*>(w.sum),
                                                                       w.uint4s, call.rep, call.lost ? j.streams : 0);
    if (cudaGetLastError() != cudaSuccess) return false;
  } else if (j.tiles > 1) {
    z = j.tiles <= 8 ? j.tiles : kMaxCluster;
    blocks *= z;
  }
  void (*k)(Job);
  if constexpr (BWD)
    k = k_scan_bwd<T, V, S, KIND>;
  else
    k = k_scan_fwd<T, V, S, KIND>;
  const size_t smem = (size_t)kStages * (BWD ? 3 : 2) * kRun * S * V * sizeof(T);  // slots
  static bool flags[kMaxDevices];
  bool* ready = device_flag(flags);
  if (!ready || !*ready) {
    if (cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess ||
        cudaFuncSetAttribute(k, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess)
      return false;
    if (ready) *ready = true;
  }
  prof::Scope ps(BWD ? prof::K_SCAN_BWD : prof::K_SCAN_FWD, s, e * (BWD ? 10 : 4), e * sizeof(T) * (BWD ? 5 : 3));
  return launch_on(k, dim3((unsigned)blocks), threads, smem, z, look, s, j);
}

template <typename T, int V, int KIND>
bool run_as(Job j, const Call& call) {
  const bool bwd = call.bwd;
  const cudaStream_t s = call.s;
  const double e = (double)j.B * j.L * j.D;
  if (j.L <= kShort) {
    prof::Scope ps(bwd ? prof::K_SCAN_BWD : prof::K_SCAN_FWD, s, e * (bwd ? 10 : 4), e * sizeof(T) * (bwd ? 5 : 3));
    const long long n = (long long)j.B * (j.D / V);
    auto k = bwd ? k_scan_short<T, V, KIND, true> : k_scan_short<T, V, KIND, false>;
    k<<<(unsigned)((n + 127) / 128), 128, 0, s>>>(j);
    return cudaGetLastError() == cudaSuccess;
  }
  if constexpr (V <= kWidest<T>)
    return bwd ? run_tiles<T, V, KIND, true>(j, call) : run_tiles<T, V, KIND, false>(j, call);
  return false;
}

template <typename T, int V>
bool run_v(const Job& j, slim_gate kind, const Call& call) {
  if (kind == SLIM_GATE_VALUE) return run_as<T, V, SLIM_GATE_VALUE>(j, call);
  if (kind == SLIM_GATE_LOG) return run_as<T, V, SLIM_GATE_LOG>(j, call);
  return run_as<T, V, SLIM_GATE_SIGMOID>(j, call);
}
// Sequences of up to kShort steps take up to 8 bytes of a step's channels to a thread.
template <typename T>
bool run_t(const Job& j, slim_gate kind, int together, const Call& call) {
  if constexpr (sizeof(T) == 2) {
    if (together >= 4 && j.L <= kShort) return run_v<T, 4>(j, kind, call);
    if (together >= 2) return run_v<T, 2>(j, kind, call);
  } else {
    if (together >= 2 && j.L <= kShort) return run_v<T, 2>(j, kind, call);
  }
  return run_v<T, 1>(j, kind, call);
}
// With arguments checked.
slim_status run(Job& j, slim_dtype dtype, slim_gate kind, int together, bool bwd, void* workspace, size_t bytes,
                cudaStream_t s, bool lost = false) {
  Call call{bwd, workspace, nullptr, s, lost};
  j.chunks = cdiv(j.L, kChunk);
  j.wide = together == (dtype == SLIM_F32 ? 4 : 8);
  size_t need = 0;
  slim_gated_scan_workspace_size(j.B, j.L, j.D, dtype, &need);
  if (need) {
    if (!workspace || bytes < need) return SLIM_ERR_WORKSPACE;
    if (reinterpret_cast<uintptr_t>(workspace) & 255) return SLIM_ERR_INVALID_ARG;
    const slim_status st = report::begin(workspace, true, &call.rep);
    if (st != SLIM_OK) return st;
    // (a direction that does not look back clears the error word, too)
    j.err = static_cast<int*>(workspace);
  } else if (workspace) {
    const slim_status st = report::pending(workspace);
    if (st != SLIM_OK) return st;
  }
  const bool ok = dtype == SLIM_F32 ? run_t<float>(j, kind, together, call)
                                    : run_t<__nv_bfloat16>(j, kind, together, call);
  return ok ? SLIM_OK : SLIM_ERR_CUDA;
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

extern "C" slim_status slim_gated_scan_workspace_size(int B, int L, int D, slim_dtype dtype,
                                                      size_t* bytes) {
  using namespace slim::layer;
  if (!bytes || !sizes_ok(B, L, D, dtype, SLIM_GATE_VALUE)) return SLIM_ERR_INVALID_ARG;
  *bytes = 0;
  for (int bwd = 0; B > 0 && bwd < 2; ++bwd) {
    if (!looks(B, L, D, dtype, bwd)) continue;
    slim::Carver cv(nullptr);
    carve(cv, B, L, D, dtype, bwd);
    if (cv.bytes() > *bytes) *bytes = cv.bytes();
  }
  return SLIM_OK;
}

extern "C" slim_status slim_gated_scan_fwd(const void* gate, long long gate_pitch, const void* x,
                                           long long x_pitch, const float* h0, int B, int L, int D,
                                           slim_dtype dtype, slim_gate kind, void* h, float* last,
                                           float* kept, void* workspace,
                                           size_t workspace_bytes, void* stream) {
  using namespace slim::layer;
  if (!sizes_ok(B, L, D, dtype, kind)) return SLIM_ERR_INVALID_ARG;
  if (!fp32_ok(h0) || !fp32_ok(last) || !fp32_ok(kept)) return SLIM_ERR_INVALID_ARG;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (B == 0 || L == 0) return pass_on(h0, last, (size_t)B * D, s);
  const int es = dtype == SLIM_F32 ? 4 : 2;
  int together = 16 / es;  // channels: as many as all rows can move in one piece
  while (D % together) together /= 2;
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
  return run(j, dtype, kind, together, false, workspace, workspace_bytes, s);
}

extern "C" slim_status slim_gated_scan_bwd(const void* gate, long long gate_pitch, const void* x,
                                           long long x_pitch, const float* kept, const void* dh,
                                           const float* dlast, int B, int L, int D, slim_dtype dtype,
                                           slim_gate kind, void* dgate, long long dgate_pitch,
                                           void* dx, long long dx_pitch, float* dh0,
                                           void* workspace, size_t workspace_bytes, void* stream) {
  using namespace slim::layer;
  if (!sizes_ok(B, L, D, dtype, kind)) return SLIM_ERR_INVALID_ARG;
  if (!fp32_ok(dlast) || !fp32_ok(dh0) || !fp32_ok(kept)) return SLIM_ERR_INVALID_ARG;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (B == 0 || L == 0) return pass_on(dlast, dh0, (size_t)B * D, s);
  const int es = dtype == SLIM_F32 ? 4 : 2;
  int together = 16 / es;  // channels: as many as all rows can move in one piece
  while (D % together) together /= 2;
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
  return run(j, dtype, kind, together, true, workspace, workspace_bytes, s);
}

extern "C" slim_status slim_diag_gated_scan_wait(const float* gate, const float* x, int L, int D, float* h,
                                                 void* workspace, size_t workspace_bytes, void* stream) {
  using namespace slim::layer;
  if (!sizes_ok(1, L, D, SLIM_F32, SLIM_GATE_LOG) || !looks(1, L, D, SLIM_F32, false)) return SLIM_ERR_INVALID_ARG;
  int together = 4;
  while (D % together) together /= 2;
  for (const Rows& r : {Rows{gate, D, false}, Rows{x, D, false}, Rows{h, D, true}})
    if (!rows_ok(r, 1, L, D, 4, &together)) return SLIM_ERR_INVALID_ARG;
  Job j{};
  j.gate = gate;
  j.x = x;
  j.gate_pitch = j.x_pitch = j.D = D;
  j.h = h;
  j.B = 1;
  j.L = L;
  return run(j, SLIM_F32, SLIM_GATE_LOG, together, false, workspace, workspace_bytes,
             static_cast<cudaStream_t>(stream), true);
}
