// Norms of queries and keys per head with the rotation by position, and their
// gradients.  Contract: include/slim_layer.h.
//
// A row of one token and head is held by 1 to 32 lanes, two vectors of up to 16 bytes
// each: in the split layout the lower and upper members of some pairs, so that a pair
// never leaves its lane.  The row's sums (of squares, and backward of g x) go over its
// lanes by shuffles; nothing else is exchanged.
//
// Angles are fractions of a turn in 64-bit fixed point: position * frequency
// mod 1 is one integer product whose overflow is the reduction.  A block takes
// the turns of its tokens once, for all heads, from shared memory.
//
// Backward, with r = 1 / sqrt(mean(x^2) + eps), n = r x and dz the incoming
// gradient turned back and scaled:
//     dweight = sum dz n,   g = weight dz,   dx = r (g - n mean(g n)).
// The weights' sums stay in registers while a block walks over its rows, leave
// it once, and are joined over blocks in order by a second kernel.
//
// Each row is read and written once.  HBM bounds fp32: 4 x 12+12 x 8192 x 64 backward
// 100 us, 6.0 TB/s.  bf16 waits for its instructions (23 an element, of which 3 for the
// turns) beside the copies: 8 x 8+8 x 4096 x 64 forward 31 us, 4.3 TB/s.  With turns
// that four lanes met in one bank for the latter took 49 us.
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

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kMaxD = 256, kMaxPairs = kMaxD / 2;
constexpr int kMaxTokens = 16;       // of a tile
constexpr int kMaxHeads = 4096;
constexpr float kMaxEps = 1e38f;     // beside a mean square below 1e38 still in range
constexpr int kBwdBlocks = 152 * 3;  // most that are resident; the workspace is for as many

struct Side {
  const void *x, *dy;  // dy: backward
  void* out;           // y, or dx
  slim_strides xs, dys, os;
  const float* w;
  float* part;         // [blocks of this side][d], or null
  int H;
  unsigned by_head;    // ceil(2^32 / H): row / H is a product
  int blocks;
};
struct Job {
  Side side[2];
  const void* positions;
  int i64, tokens, L, d, half, interleaved;
  int tile;            // tokens of a tile
  unsigned by_heads, by_half;  // ceil(2^32 / (both sides' heads)), / half
  float eps, scale;
  unsigned long long turn[kMaxPairs];  // frequencies, 2^64 = one turn per position
};
struct WeightJob {
  const float* part[2];
  float* out[2];
  int blocks[2], d;
};

// cos and sin of turn / 2^64 turns: the nearest quarter turn is taken off first, which
// leaves at most an eighth, in fp32 off by at most 2^-28 of a turn (its rounding; the
// lower half of `turn` is cut off, 2^-32).
__device__ __forceinline__ float2 cos_sin(unsigned long long turn) {
  const unsigned t = (unsigned)(turn >> 32), q = (t + 0x20000000u) >> 30;
  const float rest = (float)(int)(t - (q << 30)) * 0x1p-31f;  // half turns
  float s, c;
  sincospif(rest, &s, &c);
  if (q & 1) {
    const float u = c;
    c = -s;
    s = u;
  }
  return q & 2 ? make_float2(-c, -s) : make_float2(c, s);
}

// How a lane holds its 2 W values, two vectors of W: SPLIT, the lower and the upper
// members of W pairs; INTER, W pairs one behind the other; ANY, by elements, any layout
// and alignment.  Behind the turned features both are 2 W of them in a row.
enum { ANY = 0, SPLIT = 1, INTER = 2 };
template <typename T, int MODE, int W> struct Row {
  static constexpr int N = 2 * W;
  using Raw = typename std::conditional<W * sizeof(T) == 16, uint4, uint2>::type;
  struct Held {  // a row as it lies in memory
    Raw v[MODE == ANY ? 1 : 2];
    T e[MODE == ANY ? N : 1];
  };
  // feature of the lane's value i, lanes holding pairs W g ..
  static __device__ __forceinline__ int at(const Job& j, int g, int i) {
    if (MODE == INTER) return N * g + i;
    if (MODE == SPLIT) return W * g < j.half ? W * g + i % W + (i >= W ? j.half : 0) : N * g + i;
    const int p = W * g + i % W, up = i / W;
    if (p >= j.half || j.interleaved) return 2 * p + up;
    return p + (up ? j.half : 0);
  }
  static __device__ __forceinline__ bool turned(const Job& j, int g, int i) {
    return W * g + (MODE == ANY ? i : 0) < j.half;
  }
  static __device__ __forceinline__ void fetch(const Job& j, const T* row, int g, bool on, Held& h) {
    if constexpr (MODE == ANY) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int e = at(j, g, i);
        h.e[i] = on && e < j.d ? row[e] : T(0.0f);
      }
    } else if (on) {
      h.v[0] = *reinterpret_cast<const Raw*>(row + at(j, g, 0));
      h.v[1] = *reinterpret_cast<const Raw*>(row + at(j, g, W));
    } else {
      h.v[0] = h.v[1] = Raw{};
    }
  }
  static __device__ __forceinline__ void values(const Held& h, float* v) {
    if constexpr (MODE == ANY) {
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] = Io<T>::load(h.e, i);
    } else {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const uint32_t* u = reinterpret_cast<const uint32_t*>(&h.v[k]);
#pragma unroll
        for (int i = 0; i < (int)(W * sizeof(T) / 4); ++i) {
          if constexpr (sizeof(T) == 4)
            v[W * k + i] = __uint_as_float(u[i]);
          else
            tc::unpack_bf16(u[i], v[W * k + 2 * i], v[W * k + 2 * i + 1]);
        }
      }
    }
  }
  static __device__ __forceinline__ void store(const Job& j, T* row, int g, const float* v) {
    if constexpr (MODE == ANY) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int e = at(j, g, i);
        if (e < j.d) Io<T>::store(row, e, v[i]);
      }
    } else {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        Raw r;
        uint32_t* u = reinterpret_cast<uint32_t*>(&r);
#pragma unroll
        for (int i = 0; i < (int)(W * sizeof(T) / 4); ++i)
          u[i] = sizeof(T) == 4 ? __float_as_uint(v[W * k + i]) : tc::pack_bf16(v[W * k + 2 * i], v[W * k + 2 * i + 1]);
        *reinterpret_cast<Raw*>(row + at(j, g, W * k)) = r;
      }
    }
  }
  // sum of a b: by four pairs at a time, as lanes of narrower vectors hold them, so that
  // the bits of a row in the split layout that is turned as a whole do not depend on its
  // alignment (others' features meet in other lanes, or in another order by elements)
  static __device__ __forceinline__ float dot(const float* a, const float* b) {
    float sum[W / 4];
#pragma unroll
    for (int k = 0; k < W / 4; ++k) {
      sum[k] = 0.0f;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int e = MODE == INTER ? 8 * k + i : 4 * k + i % 4 + (i >= 4 ? W : 0);
        sum[k] = fmaf(a[e], b[e], sum[k]);
      }
    }
    return W == 8 ? sum[0] + sum[W / 4 - 1] : sum[0];
  }
  // the members of the lane's pair i
  static __device__ __forceinline__ float& low(float* v, int i) { return v[MODE == INTER ? 2 * i : i]; }
  static __device__ __forceinline__ float& high(float* v, int i) { return v[MODE == INTER ? 2 * i + 1 : i + W]; }
};

__device__ __forceinline__ float over_lanes(float v, int G) {
  for (int o = 1; o < G; o <<= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

struct TokenAt {
  long long x, dy, out;
};

// Of an SM: two vectors of 8 values, their gradients and sums fill a thread's registers.
constexpr int bwd_blocks(int W) { return W == 8 ? 2 : 3; }

// The turns of a tile's tokens lie in shared memory, for all heads.  Forward, a block has
// both sides' heads; backward one side's, whose weights' sums it keeps.  The next row is
// on its way while one is at work, the first under the turns.
//
// A token's turns are in the order in which lanes read them, two pairs at a time: the
// lanes of a row side by side (pair after pair, four lanes met in one bank).
template <typename T, int MODE, int W, bool BWD>
__global__ void __launch_bounds__(kThreads, BWD ? bwd_blocks(W) : 3) k_qk_norm(const __grid_constant__ Job j, int lanes_log2) {
  using R = Row<T, MODE, W>;
  constexpr int N = 2 * W;
  extern __shared__ float4 turns[];  // [tile][W / 2][rim]
  __shared__ TokenAt token[BWD ? 1 : 2][kMaxTokens];
  __shared__ long long position[kMaxTokens];
  __shared__ __align__(16) float weight[BWD ? 1 : 2][kMaxD];  // times scale
  __shared__ unsigned long long frequency[kMaxPairs];
  const int mine = BWD && blockIdx.x >= j.side[0].blocks;
  const Side& s = j.side[mine];
  const int block = blockIdx.x - (mine ? j.side[0].blocks : 0);
  const int H = BWD ? s.H : j.side[0].H + j.side[1].H;
  const int G = 1 << lanes_log2, g = threadIdx.x & (G - 1);
  const int first = threadIdx.x >> lanes_log2, step = kThreads >> lanes_log2;
  const int rim = (j.half + W - 1) / W;  // lanes with turned pairs
  const bool lane_on = N * g < j.d;
  const float over_d = 1.0f / j.d;
  // (lanes that read different parameters wait for each other: once a block, not a turn)
  if (threadIdx.x < j.half) frequency[threadIdx.x] = j.turn[threadIdx.x];
  if (!BWD && threadIdx.x < j.d)
    for (int k = 0; k < 2; ++k) weight[k][threadIdx.x] = (j.side[k].w ? j.side[k].w[threadIdx.x] : 1.0f) * j.scale;
  float w[BWD ? N : 1], dw[BWD ? N : 1];
  if (BWD) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int e = R::at(j, g, i);
      w[i] = (lane_on && e < j.d ? (s.w ? s.w[e] : 1.0f) : 0.0f) * j.scale;
      dw[i] = 0.0f;
    }
  }
  const int tiles = (j.tokens + j.tile - 1) / j.tile;
  for (int tile = block; tile < tiles; tile += s.blocks) {
    const int n0 = tile * j.tile, count = min(j.tile, j.tokens - n0);
    const int rows = count * H;
    __syncthreads();
    if (threadIdx.x < count) {
      const int n = n0 + threadIdx.x, b = n / j.L, l = n - b * j.L;
      position[threadIdx.x] = !j.positions ? l
                              : j.i64      ? static_cast<const long long*>(j.positions)[n]
                                           : static_cast<const int*>(j.positions)[n];
      for (int k = 0; k < (BWD ? 1 : 2); ++k) {
        const Side& t = j.side[BWD ? mine : k];
        token[k][threadIdx.x] = TokenAt{b * t.xs.b + l * t.xs.l, BWD ? b * t.dys.b + l * t.dys.l : 0,
                                        b * t.os.b + l * t.os.l};
      }
    }
    __syncthreads();
    // a row's token, side (of the block's) and head
    auto place = [&](int r, int& t, int& k, int& h) {
      r = r < rows ? r : 0;
      t = H == 1 ? r : (int)__umulhi((unsigned)r, BWD ? s.by_head : j.by_heads);
      h = r - t * H;
      k = !BWD && h >= j.side[0].H;
      if (k) h -= j.side[0].H;
    };
    typename R::Held hx, hy;
    auto fetch = [&](int r) {
      int t, k, h;
      place(r, t, k, h);
      const bool on = r < rows && lane_on;
      const Side& of = BWD ? s : k ? j.side[1] : j.side[0];
      R::fetch(j, static_cast<const T*>(of.x) + token[k][t].x + h * of.xs.h, g, on, hx);
      if (BWD) R::fetch(j, static_cast<const T*>(s.dy) + token[0][t].dy + h * s.dys.h, g, on, hy);
    };
    fetch(first);
    for (int i = threadIdx.x; i < count * j.half; i += kThreads) {
      const int t = j.half == 1 ? i : (int)__umulhi((unsigned)i, j.by_half), p = i - t * j.half, v = p % W;
      const float2 cs = cos_sin((unsigned long long)position[t] * frequency[p]);
      reinterpret_cast<float2*>(turns)[(t * (W / 2) + v / 2) * rim * 2 + p / W * 2 + v % 2] = cs;
    }
    __syncthreads();
    // whole warps walk together: their lanes exchange sums
    for (int r0 = first; r0 - first < rows; r0 += step) {
      float x[N], dz[BWD ? N : 1];
      R::values(hx, x);
      if constexpr (BWD) R::values(hy, dz);
      if (r0 + step - first < rows) fetch(r0 + step);
      int t, k, h;
      place(r0, t, k, h);
      float ss = over_lanes(R::dot(x, x), G);
      float fit = 1.0f;
      if (__any_sync(0xffffffffu, !(ss <= 1e38f))) {
        // squares past fp32's range: the row, and eps by their square, in smaller units
        if (!(ss <= 1e38f)) fit = 0x1p-80f;
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] *= fit;
        ss = over_lanes(R::dot(x, x), G);
      }
      const float rms = rsqrtf(fmaf(ss, over_d, j.eps * fit * fit));
#pragma unroll
      for (int i = 0; i < N; ++i) x[i] *= rms;
      if constexpr (!BWD) {
        if (MODE == ANY) {
#pragma unroll
          for (int i = 0; i < N; ++i) x[i] *= weight[k][min(R::at(j, g, i), kMaxD - 1)];
        } else if (lane_on) {
#pragma unroll
          for (int i = 0; i < N; i += 4) {
            const float4 f = *reinterpret_cast<const float4*>(&weight[k][R::at(j, g, i)]);
            x[i] *= f.x;
            x[i + 1] *= f.y;
            x[i + 2] *= f.z;
            x[i + 3] *= f.w;
          }
        }
      }
      if (W * g < j.half) {
        const float4* turn = turns + t * (W / 2) * rim + g;
#pragma unroll
        for (int i = 0; i < W; i += 2) {
          const float4 two = turn[i / 2 * rim];
#pragma unroll
          for (int v = 0; v < 2; ++v) {
            const float c = v ? two.z : two.x, sn = (v ? two.w : two.y) * (BWD ? -1.0f : 1.0f);
            float* y;
            if constexpr (BWD)
              y = dz;
            else
              y = x;
            if (MODE == ANY && !R::turned(j, g, i + v)) continue;
            float &a = R::low(y, i + v), &b = R::high(y, i + v);
            const float u = a;
            a = fmaf(u, c, -b * sn);
            b = fmaf(u, sn, b * c);
          }
        }
      }
      if constexpr (BWD) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
          dw[i] = fmaf(dz[i], x[i], dw[i]);
          dz[i] *= w[i];
        }
        const float gn = over_lanes(R::dot(dz, x), G) * over_d;
        const float out = fit * rms;
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = out * fmaf(-x[i], gn, dz[i]);
      }
      const Side& of = BWD ? s : k ? j.side[1] : j.side[0];
      if (r0 < rows && lane_on) R::store(j, static_cast<T*>(of.out) + token[k][t].out + h * of.os.h, g, x);
    }
  }
  if (!BWD || !s.part) return;
  // the block's sums: rows of a warp, then warps in order
  __shared__ float sum[kWarps][kMaxD];
  const int warp = threadIdx.x >> 5;
  if constexpr (BWD) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      for (int o = 16; o >= G; o >>= 1) dw[i] += __shfl_xor_sync(0xffffffffu, dw[i], o);
      const int e = R::at(j, g, i);
      if ((threadIdx.x & 31) < G && lane_on && e < j.d) sum[warp][e] = dw[i] * j.scale;
    }
  }
  __syncthreads();
  if (threadIdx.x < j.d) {
    float v = 0.0f;
#pragma unroll
    for (int i = 0; i < kWarps; ++i) v += sum[i][threadIdx.x];
    s.part[(size_t)block * j.d + threadIdx.x] = v;
  }
}

// The weights' gradients from the blocks' sums: 32 features a block, 32 threads each.
__global__ void __launch_bounds__(1024) k_qk_weights(WeightJob j) {
  tc::grid_dependency_wait();
  __shared__ float sh[32][33];
  const int which = blockIdx.y, col = threadIdx.x & 31, q = threadIdx.x >> 5;
  const int e = blockIdx.x * 32 + col, n = j.blocks[which];
  if (!j.out[which]) return;
  float v = 0.0f;
  const int per = (n + 31) / 32, to = min((q + 1) * per, n);
  if (e < j.d) {
#pragma unroll 8
    for (int b = q * per; b < to; ++b) v += j.part[which][(size_t)b * j.d + e];
  }
  sh[col][q] = v;
  __syncthreads();
  // a warp a feature: its lanes' sums in a fixed tree
  v = sh[q][col];
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  if (col == 0 && blockIdx.x * 32 + q < j.d) j.out[which][blockIdx.x * 32 + q] = v;
}

// ------------------------------------------------------------------ host
bool sizes_ok(int B, int Hq, int Hk, int L, int d) {
  if (B < 0 || L < 0 || (long long)B * L >= (1LL << 31) - kMaxTokens) return false;
  if (Hq < 1 || Hq > kMaxHeads || Hk < 0 || Hk > kMaxHeads || d < 1 || d > kMaxD) return false;
  return (long long)B * L * (Hq + Hk) <= (1LL << 40);
}

constexpr long long kMaxStride = 1LL << 40;
slim_strides strides_of(const slim_strides* s, int H, int L, int d) {
  if (s) return *s;
  return slim_strides{(long long)H * L * d, (long long)L * d, d};
}
bool strides_ok(const slim_strides& s, int B, int H, int L) {
  for (long long v : {s.b, s.h, s.l})
    if (v < 0 || v > kMaxStride) return false;
  return (double)s.b * (B - 1) + (double)s.h * (H - 1) + (double)s.l * (L - 1) < 0x1p60;
}
// No two elements of a [B, H, L, d] tensor in one place: each dimension steps past
// everything the smaller steps reach.
bool apart(const slim_strides& s, int B, int H, int L, int d) {
  long long step[3] = {s.b, s.h, s.l}, n[3] = {B, H, L}, reach = d;
  for (int i = 0; i < 3; ++i)
    for (int k = i + 1; k < 3; ++k)
      if (step[k] < step[i]) {
        const long long a = step[i], b = n[i];
        step[i] = step[k];
        n[i] = n[k];
        step[k] = a;
        n[k] = b;
      }
  for (int i = 0; i < 3; ++i) {
    if (n[i] <= 1) continue;
    if (step[i] < reach) return false;
    reach += (n[i] - 1) * step[i];
  }
  return true;
}

struct Operand {  // of a side: x, dy or out
  const void* p;
  const slim_strides* s;
};

// What all rows of all tensors can be moved in: elements, up to 16 bytes.
struct Layout {
  int together;
};
void fit(Layout* in, const void* p, const slim_strides& s, int es) {
  while (in->together > 1 && ((reinterpret_cast<uintptr_t>(p) & (in->together * es - 1)) ||
                              ((s.b | s.h | s.l) & (in->together - 1))))
    in->together /= 2;
}

// i / n is the upper half of i * by(n) for small i, n > 1.
unsigned by(int n) { return n <= 1 ? 0u : (unsigned)(((1ull << 32) + n - 1) / n); }

bool fill_side(Side* t, const Operand& x, const Operand* dy, const Operand& out, const float* w, int B,
               int H, int L, int d, int es, Layout* in) {
  t->H = H;
  if (H == 0) return true;
  t->by_head = by(H);
  const Operand none{nullptr, nullptr};
  const Operand* all[3] = {&x, dy ? dy : &none, &out};
  slim_strides* to[3] = {&t->xs, &t->dys, &t->os};
  for (int i = 0; i < 3; ++i) {
    if (i == 1 && !dy) continue;
    if (!all[i]->p || (reinterpret_cast<uintptr_t>(all[i]->p) & (es - 1))) return false;
    *to[i] = strides_of(all[i]->s, H, L, d);
    if (!strides_ok(*to[i], B, H, L)) return false;
    fit(in, all[i]->p, *to[i], es);
  }
  if (!apart(t->os, B, H, L, d)) return false;
  if (w && (reinterpret_cast<uintptr_t>(w) & 3)) return false;
  t->x = x.p;
  t->dy = dy ? dy->p : nullptr;
  t->out = const_cast<void*>(out.p);
  t->w = w;
  return true;
}

template <typename T, int MODE, int W, bool BWD>
void start(const Job& j, unsigned blocks, cudaStream_t s) {
  int lanes_log2 = 0;
  while ((2 * W << lanes_log2) < j.d) ++lanes_log2;
  const size_t smem = (size_t)j.tile * ((j.half + W - 1) / W) * (W / 2) * sizeof(float4);
  k_qk_norm<T, MODE, W, BWD><<<blocks, kThreads, smem, s>>>(j, lanes_log2);
}
// Values of a vector that all rows can be moved in, 0: elements.
template <typename T>
int vectors(const Job& j, const Layout& in) {
  constexpr int whole = 16 / sizeof(T);
  if (in.together < 4 || j.d % 8 || j.half % 4) return 0;
  return in.together >= whole && j.d % (2 * whole) == 0 && j.half % whole == 0 ? whole : 4;
}
template <typename T, bool BWD>
bool run(const Job& j, const Layout& in, cudaStream_t s) {
  const unsigned blocks = (unsigned)(j.side[0].blocks + (BWD ? j.side[1].blocks : 0));
  const double n = (double)j.tokens * (j.side[0].H + j.side[1].H) * j.d;
  prof::Scope ps(prof::K_QK_NORM, s, n * (BWD ? 20 : 8), n * sizeof(T) * (BWD ? 3 : 2));
  const int w = vectors<T>(j, in);
  if (w == 0)
    start<T, ANY, 4, BWD>(j, blocks, s);
  else if (w == 4)
    j.interleaved ? start<T, INTER, 4, BWD>(j, blocks, s) : start<T, SPLIT, 4, BWD>(j, blocks, s);
  else
    j.interleaved ? start<T, INTER, 16 / sizeof(T), BWD>(j, blocks, s) : start<T, SPLIT, 16 / sizeof(T), BWD>(j, blocks, s);
  return cudaGetLastError() == cudaSuccess;
}

// Tokens of a tile and the blocks of either side: tiles of up to kMaxTokens, fewer
// where there would not be four blocks an SM, and at most `most` blocks (0: one a
// tile) shared by the sides as their rows are.
void deal(Job* j, int most) {
  const int H = j->side[0].H + j->side[1].H;
  int tile = kMaxTokens;
  while (tile > 1 && ((j->tokens + tile - 1) / tile < 152 * 2 || (long long)tile * H > 2 * kMaxHeads))
    tile /= 2;
  j->tile = tile;
  const int tiles = (j->tokens + tile - 1) / tile;
  for (int i = 0; i < 2; ++i) {
    int n = tiles;
    if (most) {
      const int share = (int)((long long)most * j->side[i].H / H);
      if (n > share) n = share > 0 ? share : 1;
    }
    j->side[i].blocks = j->side[i].H ? n : 0;
  }
}

}  // namespace
}  // namespace layer
}  // namespace slim

extern "C" slim_status slim_qk_norm_bwd_workspace_size(int B, int Hq, int Hk, int L, int d,
                                                       size_t* bytes) {
  using namespace slim::layer;
  if (!bytes || !sizes_ok(B, Hq, Hk, L, d)) return SLIM_ERR_INVALID_ARG;
  // a side has at most its share of the blocks, or one
  *bytes = ((size_t)(kBwdBlocks + 2) * d * sizeof(float) + 255) & ~size_t(255);
  return SLIM_OK;
}

namespace slim {
namespace layer {
namespace {
// Checks and fills what both directions share.  0: nothing to do, 1: go on, -1: refused.
int set_up(Job* j, const Operand q[3], const Operand k[3], bool bwd, const float* wq, const float* wk,
           const void* positions, slim_index ptype, const double* inv_freq, int rotary,
           int interleaved, int B, int Hq, int Hk, int L, int d, slim_dtype dtype, float eps,
           float scale, Layout* in) {
  if (!sizes_ok(B, Hq, Hk, L, d) || (dtype != SLIM_F32 && dtype != SLIM_BF16)) return -1;
  if (rotary < 0 || rotary > d || (rotary & 1) || (interleaved & ~1)) return -1;
  if (rotary > 0 && (!inv_freq || (ptype != SLIM_I32 && ptype != SLIM_I64))) return -1;
  if (!(eps > 0.0f) || !(eps <= kMaxEps) || !isfinite(scale)) return -1;
  for (int p = 0; p < rotary / 2; ++p) {
    if (!isfinite(inv_freq[p])) return -1;
    double turn = inv_freq[p] * 0.15915494309189533577;
    turn -= floor(turn);
    // turn = 1 - 2^-54 and the like would round to a whole one, which is none
    const double scaled = turn * 0x1p64;
    j->turn[p] = scaled >= 0x1p64 ? 0ull : (unsigned long long)scaled;
  }
  if ((long long)B * L == 0) return 0;
  const int es = dtype == SLIM_F32 ? 4 : 2;
  in->together = 16 / es;
  if (!fill_side(&j->side[0], q[0], bwd ? &q[1] : nullptr, q[2], wq, B, Hq, L, d, es, in) ||
      !fill_side(&j->side[1], k[0], bwd ? &k[1] : nullptr, k[2], wk, B, Hk, L, d, es, in))
    return -1;
  if (positions && (reinterpret_cast<uintptr_t>(positions) & (ptype == SLIM_I64 ? 7 : 3))) return -1;
  j->positions = positions;
  j->i64 = ptype == SLIM_I64;
  j->tokens = B * L;
  j->L = L;
  j->d = d;
  j->half = rotary / 2;
  j->by_heads = by(Hq + Hk);
  j->by_half = by(rotary / 2);
  j->interleaved = interleaved;
  j->eps = eps;
  j->scale = scale;
  return 1;
}
}  // namespace
}  // namespace layer
}  // namespace slim

extern "C" slim_status slim_qk_norm_fwd(const void* q, const slim_strides* q_strides, const void* k,
                                        const slim_strides* k_strides, const float* q_weight,
                                        const float* k_weight, const void* positions,
                                        slim_index ptype, const double* inv_freq, int rotary,
                                        int interleaved, int B, int Hq, int Hk, int L, int d,
                                        slim_dtype dtype, float eps, float scale, void* q_out,
                                        const slim_strides* q_out_strides, void* k_out,
                                        const slim_strides* k_out_strides, void* stream) {
  using namespace slim::layer;
  Job j{};
  Layout in;
  const Operand qs[3] = {{q, q_strides}, {}, {q_out, q_out_strides}};
  const Operand ks[3] = {{k, k_strides}, {}, {k_out, k_out_strides}};
  const int go = set_up(&j, qs, ks, false, q_weight, k_weight, positions, ptype, inv_freq, rotary,
                        interleaved, B, Hq, Hk, L, d, dtype, eps, scale, &in);
  if (go <= 0) return go < 0 ? SLIM_ERR_INVALID_ARG : SLIM_OK;
  deal(&j, 0);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const bool ok = dtype == SLIM_F32 ? run<float, false>(j, in, s)
                                    : run<__nv_bfloat16, false>(j, in, s);
  return ok ? SLIM_OK : SLIM_ERR_CUDA;
}

extern "C" slim_status slim_qk_norm_bwd(
    const void* q, const slim_strides* q_strides, const void* k, const slim_strides* k_strides,
    const float* q_weight, const float* k_weight, const void* positions, slim_index ptype,
    const double* inv_freq, int rotary, int interleaved, int B, int Hq, int Hk, int L, int d,
    slim_dtype dtype, float eps, float scale, const void* dq_out, const slim_strides* dq_out_strides,
    const void* dk_out, const slim_strides* dk_out_strides, void* dq, const slim_strides* dq_strides,
    void* dk, const slim_strides* dk_strides, float* dq_weight, float* dk_weight, void* workspace,
    size_t workspace_bytes, void* stream) {
  using namespace slim::layer;
  Job j{};
  Layout in;
  const Operand qs[3] = {{q, q_strides}, {dq_out, dq_out_strides}, {dq, dq_strides}};
  const Operand ks[3] = {{k, k_strides}, {dk_out, dk_out_strides}, {dk, dk_strides}};
  for (const float* p : {dq_weight, dk_weight})
    if (reinterpret_cast<uintptr_t>(p) & 3) return SLIM_ERR_INVALID_ARG;
  const int go = set_up(&j, qs, ks, true, q_weight, k_weight, positions, ptype, inv_freq, rotary,
                        interleaved, B, Hq, Hk, L, d, dtype, eps, scale, &in);
  if (go < 0) return SLIM_ERR_INVALID_ARG;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (go == 0 || Hk == 0) {
    // weights whose gradient no row reaches
    float* none[2] = {go == 0 ? dq_weight : nullptr, dk_weight};
    for (float* p : none)
      if (p && cudaMemsetAsync(p, 0, d * sizeof(float), s) != cudaSuccess) return SLIM_ERR_CUDA;
    if (go == 0) return SLIM_OK;
  }
  size_t need = 0;
  slim_qk_norm_bwd_workspace_size(B, Hq, Hk, L, d, &need);
  if (!workspace || workspace_bytes < need) return SLIM_ERR_WORKSPACE;
  if (reinterpret_cast<uintptr_t>(workspace) & 255) return SLIM_ERR_INVALID_ARG;
  const int width = dtype == SLIM_F32 ? vectors<float>(j, in) : vectors<__nv_bfloat16>(j, in);
  deal(&j, 152 * bwd_blocks(width));
  float* part = static_cast<float*>(workspace);
  WeightJob wj{};
  wj.d = d;
  float* out[2] = {dq_weight, Hk ? dk_weight : nullptr};
  for (int i = 0; i < 2; ++i) {
    wj.part[i] = part;
    wj.out[i] = out[i];
    wj.blocks[i] = j.side[i].blocks;
    j.side[i].part = out[i] ? part : nullptr;
    part += (size_t)j.side[i].blocks * d;
  }
  const bool ok = dtype == SLIM_F32 ? run<float, true>(j, in, s)
                                    : run<__nv_bfloat16, true>(j, in, s);
  if (!ok) return SLIM_ERR_CUDA;
  if (out[0] || out[1]) {
    slim::prof::Scope ps(slim::prof::K_QK_WEIGHTS, s);
    if (!slim::launch_on(k_qk_weights, dim3((d + 31) / 32, 2), 1024, 0, 1, true, s, wj))
      return SLIM_ERR_CUDA;
  }
  return SLIM_OK;
}
