// Norms of queries and keys per head with the rotation by position, and their
// gradients.  Contract: include/slim_layer.h.
//
// A row of one token and head is held by 1 to 32 lanes, eight features each, as
// two vectors of four: in the split layout the lower and upper member of four
// pairs, so that a pair never leaves its lane.  The row's sums (of squares, and
// backward of g x) go over its lanes by shuffles; nothing else is exchanged.
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
// HBM bounds it: each row is read and written once.
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

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kMaxD = 256, kMaxPairs = kMaxD / 2;
constexpr int kMaxTokens = 16;       // of a tile
constexpr int kMaxHeads = 4096;
constexpr int kBwdBlocks = 152 * 4;  // all of them resident; the workspace is for as many

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
  float eps, scale;
  unsigned long long turn[kMaxPairs];  // frequencies, 2^64 = one turn per position
};
struct WeightJob {
  const float* part[2];
  float* out[2];
  int blocks[2], d;
};

// cos and sin of turn / 2^64 turns: the nearest quarter turn is taken off first,
// which leaves at most an eighth, exact to 2^-33 of a turn in fp32.
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

// MODE 0: any layout and alignment, by elements; 1: split pairs, 2: interleaved
// pairs, both in vectors of four.
enum { ANY = 0, SPLIT = 1, INTER = 2 };
template <typename T, int MODE> struct Row {
  // feature of the lane's value i, lanes holding pairs 4 g ..
  static __device__ __forceinline__ int at(const Job& j, int g, int i) {
    if (MODE == INTER) return 8 * g + i;
    if (MODE == SPLIT) return 4 * g < j.half ? 4 * g + (i & 3) + (i & 4 ? j.half : 0) : 8 * g + i;
    const int p = 4 * g + (i & 3), up = i >> 2;
    if (p >= j.half || j.interleaved) return 2 * p + up;
    return p + (up ? j.half : 0);
  }
  static __device__ __forceinline__ void load4(const T* p, float* v) {
    if constexpr (sizeof(T) == 4) {
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
  static __device__ __forceinline__ void store4(T* p, const float* v) {
    if constexpr (sizeof(T) == 4)
      *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
    else
      *reinterpret_cast<uint2*>(p) =
          make_uint2(tc::pack_bf16(v[0], v[1]), tc::pack_bf16(v[2], v[3]));
  }
  static __device__ __forceinline__ void load(const Job& j, const T* row, int g, bool on, float* v) {
    if (MODE == ANY) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int e = at(j, g, i);
        v[i] = on && e < j.d ? Io<T>::load(row, e) : 0.0f;
      }
    } else if (on) {
      load4(row + at(j, g, 0), v);
      load4(row + at(j, g, 4), v + 4);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = 0.0f;
    }
  }
  static __device__ __forceinline__ void store(const Job& j, T* row, int g, const float* v) {
    if (MODE == ANY) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int e = at(j, g, i);
        if (e < j.d) Io<T>::store(row, e, v[i]);
      }
    } else {
      store4(row + at(j, g, 0), v);
      store4(row + at(j, g, 4), v + 4);
    }
  }
  // the lane's pairs turned (sign 1) or turned back (-1)
  static __device__ __forceinline__ void rotate(const Job& j, const float2* turns, int g, float sign,
                                                float* v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (4 * g + (MODE == ANY ? i : 0) >= j.half) break;
      const float2 cs = turns[4 * g + i];
      float& a = MODE == INTER ? v[2 * i] : v[i];
      float& b = MODE == INTER ? v[2 * i + 1] : v[i + 4];
      const float s = sign * cs.y, x = a;
      a = fmaf(x, cs.x, -b * s);
      b = fmaf(x, s, b * cs.x);
    }
  }
};

__device__ __forceinline__ float over_lanes(float v, int G) {
  for (int o = G >> 1; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

struct TokenAt {
  long long x, dy, out;
};

template <typename T, int MODE, bool BWD>
__global__ void __launch_bounds__(kThreads) k_qk_norm(const __grid_constant__ Job j, int lanes_log2) {
  using R = Row<T, MODE>;
  extern __shared__ float2 turns[];  // [tile][half]
  __shared__ TokenAt token[kMaxTokens];
  const int which = blockIdx.x >= j.side[0].blocks;
  const Side& s = j.side[which];
  const int block = blockIdx.x - (which ? j.side[0].blocks : 0);
  const int G = 1 << lanes_log2, g = threadIdx.x & (G - 1);
  const int first = threadIdx.x >> lanes_log2, step = kThreads >> lanes_log2;
  const bool lane_on = 8 * g < j.d;
  const float over_d = 1.0f / j.d;
  float w[8], dw[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int e = R::at(j, g, i);
    w[i] = (lane_on && e < j.d ? (s.w ? s.w[e] : 1.0f) : 0.0f) * j.scale;
    dw[i] = 0.0f;
  }
  const int tiles = (j.tokens + j.tile - 1) / j.tile;
  for (int tile = block; tile < tiles; tile += s.blocks) {
    const int n0 = tile * j.tile, count = min(j.tile, j.tokens - n0);
    __syncthreads();
    if (threadIdx.x < count) {
      const int n = n0 + threadIdx.x, b = n / j.L, l = n - b * j.L;
      token[threadIdx.x] = TokenAt{b * s.xs.b + l * s.xs.l, BWD ? b * s.dys.b + l * s.dys.l : 0,
                                   b * s.os.b + l * s.os.l};
    }
    for (int i = threadIdx.x; i < count * j.half; i += kThreads) {
      const int t = i / j.half, p = i - t * j.half, n = n0 + t;
      long long pos = n % j.L;
      if (j.positions)
        pos = j.i64 ? static_cast<const long long*>(j.positions)[n]
                    : static_cast<const int*>(j.positions)[n];
      turns[i] = cos_sin((unsigned long long)pos * j.turn[p]);
    }
    __syncthreads();
    const int rows = count * s.H;
    // whole warps walk together: their lanes exchange sums
    for (int r0 = first; r0 - first < rows; r0 += step) {
      const bool on = r0 < rows;
      const int r = on ? r0 : 0;
      const int t = s.H == 1 ? r : (int)__umulhi((unsigned)r, s.by_head), h = r - t * s.H;
      const TokenAt at = token[t];
      float x[8], dz[8];
      R::load(j, static_cast<const T*>(s.x) + at.x + h * s.xs.h, g, on && lane_on, x);
      if (BWD) R::load(j, static_cast<const T*>(s.dy) + at.dy + h * s.dys.h, g, on && lane_on, dz);
      float ss = 0.0f;
#pragma unroll
      for (int i = 0; i < 8; ++i) ss = fmaf(x[i], x[i], ss);
      ss = over_lanes(ss, G);
      float fit = 1.0f;
      if (__any_sync(0xffffffffu, !(ss <= 1e38f))) {
        // squares past fp32's range: the row in smaller units, next to which eps is nothing
        if (!(ss <= 1e38f)) fit = 0x1p-80f;
        ss = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          x[i] *= fit;
          ss = fmaf(x[i], x[i], ss);
        }
        ss = over_lanes(ss, G);
      }
      const float rms = rsqrtf(fmaf(ss, over_d, j.eps * (fit * fit)));
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] *= rms;
      const float2* cs = turns + t * j.half;
      if (!BWD) {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] *= w[i];
        R::rotate(j, cs, g, 1.0f, x);
      } else {
        R::rotate(j, cs, g, -1.0f, dz);
        float gn = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          dw[i] = fmaf(dz[i], x[i], dw[i]);
          dz[i] *= w[i];
          gn = fmaf(dz[i], x[i], gn);
        }
        gn = over_lanes(gn, G) * over_d;
        const float out = fit * rms;
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = out * fmaf(-x[i], gn, dz[i]);
      }
      if (on && lane_on) R::store(j, static_cast<T*>(s.out) + at.out + h * s.os.h, g, x);
    }
  }
  if (!BWD || !s.part) return;
  // the block's sums: rows of a warp, then warps in order
  __shared__ float sum[kWarps][kMaxD];
  const int warp = threadIdx.x >> 5;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    for (int o = 16; o >= G; o >>= 1) dw[i] += __shfl_xor_sync(0xffffffffu, dw[i], o);
    const int e = R::at(j, g, i);
    if ((threadIdx.x & 31) < G && lane_on && e < j.d) sum[warp][e] = dw[i] * j.scale;
  }
  __syncthreads();
  if (threadIdx.x < j.d) {
    float v = 0.0f;
#pragma unroll
    for (int i = 0; i < kWarps; ++i) v += sum[i][threadIdx.x];
    s.part[(size_t)block * j.d + threadIdx.x] = v;
  }
}

// The weights' gradients from the blocks' sums: 32 features a block, eight threads each.
__global__ void __launch_bounds__(kThreads) k_qk_weights(WeightJob j) {
  tc::grid_dependency_wait();
  __shared__ float sh[8][32];
  const int which = blockIdx.y, col = threadIdx.x & 31, q = threadIdx.x >> 5;
  const int e = blockIdx.x * 32 + col, n = j.blocks[which];
  if (!j.out[which]) return;
  float v = 0.0f;
  const int per = (n + 7) / 8, to = min((q + 1) * per, n);
  if (e < j.d) {
#pragma unroll 8
    for (int b = q * per; b < to; ++b) v += j.part[which][(size_t)b * j.d + e];
  }
  sh[q][col] = v;
  __syncthreads();
  if (q == 0 && e < j.d) {
    for (int i = 1; i < 8; ++i) v += sh[i][col];
    j.out[which][e] = v;
  }
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

// Whether every row of the tensor can be moved in vectors of four elements.
bool in_fours(const void* p, const slim_strides& s, int es) {
  return (reinterpret_cast<uintptr_t>(p) & (4 * es - 1)) == 0 && ((s.b | s.h | s.l) & 3) == 0;
}

bool fill_side(Side* t, const Operand& x, const Operand* dy, const Operand& out, const float* w, int B,
               int H, int L, int d, int es, bool* fours) {
  t->H = H;
  if (H == 0) return true;
  t->by_head = H == 1 ? 0u : (unsigned)(((1ull << 32) + H - 1) / H);
  const Operand none{nullptr, nullptr};
  const Operand* all[3] = {&x, dy ? dy : &none, &out};
  slim_strides* to[3] = {&t->xs, &t->dys, &t->os};
  for (int i = 0; i < 3; ++i) {
    if (i == 1 && !dy) continue;
    if (!all[i]->p || (reinterpret_cast<uintptr_t>(all[i]->p) & (es - 1))) return false;
    *to[i] = strides_of(all[i]->s, H, L, d);
    if (!strides_ok(*to[i], B, H, L)) return false;
    *fours = *fours && in_fours(all[i]->p, *to[i], es);
  }
  if (!apart(t->os, B, H, L, d)) return false;
  if (w && (reinterpret_cast<uintptr_t>(w) & 3)) return false;
  t->x = x.p;
  t->dy = dy ? dy->p : nullptr;
  t->out = const_cast<void*>(out.p);
  t->w = w;
  return true;
}

template <typename T, bool BWD>
bool run(const Job& j, int mode, int lanes_log2, cudaStream_t s) {
  const unsigned blocks = (unsigned)(j.side[0].blocks + j.side[1].blocks);
  const size_t smem = (size_t)j.tile * j.half * sizeof(float2);
  const double n = (double)j.tokens * (j.side[0].H + j.side[1].H) * j.d;
  prof::Scope ps(prof::K_QK_NORM, s, n * (BWD ? 20 : 8), n * sizeof(T) * (BWD ? 3 : 2));
  auto k = mode == SPLIT ? k_qk_norm<T, SPLIT, BWD>
           : mode == INTER ? k_qk_norm<T, INTER, BWD>
                           : k_qk_norm<T, ANY, BWD>;
  k<<<blocks, kThreads, smem, s>>>(j, lanes_log2);
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
           float scale, int* mode, int* lanes_log2) {
  if (!sizes_ok(B, Hq, Hk, L, d) || (dtype != SLIM_F32 && dtype != SLIM_BF16)) return -1;
  if (rotary < 0 || rotary > d || (rotary & 1) || (interleaved & ~1)) return -1;
  if (rotary > 0 && (!inv_freq || (ptype != SLIM_I32 && ptype != SLIM_I64))) return -1;
  if (!(eps > 0.0f) || !isfinite(eps) || !isfinite(scale)) return -1;
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
  bool fours = true;
  if (!fill_side(&j->side[0], q[0], bwd ? &q[1] : nullptr, q[2], wq, B, Hq, L, d, es, &fours) ||
      !fill_side(&j->side[1], k[0], bwd ? &k[1] : nullptr, k[2], wk, B, Hk, L, d, es, &fours))
    return -1;
  if (positions && (reinterpret_cast<uintptr_t>(positions) & (ptype == SLIM_I64 ? 7 : 3))) return -1;
  j->positions = positions;
  j->i64 = ptype == SLIM_I64;
  j->tokens = B * L;
  j->L = L;
  j->d = d;
  j->half = rotary / 2;
  j->interleaved = interleaved;
  j->eps = eps;
  j->scale = scale;
  *mode = !fours || d % 8 || rotary % 8 ? ANY : interleaved ? INTER : SPLIT;
  *lanes_log2 = 0;
  while ((8 << *lanes_log2) < d) ++*lanes_log2;
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
  int mode, lanes;
  const Operand qs[3] = {{q, q_strides}, {}, {q_out, q_out_strides}};
  const Operand ks[3] = {{k, k_strides}, {}, {k_out, k_out_strides}};
  const int go = set_up(&j, qs, ks, false, q_weight, k_weight, positions, ptype, inv_freq, rotary,
                        interleaved, B, Hq, Hk, L, d, dtype, eps, scale, &mode, &lanes);
  if (go <= 0) return go < 0 ? SLIM_ERR_INVALID_ARG : SLIM_OK;
  deal(&j, 0);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const bool ok = dtype == SLIM_F32 ? run<float, false>(j, mode, lanes, s)
                                    : run<__nv_bfloat16, false>(j, mode, lanes, s);
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
  int mode, lanes;
  const Operand qs[3] = {{q, q_strides}, {dq_out, dq_out_strides}, {dq, dq_strides}};
  const Operand ks[3] = {{k, k_strides}, {dk_out, dk_out_strides}, {dk, dk_strides}};
  for (const float* p : {dq_weight, dk_weight})
    if (reinterpret_cast<uintptr_t>(p) & 3) return SLIM_ERR_INVALID_ARG;
  const int go = set_up(&j, qs, ks, true, q_weight, k_weight, positions, ptype, inv_freq, rotary,
                        interleaved, B, Hq, Hk, L, d, dtype, eps, scale, &mode, &lanes);
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
  deal(&j, kBwdBlocks);
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
  const bool ok = dtype == SLIM_F32 ? run<float, true>(j, mode, lanes, s)
                                    : run<__nv_bfloat16, true>(j, mode, lanes, s);
  if (!ok) return SLIM_ERR_CUDA;
  if (out[0] || out[1]) {
    slim::prof::Scope ps(slim::prof::K_QK_WEIGHTS, s);
    if (!slim::launch_on(k_qk_weights, dim3((d + 31) / 32, 2), kThreads, 0, 1, true, s, wj))
      return SLIM_ERR_CUDA;
  }
  return SLIM_OK;
}
