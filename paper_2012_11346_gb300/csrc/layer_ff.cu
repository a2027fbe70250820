// Gated feed-forward: both projections, the activation and the product in one
// kernel, and its gradients.  Contract: include/slim_layer.h.
//
// Forward: a tile is 256 rows by 128 features (64 where there are few tiles), its 256
// accumulator columns the features' gates and ups side by side (lm_gemm.cuh, GATED), so
// that the epilogue has both of a feature in one thread and writes h = act(g) u once.
//
// Backward: the projections again, with an epilogue that turns them and dh into
//     dz = [dh u act'(g), dh act(g)]
// as bf16 (three planes for fp32), and then one launch with dx = dz w and dw = dz^T x.
// One rounding of a bf16 problem's dz puts dx and dw 2.3e-3 of their norm off where their
// own rounding is 1.7e-3; a second plane of it would double the MMAs of both products.
// fp32 may keep both projections instead, and then dz is a pass over them.
//
// Measured: 16384 x 768 x 2048 bf16 forward 60 us, 1.72 PFLOP/s, bound by the tensor
// pipe (one call's kernels; call after call under the power limit 70 us).  32768 x 512 x
// 2048 bf16 step: forward 77 us, dz 111, both products 170; with only 8 stages of the
// reduction to a tile, the epilogue (dz: 192 KB of dh and dz a tile and the operands
// again, 8 TB/s through L2) takes longer than the tile's MMAs, 57 us.
#include <stdint.h>

#include "../../include/slim_layer.h"
#include "common.cuh"
#include "launch.h"
#include "layer_ff.h"
#include "lm_gemm.cuh"
#include "lm_products.cuh"
#include "profiler.h"
#include "report.h"

namespace slim {
namespace lm {
namespace {

struct FfJob {
  Product p;
  int F, act;
  int wide;          // h's (dh's) rows in 2: 32-byte sectors, 1: 16-byte pieces, 0: elements
  void* h;           // forward
  float* z;          // both projections [N][2 half], or null
  const void* dh;    // backward
  __nv_bfloat16* dz; // [NP][N][2 half]
  long long plane;
  int half;          // columns of dz's parts: F rounded up to 16
  int* err;
  unsigned* rep;
  int first;         // the call's first kernel: clears its header (else rows are staged before)
};

// 16 values of a row of h or dh (F long), from column c on.
template <typename T>
__device__ __forceinline__ void store16(T* row, int c, int F, int wide, const float* v) {
  constexpr int W = 32 / sizeof(T);
  T* to = row + c;
  if (!wide) {
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (c + i < F) Io<T>::store(to, i, v[i]);
    return;
  }
#pragma unroll
  for (int i = 0; i < 16; i += W) {
    uint32_t u[8];
#pragma unroll
    for (int e = 0; e < 8; ++e)
      u[e] = sizeof(T) == 2 ? tc::pack_bf16(v[i + 2 * e % W], v[i + (2 * e + 1) % W])
                            : __float_as_uint(v[i + e % W]);
    if (wide == 2) {
      if (c + i < F) store32(to + i, u);
    } else {
      if (c + i < F) *reinterpret_cast<uint4*>(to + i) = make_uint4(u[0], u[1], u[2], u[3]);
      if (c + i + W / 2 < F)
        *reinterpret_cast<uint4*>(to + i + W / 2) = make_uint4(u[4], u[5], u[6], u[7]);
    }
  }
}
template <typename T>
__device__ __forceinline__ void load16(const T* row, int c, int F, int wide, float* v) {
  constexpr int W = 16 / sizeof(T);
#pragma unroll
  for (int i = 0; i < 16; i += W) {
    if (!wide) {
#pragma unroll
      for (int e = 0; e < W; ++e) v[i + e] = c + i + e < F ? Io<T>::load(row, c + i + e) : 0.0f;
      continue;
    }
    const uint4 u = c + i < F ? *reinterpret_cast<const uint4*>(row + c + i) : make_uint4(0, 0, 0, 0);
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if constexpr (sizeof(T) == 2)
        tc::unpack_bf16(w[e], v[i + 2 * e], v[i + 2 * e + 1]);
      else
        v[i + e] = __uint_as_float(w[e]);
    }
  }
}

template <int NP>
struct FfFwdEpi {
  using T = typename std::conditional<NP == 1, __nv_bfloat16, float>::type;
  const FfJob& j;
  int row = 0, col = 0;
  bool in = false;
  __device__ explicit FfFwdEpi(const FfJob& job) : j(job) {}
  __device__ void begin(const Work& w, int r, int c) {
    row = r;
    col = c;
    in = r < w.p->M;
  }
  __device__ __forceinline__ void pair(int c, float* g, float* u) {
    if (!in) return;
    if (NP > 1 && j.z) {
      // (columns past F are of no use, and are not used)
      float* row_z = j.z + (size_t)row * (2 * j.half);
      store16(row_z, col + c, j.half, 2, g);
      store16(row_z + j.half, col + c, j.half, 2, u);
    }
    layer::with_act(j.act, [&](auto act) {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        float a, none;
        layer::activate<decltype(act)::value, NP == 1, false>(g[i], a, none);
        u[i] *= a;
      }
    });
    store16(static_cast<T*>(j.h) + (size_t)row * j.F, col + c, j.F, j.wide, u);
  }
};

template <int NP>
struct FfBwdEpi {
  using T = typename std::conditional<NP == 1, __nv_bfloat16, float>::type;
  const FfJob& j;
  int row = 0, col = 0;
  bool in = false;
  // bf16: dh is on its way before the tile's products are done (16 registers)
  static constexpr bool AHEAD = NP == 1;
  uint4 ahead[AHEAD ? 4 : 1];
  __device__ explicit FfBwdEpi(const FfJob& job) : j(job) {}
  __device__ void begin(const Work& w, int r, int c) {
    row = r;
    col = c;
    in = r < w.p->M;
    if (AHEAD && in && j.wide) {
      const T* from = static_cast<const T*>(j.dh) + (size_t)r * j.F + c;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        ahead[i] = c + 8 * i < j.F ? *reinterpret_cast<const uint4*>(from + 8 * i) : make_uint4(0, 0, 0, 0);
      // the next tile's, most often of the same rows
      if (c + kTN / kPair < j.F) asm volatile("prefetch.global.L2 [%0];" ::"l"(from + kTN / kPair));
    }
  }
  __device__ __forceinline__ void pair(int c, float* g, float* u) {
    if (!in) return;
    float dh[16];
    if (AHEAD && j.wide) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint4 a = c ? ahead[AHEAD ? 2 + i : 0] : ahead[AHEAD ? i : 0];
        const uint32_t v[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) tc::unpack_bf16(v[e], dh[8 * i + 2 * e], dh[8 * i + 2 * e + 1]);
      }
    } else {
      load16(static_cast<const T*>(j.dh) + (size_t)row * j.F, col + c, j.F, j.wide, dh);
    }
    layer::with_act(j.act, [&](auto act) {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        float a, da;
        layer::activate<decltype(act)::value, NP == 1, true>(g[i], a, da);
        g[i] = dh[i] * u[i] * da;
        u[i] = dh[i] * a;
      }
    });
    if (col + c + 16 > j.F) {  // columns that only round the parts up
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (col + c + i >= j.F) g[i] = u[i] = 0.0f;
    }
    __nv_bfloat16* to = j.dz + (size_t)row * (2 * j.half) + col + c;
#pragma unroll
    for (int q = 0; q < NP; ++q) {
      uint32_t v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = take_plane<NP>(g[2 * e], g[2 * e + 1]);
      store32(to + q * j.plane, v);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = take_plane<NP>(u[2 * e], u[2 * e + 1]);
      store32(to + q * j.plane + j.half, v);
    }
  }
};

template <int NP, bool HOLD, bool BWD, int COLS>
__global__ void __launch_bounds__(kGemmThreads, 1) k_ff(const __grid_constant__ FfJob job) {
  using T = Tile<NP, (NP > 1), HOLD, true, COLS>;
  __shared__ GemmShared sh;
  if (job.first) {
    if (blockIdx.x == 0 && threadIdx.x < 8) job.err[threadIdx.x] = 0;
    __syncthreads();
    if (blockIdx.x == 0 && threadIdx.x == 0) tc::set_report(job.err, job.rep);
  }
  typename std::conditional<BWD, FfBwdEpi<NP>, FfFwdEpi<NP>>::type epi(job);
  gemm_roles<T>(sh, stage_memory<T>(), run_of(job.p), epi, job.err);
}

// dz from projections that the forward kept: eight features a thread.  z and dh are
// read, dz's three planes written: 24 bytes a feature and row, where computing the
// projections again takes 24 D operations on the tensor cores.
__global__ void __launch_bounds__(256) k_ff_kept(const __grid_constant__ FfJob j, long long N) {
  tc::grid_dependency_wait();
  const int per = j.half / 8;
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < N * per; i += (long long)gridDim.x * 256) {
    const long long row = i / per;
    const int c = (int)(i - row * per) * 8;
    float v[3][8];  // g, u, dh
    const float* z = j.z + row * (2 * j.half) + c;
    const float* dh = static_cast<const float*>(j.dh) + row * j.F + c;
#pragma unroll
    for (int e = 0; e < 8; e += 4) {
      const float4 g = *reinterpret_cast<const float4*>(z + e), u = *reinterpret_cast<const float4*>(z + j.half + e);
      float4 d = make_float4(0, 0, 0, 0);
      if (j.wide) {
        if (c + e < j.F) d = *reinterpret_cast<const float4*>(dh + e);
      } else {
        if (c + e < j.F) d.x = dh[e];
        if (c + e + 1 < j.F) d.y = dh[e + 1];
        if (c + e + 2 < j.F) d.z = dh[e + 2];
        if (c + e + 3 < j.F) d.w = dh[e + 3];
      }
      const float4 all[3] = {g, u, d};
#pragma unroll
      for (int k = 0; k < 3; ++k) {
        v[k][e] = all[k].x;
        v[k][e + 1] = all[k].y;
        v[k][e + 2] = all[k].z;
        v[k][e + 3] = all[k].w;
      }
    }
    layer::with_act(j.act, [&](auto act) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float a, da;
        layer::activate<decltype(act)::value, false, true>(v[0][e], a, da);
        v[0][e] = c + e < j.F ? v[2][e] * v[1][e] * da : 0.0f;
        v[1][e] = c + e < j.F ? v[2][e] * a : 0.0f;
      }
    });
    __nv_bfloat16* to = j.dz + row * (2 * j.half) + c;
#pragma unroll
    for (int q = 0; q < 3; ++q)
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        uint32_t u[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) u[e] = take_plane<3>(v[k][2 * e], v[k][2 * e + 1]);
        *reinterpret_cast<uint4*>(to + q * j.plane + k * j.half) = make_uint4(u[0], u[1], u[2], u[3]);
      }
  }
}

// ------------------------------------------------------------------ host
// Keeping both projections is the quicker for fp32 rows: 8192 x 1024 x 2048, a step of 805
// us (1002 with them computed again), 32768 x 64 x 1024 462 (506).  bf16 would have to
// round them to gain.
bool keeps(long long N, int D, int F, slim_dtype dtype) {
  return dtype == SLIM_F32 && N > 0 && !layer::ff_rows_fit(N, D, F, dtype);
}

struct FfSizes {
  long long N;
  int D, F;
  slim_dtype dtype;
  int np() const { return dtype == SLIM_F32 ? 3 : 1; }
  int es() const { return dtype == SLIM_F32 ? 4 : 2; }
  int ld() const { return (D + 7) / 8 * 8; }  // of a staged row
  bool even_rows() const { return D % (dtype == SLIM_F32 ? 4 : 8) == 0; }
  // bf16 rows that TMA can step over are read where they are
  bool stage_x() const { return dtype == SLIM_F32 || !even_rows(); }
  int half() const { return (F + 15) / 16 * 16; }
  // backward, w's two parts lie as dz's do
  bool stage_w(bool bwd) const { return stage_x() || (bwd && half() != F); }
  int w_half(bool bwd) const { return bwd ? half() : F; }
};

bool ff_sizes_ok(long long N, int D, int F, slim_dtype dtype, slim_act act) {
  if (N < 0 || N >= (1LL << 31) - 512 || D < 1 || D > (1 << 30) || F < 1 || F > (1 << 29)) return false;
  if (dtype != SLIM_F32 && dtype != SLIM_BF16) return false;
  if (act < SLIM_ACT_SILU || act > SLIM_ACT_SIGMOID) return false;
  if (N > 0 && F > (1LL << 45) / N) return false;  // a worker's tiles fit 31 bits
  return (long long)D <= (1LL << 40) / (N > 0 ? N : 1) && (long long)D <= (1LL << 40) / (2LL * F);
}

void ff_splits(const FfSizes& z, int splits[2]) {
  const long long tn = cdiv(z.D, kTN), wide = 2LL * z.half();
  const long long tiles[2] = {cdiv(wide, kTM * kPair) * tn, cdiv(z.N, kTM * kPair) * tn};
  const long long kb[2] = {cdiv(z.N, kTK), cdiv(wide, kTK)};
  split_long(tiles, kb, z.np(), kMaxWorkers / kPair, splits);
}

struct FfWs {
  int* header;  // error word, report address
  __nv_bfloat16 *x, *w, *dz;
  float* split_sum[2];
};
FfWs ff_carve(Carver& cv, const FfSizes& z, bool bwd) {
  FfWs w{};
  const size_t np = z.np();
  w.header = cv.take<int>(kHeaderInts);
  if (z.stage_w(bwd)) {
    // together: one launch
    if (z.stage_x()) w.x = cv.take<__nv_bfloat16>(np * z.N * z.ld());
    w.w = cv.take<__nv_bfloat16>(np * 2 * z.w_half(bwd) * z.ld());
  }
  if (bwd) {
    w.dz = cv.take<__nv_bfloat16>(np * z.N * 2 * z.half());
    int splits[2];
    ff_splits(z, splits);
    for (int i = 0; i < 2; ++i) {
      const bool parts = splits[i] > 1 || !z.even_rows();
      const size_t rows = i ? z.N : 2LL * z.half();
      w.split_sum[i] = cv.take<float>(parts ? splits[i] * rows * acc_ld(z.D) : 0);
    }
  }
  return w;
}

// The rows of h and dh: see FfJob::wide.
int row_steps(const FfSizes& z, const void* p) {
  const int bytes = z.F % (64 / z.es()) * z.es();  // of a row, mod 64
  if (bytes % 16 || (reinterpret_cast<uintptr_t>(p) & 15)) return 0;
  return bytes % 32 || (reinterpret_cast<uintptr_t>(p) & 31) ? 1 : 2;
}

template <int NP, bool HOLD, bool BWD, int COLS>
bool ff_launch(long long wk, bool staged, cudaStream_t s, const FfJob& j) {
  using T = Tile<NP, (NP > 1), HOLD, true, COLS>;
  return launch<T>(k_ff<NP, HOLD, BWD, COLS>, (unsigned)wk * kPair, staged, s, j,
                   once<T, std::integral_constant<bool, BWD>>());
}

template <int NP, bool BWD>
slim_status ff_tiles(const FfSizes& z, FfJob& j, const Planes& x, const Planes& w, const FfWs& ws,
                     bool staged, unsigned* rep, cudaStream_t s) {
  const int columns = BWD ? z.half() : z.F;
  // Few tiles: of half the columns, for twice the SMs (1021 x 200 x 533 fp32, 20 tiles of
  // 128 features for 76 pairs of blocks: forward 27 us, with 36 of 64 features 18; dz 38
  // and 20).
  const bool narrow = 2LL * cdiv(z.N, kTM * kPair) * cdiv(columns, kTN / kPair) <= workers();
  const int tile_n = narrow ? kTN / 2 : kTN;
  // B's box covers both matrices; the second begins w_half rows on
  if (!make_product<NP>(&j.p, x, false, w, false, z.N, columns, z.D, tile_n)) return SLIM_ERR_CUDA;
  j.p.tn = cdiv(columns, tile_n / kPair);
  j.p.up = z.w_half(BWD);
  j.F = z.F;
  j.half = z.half();
  j.err = ws.header;
  j.rep = rep;
  j.first = !staged;
  const long long tiles = (long long)j.p.tm * j.p.tn;
  const long long wk = tiles < workers() ? tiles : workers();
  const double n = z.N, f = z.F;
  prof::Scope ps(BWD ? prof::K_FF_DZ : prof::K_FF, s, 4.0 * n * z.D * f,
                 (n + 2 * f) * z.D * 2 * NP + n * f * (z.es() + (BWD ? 4.0 * NP : 0.0)));
  bool ok;
  if (narrow)
    ok = ff_launch<NP, false, BWD, kTN / 2>(wk, staged, s, j);
  else if (NP == 1 && hold_rows(j.p))
    ok = ff_launch<1, true, BWD, kTN>(wk, staged, s, j);
  else
    ok = ff_launch<NP, false, BWD, kTN>(wk, staged, s, j);
  return ok ? SLIM_OK : SLIM_ERR_CUDA;
}

template <int NP>
slim_status ff_stage(const FfSizes& z, const void* x, const void* w, const FfWs& ws, bool bwd,
                     unsigned* rep, cudaStream_t s) {
  const int half = z.w_half(bwd);
  StageJob j{{x, w}, {ws.x, ws.w}, {ws.x ? z.N : 0, 2LL * half}, z.D, z.ld(), nullptr, 0, 0, ws.header, rep};
  j.half = half == z.F ? 0 : half;
  j.real = z.F;
  return stage<NP>(j, s, prof::K_FF_PREP);
}

template <int NP>
slim_status ff_fwd(const FfSizes& z, const void* x, const void* w, slim_act act, void* h, float* kept,
                   const FfWs& ws, unsigned* rep, cudaStream_t s) {
  if (ws.w) {
    const slim_status st = ff_stage<NP>(z, x, w, ws, false, rep, s);
    if (st != SLIM_OK) return st;
  }
  const int ld = z.ld();
  const Planes xm{ws.x ? ws.x : static_cast<const __nv_bfloat16*>(x), z.N, z.D, ld, z.N * ld};
  const Planes wm{ws.w ? ws.w : static_cast<const __nv_bfloat16*>(w), 2LL * z.F, z.D, ld, 2LL * z.F * ld};
  FfJob j{};
  j.act = act;
  j.h = h;
  j.wide = row_steps(z, h);
  j.z = kept;
  return ff_tiles<NP, false>(z, j, xm, wm, ws, ws.w != nullptr, rep, s);
}

template <int NP>
slim_status ff_bwd(const FfSizes& z, const void* x, const void* w, const void* dh, slim_act act,
                   const float* kept, void* dx, void* dw, const FfWs& ws, unsigned* rep, cudaStream_t s) {
  using T = typename std::conditional<NP == 1, __nv_bfloat16, float>::type;
  if (ws.w) {
    const slim_status st = ff_stage<NP>(z, x, w, ws, true, rep, s);
    if (st != SLIM_OK) return st;
  }
  const int ld = z.ld(), wide = 2 * z.half();
  const Planes xm{ws.x ? ws.x : static_cast<const __nv_bfloat16*>(x), z.N, z.D, ld, z.N * ld};
  const Planes wm{ws.w ? ws.w : static_cast<const __nv_bfloat16*>(w), wide, z.D, ld, (long long)wide * ld};
  const Planes zm{ws.dz, z.N, wide, wide, z.N * wide};
  FfJob j{};
  j.act = act;
  j.dh = dh;
  j.wide = row_steps(z, dh);
  j.dz = ws.dz;
  j.plane = z.N * wide;
  if (kept) {
    j.z = const_cast<float*>(kept);
    j.F = z.F;
    j.half = z.half();
    const long long n = z.N * (z.half() / 8);
    prof::Scope sd(prof::K_FF_DZ, s, 20.0 * z.N * z.F, 24.0 * z.N * z.F);
    if (!launch_on(k_ff_kept, (unsigned)(cdiv(n, 256) < 152 * 8 ? cdiv(n, 256) : 152 * 8), 256, 0, 1, true, s, j, z.N))
      return SLIM_ERR_CUDA;
  } else {
    const slim_status st = ff_tiles<NP, true>(z, j, xm, wm, ws, ws.w != nullptr, rep, s);
    if (st != SLIM_OK) return st;
  }
  GradJob q{};
  if (!make_product<NP>(&q.p[0], zm, true, xm, true, wide, z.D, z.N) ||
      !make_product<NP>(&q.p[1], zm, false, wm, true, z.N, z.D, wide))
    return SLIM_ERR_CUDA;
  q.to[0] = dw;
  q.to[1] = dx;
  q.wide = !z.even_rows() ? 0
           : z.D * sizeof(T) % 32 == 0 && (((uintptr_t)dw | (uintptr_t)dx) & 31) == 0 ? 2 : 1;
  q.err = ws.header;
  q.rep = rep;
  q.acc_ld = acc_ld(z.D);
  q.first = q.last = 1;
  if (z.half() != z.F) {
    q.half = z.half();
    q.real = z.F;
  }
  int splits[2];
  ff_splits(z, splits);
  long long nt[2], cost[2];
  for (int k = 0; k < 2; ++k) {
    q.parts[k] = splits[k] > 1 || !q.wide;
    q.p[k].splits = splits[k];
    q.part[k] = ws.split_sum[k];
    nt[k] = (long long)q.p[k].tm * q.p[k].tn * splits[k];
    cost[k] = cdiv(q.p[k].kb, splits[k]);
  }
  const int wk = (int)(nt[0] + nt[1] < workers() ? nt[0] + nt[1] : workers());
  deal_tiles(nt, cost, wk, &q.deal);
  {
    const double n = z.N;
    prof::Scope sc(prof::K_FF_GRAD, s, 8.0 * n * z.D * z.F, (n + wide) * z.D * 2 * NP + 4.0 * NP * n * wide);
    if (!launch<Tile<NP>>(k_loss_grad<NP>, (unsigned)wk * kPair, true, s, q, once<GradEpi<NP>>()))
      return SLIM_ERR_CUDA;
  }
  if (q.parts[0] || q.parts[1]) {
    const long long e = ((q.parts[0] ? wide : 0) + (q.parts[1] ? z.N : 0)) * cdiv(z.D, 4);
    prof::Scope sp(prof::K_FF_PARTS, s);
    if (!launch_on(k_loss_parts<T>, (unsigned)(cdiv(e, 256) < 152 * 8 ? cdiv(e, 256) : 152 * 8), 256, 0, 1,
                   true, s, q))
      return SLIM_ERR_CUDA;
  }
  return SLIM_OK;
}

}  // namespace
}  // namespace lm
}  // namespace slim

extern "C" slim_status slim_gated_ff_workspace_size(long long N, int D, int F, slim_dtype dtype,
                                                    int backward, size_t* bytes) {
  using namespace slim::lm;
  if (!bytes || !ff_sizes_ok(N, D, F, dtype, SLIM_ACT_SILU) || (backward & ~1)) return SLIM_ERR_INVALID_ARG;
  *bytes = 0;
  if (!backward && slim::layer::ff_rows_fit(N, D, F, dtype)) return SLIM_OK;
  slim::Carver cv(nullptr);
  ff_carve(cv, FfSizes{N, D, F, dtype}, backward != 0);
  *bytes = cv.bytes();
  return SLIM_OK;
}

extern "C" slim_status slim_gated_ff_kept_size(long long N, int D, int F, slim_dtype dtype, size_t* bytes) {
  using namespace slim::lm;
  if (!bytes || !ff_sizes_ok(N, D, F, dtype, SLIM_ACT_SILU)) return SLIM_ERR_INVALID_ARG;
  *bytes = keeps(N, D, F, dtype) ? (size_t)N * 2 * FfSizes{N, D, F, dtype}.half() * sizeof(float) : 0;
  return SLIM_OK;
}

namespace {
// The call's workspace: checked, and its earlier waits' failures reported.
slim_status ff_begin(long long N, int D, int F, slim_dtype dtype, int backward, void* workspace,
                     size_t bytes, bool waits, unsigned** rep) {
  size_t need = 0;
  slim_gated_ff_workspace_size(N, D, F, dtype, backward, &need);
  if (need == 0 && workspace == nullptr) return SLIM_OK;
  if (workspace == nullptr || bytes < need) return SLIM_ERR_WORKSPACE;
  if (!slim::lm::aligned(workspace, 256)) return SLIM_ERR_INVALID_ARG;
  return waits ? slim::report::begin(workspace, true, rep) : slim::report::pending(workspace);
}
}  // namespace

extern "C" slim_status slim_gated_ff_fwd(const void* x, const void* w, long long N, int D, int F,
                                         slim_dtype dtype, slim_act act, void* h, float* kept,
                                         void* workspace, size_t workspace_bytes, void* stream) {
  using namespace slim::lm;
  if (!ff_sizes_ok(N, D, F, dtype, act) || !aligned(w, 16)) return SLIM_ERR_INVALID_ARG;
  if (kept && (!keeps(N, D, F, dtype) || !aligned(kept, 32))) return SLIM_ERR_INVALID_ARG;
  if (N == 0) return SLIM_OK;
  if (!aligned(x, 16) || !aligned(h, 16)) return SLIM_ERR_INVALID_ARG;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const bool rows = slim::layer::ff_rows_fit(N, D, F, dtype);
  unsigned* rep = nullptr;
  const slim_status st = ff_begin(N, D, F, dtype, 0, workspace, workspace_bytes, !rows, &rep);
  if (st != SLIM_OK) return st;
  if (rows) {
    // nothing waits; a workspace given all the same starts anew
    if (workspace && workspace_bytes >= 16 && cudaMemsetAsync(workspace, 0, 16, s) != cudaSuccess)
      return SLIM_ERR_CUDA;
    return slim::layer::ff_rows_fwd(x, w, (int)N, D, F, dtype, act, h, s);
  }
  const FfSizes z{N, D, F, dtype};
  slim::Carver cv(workspace);
  const FfWs ws = ff_carve(cv, z, false);
  return dtype == SLIM_BF16 ? ff_fwd<1>(z, x, w, act, h, kept, ws, rep, s)
                            : ff_fwd<3>(z, x, w, act, h, kept, ws, rep, s);
}

extern "C" slim_status slim_gated_ff_bwd(const void* x, const void* w, const void* dh, long long N,
                                         int D, int F, slim_dtype dtype, slim_act act,
                                         const float* kept, void* dx, void* dw, void* workspace, size_t workspace_bytes,
                                         void* stream) {
  using namespace slim::lm;
  if (!ff_sizes_ok(N, D, F, dtype, act) || !aligned(w, 16) || !aligned(dw, 16)) return SLIM_ERR_INVALID_ARG;
  if (kept && (!keeps(N, D, F, dtype) || !aligned(kept, 32))) return SLIM_ERR_INVALID_ARG;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (N == 0) {
    const size_t n = 2 * (size_t)F * D * (dtype == SLIM_F32 ? 4 : 2);
    return cudaMemsetAsync(dw, 0, n, s) == cudaSuccess ? SLIM_OK : SLIM_ERR_CUDA;
  }
  if (!aligned(x, 16) || !aligned(dh, 16) || !aligned(dx, 16)) return SLIM_ERR_INVALID_ARG;
  unsigned* rep = nullptr;
  const slim_status st = ff_begin(N, D, F, dtype, 1, workspace, workspace_bytes, true, &rep);
  if (st != SLIM_OK) return st;
  const FfSizes z{N, D, F, dtype};
  slim::Carver cv(workspace);
  const FfWs ws = ff_carve(cv, z, true);
  return dtype == SLIM_BF16 ? ff_bwd<1>(z, x, w, dh, act, nullptr, dx, dw, ws, rep, s)
                            : ff_bwd<3>(z, x, w, dh, act, kept, dx, dw, ws, rep, s);
}
