// What the kernels of the tile products share beyond their roles (lm_gemm.cuh):
// rows staged as bf16 planes, workers' runs of tiles, the launch of both gradient
// products of g = d loss / d (A B^T) and the join of their parts.
#pragma once
#include <stdint.h>

#include <type_traits>

#include "common.cuh"
#include "launch.h"
#include "lm_gemm.cuh"
#include "lm_loss_dev.cuh"
#include "profiler.h"
#include "tma_map.h"

namespace slim {
namespace lm {
namespace {

// Packs the leading bf16 plane of two values and leaves their remainders (both
// exact).  With one plane there is no remainder to keep.
template <int NP>
__device__ __forceinline__ float lead_bf16(float v) {
  const float h = __bfloat162float(__float2bfloat16_rn(v));
  // a finite value that rounds up to infinity is cut off instead
  return NP > 1 && isinf(h) && !isinf(v) ? __uint_as_float(__float_as_uint(v) & 0xffff0000u) : h;
}
template <int NP>
__device__ __forceinline__ uint32_t take_plane(float& a, float& b) {
  if (NP == 1) return tc::pack_bf16(a, b);
  const float ha = lead_bf16<NP>(a), hb = lead_bf16<NP>(b);
  // an infinity or NaN is all in its first plane
  a = isfinite(a) ? a - ha : 0.0f;
  b = isfinite(b) ? b - hb : 0.0f;
  return tc::pack_bf16(ha, hb);
}

// ------------------------------------------------------------------ staging
// Rows as bf16 planes [NP][R][ld]: fp32 values split into three, rows padded to
// a multiple of 8 elements so that TMA can step over them.  Rows that `targets`
// marks as ignored become zero.  `half`: the second source is two matrices of
// `real` rows, which come to lie `half` rows apart with zeros between.
struct StageJob {
  const void* src[2];
  __nv_bfloat16* dst[2];
  long long rows[2];    // written
  int D, ld;
  const void* targets;  // of the first source's rows, or null
  int i64;
  long long ignore;
  int* header;          // cleared: the call's first kernel
  unsigned* rep;
  int half, real;       // 0: one matrix
};
template <typename T, int NP>
__global__ void __launch_bounds__(256) k_stage(StageJob j) {
  tc::grid_dependency_wait();  // (of nothing) lets the next kernel set up meanwhile
  if (blockIdx.x == 0 && threadIdx.x < 8) j.header[threadIdx.x] = 0;
  __syncthreads();
  if (blockIdx.x == 0 && threadIdx.x == 0) tc::set_report(j.header, j.rep);
  const int per = j.ld / 8;
  const long long n0 = j.rows[0] * per, total = n0 + j.rows[1] * per;
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < total;
       i += (long long)gridDim.x * 256) {
    const int which = i >= n0;
    const long long k = which ? i - n0 : i, r = k / per;
    const int c = (int)(k - r * per) * 8;
    bool live = which || !j.targets || load_target(j.targets, j.i64, r) != j.ignore;
    long long from = r;
    if (which && j.half) {
      const long long up = r >= j.half;
      live = r - up * j.half < j.real;
      from = r - up * (j.half - j.real);
    }
    const T* src = static_cast<const T*>(j.src[which]) + (size_t)from * j.D + c;
    float v[8];
    if (live && c + 8 <= j.D && (j.D * sizeof(T)) % 16 == 0) {
      constexpr int W = 16 / sizeof(T);
#pragma unroll
      for (int q = 0; q < 8; q += W) {
        union {
          uint4 u;
          T e[W];
        } x;
        x.u = *reinterpret_cast<const uint4*>(src + q);
#pragma unroll
        for (int e = 0; e < W; ++e) v[q + e] = Io<T>::load(x.e, e);
      }
    } else {
#pragma unroll
      for (int q = 0; q < 8; ++q) v[q] = live && c + q < j.D ? Io<T>::load(src, q) : 0.0f;
    }
    __nv_bfloat16* dst = j.dst[which] + r * j.ld + c;
    const long long plane = j.rows[which] * j.ld;
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      uint32_t u[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) u[q] = take_plane<NP>(v[2 * q], v[2 * q + 1]);
      *reinterpret_cast<uint4*>(dst + p * plane) = make_uint4(u[0], u[1], u[2], u[3]);
    }
  }
}
// ------------------------------------------------------------------ runs of tiles
// A worker (a pair of blocks) takes a contiguous run of the tiles, columns
// fastest, so that it stays with the same rows as long as it can.
struct RunNext {
  TileRange r;
  __device__ __forceinline__ bool operator()(Work& w) { return r.next(w); }
};
__host__ __device__ inline long long run_begin(long long worker, long long tiles, long long workers) {
  return worker * tiles / workers;
}
// The worker that has tile t.
__host__ __device__ inline long long run_owner(long long t, long long tiles, long long workers) {
  return ((t + 1) * workers - 1) / tiles;
}
template <typename T>
__device__ __forceinline__ uint8_t* stage_memory() {
  extern __shared__ uint8_t smem_raw[];
  return reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                    ~uintptr_t(1023));
}
__device__ __forceinline__ RunNext run_of(const Product& p) {
  const long long tiles = (long long)p.tm * p.tn;
  const long long worker = blockIdx.x / kPair, workers = gridDim.x / kPair;
  return RunNext{
      TileRange(&p, run_begin(worker, tiles, workers), run_begin(worker + 1, tiles, workers))};
}
// Up to 512 features a worker can
// hold its rows of x while it walks along the vocabulary: 16384 x 512 x 50021
// statistics 424 -> 400 us, the softmax kernel of 32768 x 512 x 32768 735 -> 685 us.
// Changing rows then drains the MMAs, so it has to be for a walk of some tiles
// (65536 x 512, statistics / softmax, ring -> held: 2 tile columns 31 -> 37 / 34 ->
// 39 us, 4 46 -> 52 / 55 -> 58, 8 78 -> 82 / 98 -> 95, 16 145 -> 146 / 186 -> 174).
bool hold_rows(const Product& p) { return p.kb <= kHeld && p.tn >= 8; }
// ------------------------------------------------------------------ gradients
// A worker's tiles of the two products: a contiguous range of each, dealt on the
// host so that the workers' reductions come out even.
constexpr int kMaxWorkers = 152;
struct Deal {
  unsigned lo[2][kMaxWorkers + 1];
};
struct DealNext {
  TileRange a, b;
  __device__ __forceinline__ bool operator()(Work& w) { return a.next(w) || b.next(w); }
};

struct GradJob {
  Product p[2];            // dw of the piece's words, and dx
  Deal deal;
  void* to[2];             // their results
  int parts[2];            // whether a product's tiles go to `part`:
  float* part[2];          // [splits][M][acc_ld] partial sums
  float* acc;              // [N][acc_ld] running sum of dx over pieces
  int acc_ld;
  // 2: the results' rows are whole 32-byte sectors, 1: 16-byte pieces, 0: neither;
  // their values then go to `part` and out from there
  int wide;
  int first, last;         // of the pieces
  const float *scale, *count;  // the results' factor: (scale or 1) / (count or 1)
  const void* targets;     // null: every row counts
  int i64;
  long long ignore;
  int* err;
  unsigned* rep;
  // the first product's rows are two matrices of `real` rows, `half` rows apart
  // (0: one matrix); its result has them one behind the other
  int half, real;
};
// Row of the first product's result that row r of the product goes to, or -1.
__device__ __forceinline__ int half_row(const GradJob& j, int r) {
  if (!j.half) return r;
  const int up = r >= j.half ? 1 : 0;
  return r - up * j.half < j.real ? r - up * (j.half - j.real) : -1;
}

__device__ __forceinline__ float grad_scale(const GradJob& j) {
  float s = j.scale ? *j.scale : 1.0f;
  if (j.count) s = *j.count == 0.0f ? 0.0f : s / *j.count;
  return s;
}

template <int NP>
struct GradEpi {
  using T = typename std::conditional<NP == 1, __nv_bfloat16, float>::type;
  const GradJob& j;
  const Product* p = nullptr;
  int row = 0, col = 0, which = 0;
  bool in = false, live = true;
  float scale;
  float* part = nullptr;
  __device__ explicit GradEpi(const GradJob& job) : j(job), scale(grad_scale(job)) {}
  __device__ void begin(const Work& w, int r, int c) {
    p = w.p;
    row = r;
    col = c;
    in = r < p->M;
    which = p == &j.p[1];
    live = true;
    part = j.parts[which] ? j.part[which] + ((size_t)w.split * p->M + r) * j.acc_ld + c : nullptr;
    if (in && which == 1 && j.last && j.targets)
      live = load_target(j.targets, j.i64, r) != j.ignore;
    if (in && which == 0 && !part) {
      row = half_row(j, r);
      in = row >= 0;
    }
  }
  __device__ __forceinline__ void chunk(int c, float* f) {
    if (!in) return;
    const int D = p->N, left = D - (col + c);
    uint32_t u[8];
    if (part) {
#pragma unroll
      for (int i = 0; i < 32; i += 8) {
#pragma unroll
        for (int e = 0; e < 8; ++e) u[e] = __float_as_uint(f[i + e]);
        store32(part + c + i, u);
      }
      return;
    }
    if (which == 1) {  // the pieces' sum of dx; its rows are padded to whole chunks
      float* acc = j.acc + (size_t)row * j.acc_ld + col + c;
      if (!j.first) {
#pragma unroll
        for (int i = 0; i < 32; i += 8) {
          load32(acc + i, u);
#pragma unroll
          for (int e = 0; e < 8; ++e) f[i + e] += __uint_as_float(u[e]);
        }
      }
      if (!j.last) {
#pragma unroll
        for (int i = 0; i < 32; i += 8) {
#pragma unroll
          for (int e = 0; e < 8; ++e) u[e] = __float_as_uint(f[i + e]);
          store32(acc + i, u);
        }
        return;
      }
    }
#pragma unroll
    for (int i = 0; i < 32; ++i) f[i] = live ? f[i] * scale : 0.0f;
    T* out = static_cast<T*>(j.to[which]) + (size_t)row * D + col + c;
    constexpr int W = 32 / sizeof(T);
#pragma unroll
    for (int i = 0; i < 32; i += W) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        u[e] = NP == 1 ? tc::pack_bf16(f[i + 2 * e % W], f[i + (2 * e + 1) % W])
                       : __float_as_uint(f[i + e % W]);
      if (j.wide == 2) {
        if (i < left) store32(out + i, u);
      } else {
        if (i < left) *reinterpret_cast<uint4*>(out + i) = make_uint4(u[0], u[1], u[2], u[3]);
        if (i + W / 2 < left)
          *reinterpret_cast<uint4*>(out + i + W / 2) = make_uint4(u[4], u[5], u[6], u[7]);
      }
    }
  }
};

template <int NP>
__global__ void __launch_bounds__(kGemmThreads, 1)
    k_loss_grad(const __grid_constant__ GradJob job) {
  using T = Tile<NP>;
  __shared__ GemmShared sh;
  const int w = blockIdx.x / kPair;
  const DealNext next{TileRange(&job.p[0], job.deal.lo[0][w], job.deal.lo[0][w + 1]),
                      TileRange(&job.p[1], job.deal.lo[1][w], job.deal.lo[1][w + 1])};
  GradEpi<NP> epi(job);
  gemm_roles<T>(sh, stage_memory<T>(), next, epi, job.err);
}

// The split products' partial sums, added in order, and the way out for rows that
// the tiles cannot store in aligned pieces (a scalar store per column and row took
// 449 us of a 551 us step at 60000 x 300 x 100 bf16): four columns a thread.
template <typename T>
__global__ void __launch_bounds__(256) k_loss_parts(const __grid_constant__ GradJob j) {
  tc::grid_dependency_wait();
  const float scale = grad_scale(j);
  const int D = j.p[0].N, per = (D + 3) / 4;
  const long long n0 = j.parts[0] ? (long long)j.p[0].M * per : 0;
  const long long n1 = j.parts[1] ? (long long)j.p[1].M * per : 0;
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < n0 + n1;
       i += (long long)gridDim.x * 256) {
    const int which = i >= n0;
    const long long k = which ? i - n0 : i, row = k / per;
    const int c = (int)(k - row * per) * 4;
    const Product& p = j.p[which];
    const float* part = j.part[which] + row * j.acc_ld + c;
    const size_t step = (size_t)p.M * j.acc_ld;
    float f[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    auto add = [&](const float* q) {
      const float4 x = *reinterpret_cast<const float4*>(q);
      f[0] += x.x;
      f[1] += x.y;
      f[2] += x.z;
      f[3] += x.w;
    };
#pragma unroll 4
    for (int s = 0; s < p.splits; ++s) add(part + s * step);
    bool live = true;
    if (which) {
      float* acc = j.acc + row * j.acc_ld + c;
      if (!j.first) add(acc);
      if (!j.last) {
        *reinterpret_cast<float4*>(acc) = make_float4(f[0], f[1], f[2], f[3]);
        continue;
      }
      live = !j.targets || load_target(j.targets, j.i64, row) != j.ignore;
    }
    const long long to = which ? row : half_row(j, (int)row);
    if (to < 0) continue;
    T* out = static_cast<T*>(j.to[which]) + to * D + c;
#pragma unroll
    for (int e = 0; e < 4; ++e) f[e] = live ? f[e] * scale : 0.0f;
    if (D % 4 == 0) {
      if constexpr (sizeof(T) == 4)
        *reinterpret_cast<float4*>(out) = make_float4(f[0], f[1], f[2], f[3]);
      else
        *reinterpret_cast<uint2*>(out) =
            make_uint2(tc::pack_bf16(f[0], f[1]), tc::pack_bf16(f[2], f[3]));
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (c + e < D) Io<T>::store(out, e, f[e]);
    }
  }
}
// ------------------------------------------------------------------ host
int sm_count() {
  static const int n = [] {
    int dev = 0, v = 0;
    if (cudaGetDevice(&dev) != cudaSuccess ||
        cudaDeviceGetAttribute(&v, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || v < 2)
      v = 152;
    cudaGetLastError();
    return v;
  }();
  return n;
}

// Workspace sizes do not depend on the device: they, and the gradients' splits, are
// for kMaxWorkers blocks.
int workers() {  // pairs
  const int n = sm_count() < kMaxWorkers ? sm_count() : kMaxWorkers;
  return n / kPair;
}

int cdiv(long long a, long long b) { return (int)((a + b - 1) / b); }

// A long reduction over few tiles is split, where it would otherwise take more
// than one and a half times the even share of all workers, into parts of about
// that share.  100 rows of 1024 against 50000 words: dx is four tiles of 782
// stages beside 784 tiles of two, and unsplit took all of the launch's 221 us.
// With one plane a part is also at most 32768 terms long: the longer a sum of one
// sign, the more of each term the tensor core cuts off.  dw over 2^20 rows came out
// low by 6.6e-3 of itself unbroken, more than the result's own rounding (2^-9), and
// in parts of 65536 by 3.8e-4; the parts are joined in fp32.
constexpr long long kPartMost = 32768 / kTK;
void split_long(const long long tiles[2], const long long kb[2], int np, int w, int splits[2]) {
  const long long total = tiles[0] * kb[0] + tiles[1] * kb[1];
  const long long least = np == 1 ? 16 : 4;  // stages worth a tile of their own
  const long long even = (total + w - 1) / w, share = even > least ? even : least;
  for (int i = 0; i < 2; ++i) {
    splits[i] = 1;
    if (2 * kb[i] >= 3 * share) splits[i] = (int)((kb[i] + share - 1) / share);
    if (np == 1 && (long long)splits[i] * kPartMost < kb[i])
      splits[i] = (int)((kb[i] + kPartMost - 1) / kPartMost);
  }
}
constexpr size_t kHeaderInts = 32;
int acc_ld(int D) { return (D + 31) / 32 * 32; }

// A tensor map over planes of [rows][cols] bf16 (row stride ld elements),
// boxes of 64 columns x box_rows rows, 128-byte swizzle.
bool plane_map(CUtensorMap* m, const __nv_bfloat16* base, long long rows, long long cols,
               long long ld, long long plane, int np, int box_rows) {
  const EncodeTiledFn fn = encode_tiled();
  if (!fn) return false;
  const cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)np};
  const cuuint64_t strides[2] = {(cuuint64_t)ld * 2, (cuuint64_t)plane * 2};
  const cuuint32_t box[3] = {(cuuint32_t)kTK, (cuuint32_t)box_rows, 1};
  const cuuint32_t es[3] = {1, 1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<__nv_bfloat16*>(base), dims, strides,
            box, es, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Tiles 0 .. n[k]-1 of two products, costing cost[k] each, to w workers in
// contiguous ranges: the dearer product's tiles evenly, then the other's so that
// the workers' totals come level.
void deal_tiles(const long long n[2], const long long cost[2], int w, Deal* d) {
  const int a = cost[0] >= cost[1] ? 0 : 1, b = 1 - a;
  long long load[kMaxWorkers], give[kMaxWorkers], most = 0;
  d->lo[a][0] = 0;
  for (int i = 0; i < w; ++i) {
    const long long k = n[a] / w + (i < n[a] % w);
    d->lo[a][i + 1] = d->lo[a][i] + (unsigned)k;
    load[i] = k * cost[a];
    if (load[i] > most) most = load[i];
  }
  // the lowest level at which all of b's tiles fit
  auto fits = [&](long long level) {
    long long s = 0;
    for (int i = 0; i < w; ++i)
      if (level > load[i]) s += (level - load[i]) / cost[b];
    return s >= n[b];
  };
  long long lo = 0, hi = most + (n[b] / w + 1) * cost[b];
  while (lo < hi) {
    const long long mid = (lo + hi) / 2;
    if (fits(mid))
      hi = mid;
    else
      lo = mid + 1;
  }
  long long left = n[b];
  for (int i = w - 1; i >= 0; --i) {  // those with the least of a first
    long long k = lo > load[i] ? (lo - load[i]) / cost[b] : 0;
    if (k > left) k = left;
    give[i] = k;
    left -= k;
  }
  d->lo[b][0] = 0;
  for (int i = 0; i < w; ++i) d->lo[b][i + 1] = d->lo[b][i] + (unsigned)give[i];
}

struct Planes {
  const __nv_bfloat16* p;
  long long rows, cols, ld, plane;
};

template <int NP>
bool make_product(Product* p, const Planes& a, bool a_mn, const Planes& b, bool b_mn, long long M,
                  long long N, long long K, int tile_n = kTN) {
  if (!plane_map(&p->a, a.p, a.rows, a.cols, a.ld, a.plane, NP, a_mn ? kTK : kTM) ||
      !plane_map(&p->b, b.p, b.rows, b.cols, b.ld, b.plane, NP, b_mn ? kTK : tile_n / kPair))
    return false;
  p->a_mn = a_mn;
  p->b_mn = b_mn;
  p->M = (int)M;
  p->N = (int)N;
  p->tm = cdiv(M, kTM * kPair);
  p->tn = cdiv(N, tile_n);
  p->kb = cdiv(K, kTK);
  p->splits = 1;
  p->up = 0;
  return true;
}

template <int NP>
slim_status stage(StageJob j, cudaStream_t s, prof::Kid kid = prof::K_LOSS_PREP) {
  using T = typename std::conditional<NP == 1, __nv_bfloat16, float>::type;
  const long long n = (j.rows[0] + j.rows[1]) * (j.ld / 8);
  const unsigned blocks = (unsigned)(cdiv(n, 256) < 152 * 8 ? cdiv(n, 256) : 152 * 8);
  prof::Scope ps(kid, s, 0.0, (double)n * 8 * (sizeof(T) + 2 * NP));
  k_stage<T, NP><<<blocks, 256, 0, s>>>(j);
  return cudaGetLastError() == cudaSuccess ? SLIM_OK : SLIM_ERR_CUDA;
}

// Launches a kernel of the tile products on `blocks` blocks, in pairs.
template <typename T, typename Job>
bool launch(void (*k)(Job), unsigned blocks, bool after, cudaStream_t s, const Job& job,
            bool* ready) {
  constexpr size_t smem = T::smem();
  if (ready == nullptr || !*ready) {
    if (cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) !=
        cudaSuccess)
      return false;
    if (ready) *ready = true;
  }
  return launch_on(k, blocks, kGemmThreads, smem, kPair, after, s, job);
}

template <typename... T>
bool* once() {
  static bool flags[kMaxDevices];
  return device_flag(flags);
}

bool aligned(const void* p, size_t to) {
  return p != nullptr && (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0;
}

}  // namespace
}  // namespace lm
}  // namespace slim
