// Softmax cross entropy over a vocabulary in pieces, without keeping the
// logits, and its gradients.  Contract: include/slim_lm.h.
//
// Forward: z = x w^T by tiles on the tensor cores; a tile's epilogue folds its
// columns into a running (maximum, sum of exponentials) per row, which stays in
// registers while a worker walks along the vocabulary for the same rows.  The
// row's own target is left out of the sum and its logit kept apart: the loss is
// log1p(rest / target), which keeps its digits when it is small.  A second
// kernel joins the workers' partial statistics of each row in a fixed order.
//
// Backward, for each piece of the vocabulary: the logits again, with an epilogue
// that turns them into g = c (p - onehot), kept for this piece only, and then one
// launch with both products, dx += g w and dw = g^T x.
//
// What bounds them, on GB300 (kernel times; peak = 1978 TFLOP/s bf16):
//   statistics  16384 x 512 x 50021 bf16  404 us, 2.1 PFLOP/s: the tensor pipe;
//               8192 x 768 x 10000 fp32   360 us, 2.1 PFLOP/s of plane products.
//   softmax     32768 x 512 x 32768 bf16  705 us: g's stores share L1 with the
//               MMAs' operands (the statistics of the same tiles: 540 us).
//   products    the same sizes            1345 us, 1.6 PFLOP/s at 1.7 GHz: power.
// The logits are computed twice because a row's statistics are not known until
// its last word; keeping them would be N x V, the thing to avoid.
#include <stdint.h>

#include "../../include/slim_lm.h"
#include "common.cuh"
#include "launch.h"
#include "lm_gemm.cuh"
#include "lm_loss_dev.cuh"
#include "lm_loss_rows.h"
#include "profiler.h"
#include "report.h"
#include "tma_map.h"

namespace slim {
namespace lm {
namespace {

constexpr int kPieceStep = 256;  // pieces are multiples of this

// 2^x.  The fast form is within a few units of 2^-22; fp32 problems take the
// accurate one.
template <int NP>
__device__ __forceinline__ float exp2_of(float x) {
  return NP == 1 ? tc::ex2_approx(x) : exp2f(x);
}

// The fast form that keeps weights below 2^-126: multiplied by a large x they are
// all that some words' gradients have.
__device__ __forceinline__ float exp2_small(float x) {
  float y;
  asm("ex2.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

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
// marks as ignored become zero.
struct StageJob {
  const void* src[2];
  __nv_bfloat16* dst[2];
  long long rows[2];
  int D, ld;
  const void* targets;  // of the first source's rows, or null
  int i64;
  long long ignore;
  int* header;          // cleared: the call's first kernel
  unsigned* rep;
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
    const bool live = which || !j.targets || load_target(j.targets, j.i64, r) != j.ignore;
    const T* src = static_cast<const T*>(j.src[which]) + (size_t)r * j.D + c;
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

// ------------------------------------------------------------------ logits
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

struct StatJob {
  Product p;
  const void* targets;
  int i64;
  long long ignore;
  int V;
  int slots;       // partial statistics per row: 4 per worker that shares it
  float2* part;    // [tm][slots][rows of a tile]: base, sum of 2^(z log2 e - base)
  float* zt;       // [N] target logits
  int* err;
  unsigned* rep;
  int first;       // the call's first kernel: clears its header
};

// A row's logits but the target's, over a worker's run, as (base, sum): sum =
// sum_v 2^(z_v log2 e - base), base the largest exponent so far.  The base is
// kept as it was used, in units of log2, so that it means the same to every
// term and to the join.
template <int NP>
struct StatEpi {
  const StatJob& j;
  long long worker, workers;
  int m_now = -1;
  float base = -INFINITY, sum = 0.0f;
  int row = 0, col = 0, target = -1, slot_row = 0;
  __device__ StatEpi(const StatJob& job, long long w, long long ws)
      : j(job), worker(w), workers(ws) {}
  __device__ void begin(const Work& w, int r, int c) {
    if (w.m != m_now) {
      flush();
      m_now = w.m;
      base = -INFINITY;
      sum = 0.0f;
      row = r;
      slot_row = r - w.m * kTM * kPair;
      target = -1;
      if (r < w.p->M) {
        const long long t = load_target(j.targets, j.i64, r);
        if (t != j.ignore && t >= 0 && t < j.V) target = (int)t;
      }
    }
    col = c;
  }
  __device__ __forceinline__ void chunk(int c, float* v) {
    float* z = v;
    const int left = j.V - (col + c), at = target - (col + c);
    if (at >= 0 && at < 32) {
#pragma unroll
      for (int i = 0; i < 32; ++i)
        if (i == at) {
          j.zt[row] = z[i];
          z[i] = -INFINITY;
        }
    }
    if (left < 32) {
#pragma unroll
      for (int i = 0; i < 32; ++i)
        if (i >= left) z[i] = -INFINITY;
    }
    float q[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
    for (int i = 0; i < 32; ++i) q[i & 3] = fmaxf(q[i & 3], z[i]);
    const float to = fmaxf(base, fmaxf(fmaxf(q[0], q[1]), fmaxf(q[2], q[3])) * kLog2e);
    // with nothing but -inf so far the sum stays 0: 2^(-inf - 0)
    const float ref = to == -INFINITY ? 0.0f : to;
    // 32 terms are added among themselves first: a run is tens of thousands long
    float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < 32; ++i) s[i & 3] += exp2_of<NP>(fmaf(z[i], kLog2e, -ref));
    sum = fmaf(sum, exp2_of<NP>(base - ref), (s[0] + s[1]) + (s[2] + s[3]));
    base = to;
  }
  __device__ void flush() {
    if (m_now < 0) return;
    const long long tiles = (long long)j.p.tm * j.p.tn;
    const int slot = (int)(worker - run_owner((long long)m_now * j.p.tn, tiles, workers)) * 4 +
                     (threadIdx.x / 32 - 4) / 4;
    j.part[((size_t)m_now * j.slots + slot) * (kTM * kPair) + slot_row] = make_float2(base, sum);
  }
};

struct SoftJob {
  Product p;
  const void* targets;
  int i64;
  long long ignore;
  int V, v0;                  // vocabulary, and the piece's first word
  const float *lse, *dloss;   // dloss: per row, or null (1; the products are scaled)
  __nv_bfloat16* g;           // [NP][M][ld], ld a multiple of 256
  long long plane;
  int ld;
  int* err;
  unsigned* rep;
};

// g = c (exp(z - lse) - onehot), rounded to NP bf16 pieces.  A factor that all
// rows share is left to the products' epilogues: rounded into g it would put the
// same error on every row, and without it a target with little weight is -1
// exactly.
template <int NP>
struct SoftEpi {
  const SoftJob& j;
  int row = 0, col = 0, target = -1;
  float coef = 0.0f, lse = 0.0f;
  bool in = false, live = false;
  __device__ explicit SoftEpi(const SoftJob& job) : j(job) {}
  int m_now = -1;
  __device__ void begin(const Work& w, int r, int c) {
    col = c;
    if (w.m == m_now) return;  // the same rows as the last tile's
    m_now = w.m;
    row = r;
    in = r < w.p->M;
    live = false;
    target = -1;
    coef = 0.0f;
    lse = INFINITY;  // exp(z - inf) = 0: nothing from rows that are ignored
    if (!in) return;
    const long long t = load_target(j.targets, j.i64, r);
    if (t == j.ignore) return;
    live = true;
    lse = j.lse[r];
    coef = j.dloss ? j.dloss[r] : 1.0f;
    if (t >= 0 && t < j.V)
      target = (int)t - j.v0;
    else
      coef = __int_as_float(0x7fffffff);
  }
  __device__ __forceinline__ void chunk(int c, float* v) {
    const int at = target - (col + c);
    float* g = v;
    if (NP == 1) {
      const float l2 = lse * kLog2e;
#pragma unroll
      for (int i = 0; i < 32; ++i) g[i] = exp2_small(fmaf(v[i], kLog2e, -l2));
    } else {
#pragma unroll
      for (int i = 0; i < 32; ++i) g[i] = expf(v[i] - lse);
    }
    if (live && at >= 0 && at < 32) {
#pragma unroll
      for (int i = 0; i < 32; ++i)
        if (i == at) g[i] -= 1.0f;
    }
#pragma unroll
    for (int i = 0; i < 32; ++i) g[i] = live ? g[i] * coef : 0.0f;
    if (!in) return;
    // columns past the piece's end stay inside the row's ld, and nothing reads them
    __nv_bfloat16* to = j.g + (size_t)row * j.ld + col + c;
#pragma unroll
    for (int q = 0; q < NP; ++q) {
#pragma unroll
      for (int i = 0; i < 32; i += 16) {
        uint32_t u[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) u[e] = take_plane<NP>(g[i + 2 * e], g[i + 2 * e + 1]);
        store32(to + q * j.plane + i, u);
      }
    }
  }
};

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

// A bf16 logit over more than 512 features is summed in chains: its loss shows
// in the fp32 results otherwise (2e-6 of a logit at 2048).  The gradients' logits
// are summed as the statistics' are, to the same bits: where a row is sure of its
// target, p - 1 is what their difference leaves.  Up to 512 features a worker can
// hold its rows of x while it walks along the vocabulary: 16384 x 512 x 50021
// statistics 424 -> 400 us, the softmax kernel of 32768 x 512 x 32768 735 -> 685 us.
// Changing rows then drains the MMAs, so it has to be for a walk of some tiles
// (65536 x 512, statistics / softmax, ring -> held: 2 tile columns 31 -> 37 / 34 ->
// 39 us, 4 46 -> 52 / 55 -> 58, 8 78 -> 82 / 98 -> 95, 16 145 -> 146 / 186 -> 174).
bool hold_rows(const Product& p) { return p.kb <= kHeld && p.tn >= 8; }

template <int NP, bool JOIN, bool HOLD>
__global__ void __launch_bounds__(kGemmThreads, 1)
    k_loss_stats(const __grid_constant__ StatJob job) {
  using T = Tile<NP, JOIN, HOLD>;
  __shared__ GemmShared sh;
  if (job.first) {
    if (blockIdx.x == 0 && threadIdx.x < 8) job.err[threadIdx.x] = 0;
    __syncthreads();
    if (blockIdx.x == 0 && threadIdx.x == 0) tc::set_report(job.err, job.rep);
  }
  StatEpi<NP> epi(job, blockIdx.x / kPair, gridDim.x / kPair);
  gemm_roles<T>(sh, stage_memory<T>(), run_of(job.p), epi, job.err);
  if (threadIdx.x >= 128) epi.flush();
}

template <int NP, bool JOIN, bool HOLD>
__global__ void __launch_bounds__(kGemmThreads, 1)
    k_loss_softmax(const __grid_constant__ SoftJob job) {
  using T = Tile<NP, JOIN, HOLD>;
  __shared__ GemmShared sh;
  SoftEpi<NP> epi(job);
  gemm_roles<T>(sh, stage_memory<T>(), run_of(job.p), epi, job.err);
}

// ------------------------------------------------------------------ join
struct JoinJob {
  const float2* part;
  const float* zt;
  const void* targets;
  int i64;
  long long ignore, N;
  int V, tn, slots, tile_rows;
  long long tiles, workers;
  int lanes_log2;  // threads per row
  float *loss, *lse;
  float* block_sum;  // [blocks][2]
  unsigned* done;
  float* total;
};

// One row by 2^lanes_log2 threads: the partial statistics joined, the loss and
// its log-sum; then the sums over rows, by block and, by the block that is done
// last, over blocks in order.
__global__ void __launch_bounds__(256) k_loss_join(JoinJob j) {
  tc::grid_dependency_wait();
  const int lanes = 1 << j.lanes_log2, lane = threadIdx.x & (lanes - 1);
  const long long row = (long long)blockIdx.x * (256 >> j.lanes_log2) + (threadIdx.x >> j.lanes_log2);
  const bool in = row < j.N;
  LogSum a;
  if (in) {
    const long long m = row / j.tile_rows;
    const long long first = run_owner(m * j.tn, j.tiles, j.workers);
    const long long last = run_owner(m * j.tn + j.tn - 1, j.tiles, j.workers);
    const int n = (int)(last - first + 1) * 4;
    const float2* p = j.part + (size_t)m * j.slots * j.tile_rows + (row - m * j.tile_rows);
    for (int s = lane; s < n; s += lanes) {
      const float2 x = p[(size_t)s * j.tile_rows];
      a.add(x.x, x.y);
    }
  }
  for (int o = lanes >> 1; o; o >>= 1)
    a.add(__shfl_xor_sync(0xffffffffu, a.base, o), __shfl_xor_sync(0xffffffffu, a.sum, o));
  float loss = 0.0f, counted = 0.0f;
  if (in && lane == 0) {
    float lse;
    if (finish_loss(a, load_target(j.targets, j.i64, row), j.ignore, j.V, j.zt + row, loss, lse))
      counted = 1.0f;
    j.loss[row] = loss;
    j.lse[row] = lse;
  }
  // sums over the block's rows, in a fixed order
  __shared__ float sl[8], sc[8];
  __shared__ bool last;
  float ls = loss, cs = counted;
  for (int o = 16; o; o >>= 1) {
    ls += __shfl_xor_sync(0xffffffffu, ls, o);
    cs += __shfl_xor_sync(0xffffffffu, cs, o);
  }
  if ((threadIdx.x & 31) == 0) {
    sl[threadIdx.x >> 5] = ls;
    sc[threadIdx.x >> 5] = cs;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    ls = cs = 0.0f;
    for (int i = 0; i < 8; ++i) {
      ls += sl[i];
      cs += sc[i];
    }
    j.block_sum[2 * blockIdx.x] = ls;
    j.block_sum[2 * blockIdx.x + 1] = cs;
    __threadfence();
    last = atomicAdd(j.done, 1u) == gridDim.x - 1;
  }
  __syncthreads();
  if (!last) return;
  __threadfence();
  double da = 0.0, db = 0.0;
  for (unsigned i = threadIdx.x; i < gridDim.x; i += 256) {
    da += __ldcg(j.block_sum + 2 * i);
    db += __ldcg(j.block_sum + 2 * i + 1);
  }
  __shared__ double dl[8], dc[8];
  for (int o = 16; o; o >>= 1) {
    da += __shfl_xor_sync(0xffffffffu, da, o);
    db += __shfl_xor_sync(0xffffffffu, db, o);
  }
  if ((threadIdx.x & 31) == 0) {
    dl[threadIdx.x >> 5] = da;
    dc[threadIdx.x >> 5] = db;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    da = db = 0.0;
    for (int i = 0; i < 8; ++i) {
      da += dl[i];
      db += dc[i];
    }
    j.total[0] = (float)da;
    j.total[1] = (float)db;
  }
}

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
  const void* targets;
  int i64;
  long long ignore;
  int* err;
  unsigned* rep;
};

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
    if (in && which == 1 && j.last) live = load_target(j.targets, j.i64, r) != j.ignore;
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
      live = load_target(j.targets, j.i64, row) != j.ignore;
    }
    T* out = static_cast<T*>(j.to[which]) + row * D + c;
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
struct Sizes {
  long long N;
  int D, V;
  slim_dtype dtype;
  int np() const { return dtype == SLIM_F32 ? 3 : 1; }
  int ld() const { return (D + 7) / 8 * 8; }  // of a staged row
  bool even_rows() const { return D % (dtype == SLIM_F32 ? 4 : 8) == 0; }  // 16-byte pieces
  // bf16 rows that TMA can step over are read where they are
  bool stage_w() const { return dtype == SLIM_F32 || !even_rows(); }
  bool stage_x(bool bwd) const { return bwd || stage_w(); }
};

bool sizes_ok(long long N, int D, int V, slim_dtype dtype) {
  if (N < 0 || N >= (1LL << 31) - 512 || D < 1 || V < 1 || V > (1 << 30)) return false;
  if (dtype != SLIM_F32 && dtype != SLIM_BF16) return false;
  if (D > (1 << 30)) return false;  // rounded up to whole stages, 32 bits hold it
  if (N > 0 && (long long)V > (1LL << 50) / N) return false;  // a worker's tiles fit 31 bits
  return (long long)D <= (1LL << 40) / (N > 0 ? N : 1) && (long long)D <= (1LL << 40) / V;
}

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

// Partial statistics per row of a forward on `tm` x `tn` tiles.
int stat_slots(long long tm, long long tn, long long w) {
  long long s = w / tm + 2;
  if (s > tn) s = tn;
  if (s > w) s = w;
  return (int)s * 4;
}

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

struct Ws {
  int* header;        // error word, report address; [4]: the join's counter
  __nv_bfloat16 *x, *w;
  float2* part;
  float *zt, *block_sum;
  __nv_bfloat16* g;
  float *acc, *split_sum[2];
};
constexpr size_t kHeaderInts = 32;

int round_piece(int piece, int V) {
  const long long p = ((long long)(piece < V ? piece : V) + kPieceStep - 1) / kPieceStep * kPieceStep;
  return (int)p;
}
int acc_ld(int D) { return (D + 31) / 32 * 32; }

// Splits of dw and dx for a piece of n words.
void grad_splits(const Sizes& z, long long n, int splits[2]) {
  const long long tn = cdiv(z.D, kTN);
  const long long tiles[2] = {cdiv(n, kTM * kPair) * tn, cdiv(z.N, kTM * kPair) * tn};
  const long long kb[2] = {cdiv(z.N, kTK), cdiv(n, kTK)};
  split_long(tiles, kb, z.np(), kMaxWorkers / kPair, splits);
}

Ws carve(Carver& cv, const Sizes& z, int piece, bool bwd) {
  Ws w{};
  const int np = z.np();
  w.header = cv.take<int>(kHeaderInts);
  if (z.stage_x(bwd)) w.x = cv.take<__nv_bfloat16>((size_t)np * z.N * z.ld());
  if (z.stage_w()) w.w = cv.take<__nv_bfloat16>((size_t)np * z.V * z.ld());
  if (!bwd) {
    const int rows = kTM * kPair;
    const long long tm = cdiv(z.N, rows), tn = cdiv(z.V, kTN);
    w.part = cv.take<float2>((size_t)tm * stat_slots(tm, tn, kMaxWorkers / kPair) * rows);
    w.zt = cv.take<float>(z.N);
    w.block_sum = cv.take<float>(2 * (size_t)cdiv(z.N, 8));
  } else {
    const int p = round_piece(piece, z.V);
    w.g = cv.take<__nv_bfloat16>((size_t)np * z.N * p);
    if (p < z.V) w.acc = cv.take<float>((size_t)z.N * acc_ld(z.D));
    // the largest piece, and the last one if it is shorter
    size_t need[2] = {0, 0};
    const int last = z.V - (z.V - 1) / p * p;
    for (int n : {z.V < p ? z.V : p, last}) {
      int splits[2];
      grad_splits(z, n, splits);
      for (int i = 0; i < 2; ++i) {
        const bool parts = splits[i] > 1 || !z.even_rows();
        const size_t k = parts ? (size_t)splits[i] * (i ? z.N : n) * acc_ld(z.D) : 0;
        if (k > need[i]) need[i] = k;
      }
    }
    for (int i = 0; i < 2; ++i) w.split_sum[i] = cv.take<float>(need[i]);
  }
  return w;
}

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
                  long long N, long long K) {
  if (!plane_map(&p->a, a.p, a.rows, a.cols, a.ld, a.plane, NP, a_mn ? kTK : kTM) ||
      !plane_map(&p->b, b.p, b.rows, b.cols, b.ld, b.plane, NP, b_mn ? kTK : kTN / kPair))
    return false;
  p->a_mn = a_mn;
  p->b_mn = b_mn;
  p->M = (int)M;
  p->N = (int)N;
  p->tm = cdiv(M, kTM * kPair);
  p->tn = cdiv(N, kTN);
  p->kb = cdiv(K, kTK);
  p->splits = 1;
  return true;
}

template <int NP>
slim_status stage(StageJob j, cudaStream_t s) {
  using T = typename std::conditional<NP == 1, __nv_bfloat16, float>::type;
  const long long n = (j.rows[0] + j.rows[1]) * (j.ld / 8);
  const unsigned blocks = (unsigned)(cdiv(n, 256) < 152 * 8 ? cdiv(n, 256) : 152 * 8);
  prof::Scope ps(prof::K_LOSS_PREP, s, 0.0, (double)n * 8 * (sizeof(T) + 2 * NP));
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

// Calls go(join, hold) with the form of the tiles that logits `p` take, as types.
template <int NP, typename Go>
bool with_form(const Product& p, Go go) {
  using No = std::integral_constant<bool, (NP > 1)>;  // three planes: always in chains
  using Hold = std::integral_constant<bool, NP == 1>;
  return p.kb > Tile<1>::CHAIN ? go(std::true_type(), std::false_type())
         : hold_rows(p)        ? go(No(), Hold())
                               : go(No(), std::false_type());
}

template <int NP>
slim_status fwd(const Sizes& z, const void* x, const void* w, const void* targets, slim_index it,
                long long ignore, float* loss, float* lse, float* total, const Ws& ws,
                unsigned* rep, cudaStream_t s) {
  const int ld = z.ld();
  const __nv_bfloat16* xp = ws.x ? ws.x : static_cast<const __nv_bfloat16*>(x);
  const __nv_bfloat16* wp = ws.w ? ws.w : static_cast<const __nv_bfloat16*>(w);
  StatJob j{};
  if (!make_product<NP>(&j.p, Planes{xp, z.N, z.D, ld, z.N * ld}, false,
                            Planes{wp, z.V, z.D, ld, (long long)z.V * ld}, false, z.N, z.V, z.D))
    return SLIM_ERR_CUDA;
  if (ws.w) {
    const slim_status st = stage<NP>(
        StageJob{{x, w}, {ws.x, ws.w}, {z.N, z.V}, z.D, ld, nullptr, 0, 0, ws.header, rep}, s);
    if (st != SLIM_OK) return st;
  }
  j.first = ws.w == nullptr;
  const long long tiles = (long long)j.p.tm * j.p.tn;
  const long long wk = tiles < workers() ? tiles : workers();
  j.targets = targets;
  j.i64 = it == SLIM_I64;
  j.ignore = ignore;
  j.V = z.V;
  j.slots = stat_slots(j.p.tm, j.p.tn, wk);
  j.part = ws.part;
  j.zt = ws.zt;
  j.err = ws.header;
  j.rep = rep;
  {
    prof::Scope ps(prof::K_LOSS_STATS, s, 2.0 * z.N * z.D * z.V, ((double)z.N + z.V) * z.D * 2 * NP);
    const bool ok = with_form<NP>(j.p, [&](auto join, auto hold) {
      using T = Tile<NP, decltype(join)::value, decltype(hold)::value>;
      return launch<T>(k_loss_stats<NP, T::ACC, T::HOLD>, (unsigned)wk * kPair, !j.first, s, j,
                       once<StatEpi<NP>, T>());
    });
    if (!ok) return SLIM_ERR_CUDA;
  }
  JoinJob q{};
  q.part = ws.part;
  q.zt = ws.zt;
  q.targets = targets;
  q.i64 = j.i64;
  q.ignore = ignore;
  q.N = z.N;
  q.V = z.V;
  q.tn = j.p.tn;
  q.slots = j.slots;
  q.tile_rows = kTM * kPair;
  q.tiles = tiles;
  q.workers = wk;
  // neighbouring threads take neighbouring rows (their statistics lie side by
  // side); several per row only where the rows alone are too few
  while (q.lanes_log2 < 5 && (1 << q.lanes_log2) < j.slots && (z.N << q.lanes_log2) < 65536)
    ++q.lanes_log2;
  q.loss = loss;
  q.lse = lse;
  q.block_sum = ws.block_sum;
  q.done = reinterpret_cast<unsigned*>(ws.header + 4);
  q.total = total;
  prof::Scope ps(prof::K_LOSS_JOIN, s);
  return launch_on(k_loss_join, (unsigned)cdiv(z.N, 256 >> q.lanes_log2), 256, 0, 1, true, s, q)
             ? SLIM_OK
             : SLIM_ERR_CUDA;
}

template <int NP>
slim_status bwd(const Sizes& z, const void* x, const void* w, const void* targets, slim_index it,
                long long ignore, const float* lse, const float* dloss, int dstride,
                const float* count, int piece, void* dx, void* dw, const Ws& ws, unsigned* rep,
                cudaStream_t s) {
  using T = typename std::conditional<NP == 1, __nv_bfloat16, float>::type;
  const int ld = z.ld(), ps = round_piece(piece, z.V);
  const int pieces = cdiv(z.V, ps);
  const __nv_bfloat16* wp = ws.w ? ws.w : static_cast<const __nv_bfloat16*>(w);
  const slim_status st =
      stage<NP>(StageJob{{x, w}, {ws.x, ws.w}, {z.N, ws.w ? z.V : 0}, z.D, ld, targets,
                         it == SLIM_I64, ignore, ws.header, rep},
                s);
  if (st != SLIM_OK) return st;
  const Planes xm{ws.x, z.N, z.D, ld, z.N * ld};
  for (int i = 0; i < pieces; ++i) {
    const int v0 = i * ps, n = z.V - v0 < ps ? z.V - v0 : ps;
    const Planes wm{wp + (size_t)v0 * ld, n, z.D, ld, (long long)z.V * ld};
    const Planes gm{ws.g, z.N, n, ps, z.N * ps};
    SoftJob j{};
    GradJob q{};
    if (!make_product<NP>(&j.p, xm, false, wm, false, z.N, n, z.D) ||
        !make_product<NP>(&q.p[0], gm, true, xm, true, n, z.D, z.N) ||
        !make_product<NP>(&q.p[1], gm, false, wm, true, z.N, z.D, n))
      return SLIM_ERR_CUDA;
    q.to[0] = static_cast<T*>(dw) + (size_t)v0 * z.D;
    q.to[1] = dx;
    q.wide = !z.even_rows() ? 0
             : z.D * sizeof(T) % 32 == 0 && (((uintptr_t)dw | (uintptr_t)dx) & 31) == 0 ? 2 : 1;
    j.targets = q.targets = targets;
    j.i64 = q.i64 = it == SLIM_I64;
    j.ignore = q.ignore = ignore;
    j.V = z.V;
    j.v0 = v0;
    j.lse = lse;
    j.dloss = dstride ? dloss : nullptr;
    q.scale = dstride ? nullptr : dloss;
    q.count = count;
    j.g = ws.g;
    j.plane = z.N * ps;
    j.ld = ps;
    j.err = q.err = ws.header;
    j.rep = q.rep = rep;
    const double fl = 2.0 * z.N * z.D * n, gb = 2.0 * NP * z.N * n;
    const long long tiles = (long long)j.p.tm * j.p.tn;
    {
      const long long wk = tiles < workers() ? tiles : workers();
      prof::Scope sc(prof::K_LOSS_SOFTMAX, s, fl, ((double)z.N + n) * z.D * 2 * NP + gb);
      const bool ok = with_form<NP>(j.p, [&](auto join, auto hold) {
        using T = Tile<NP, decltype(join)::value, decltype(hold)::value>;
        return launch<T>(k_loss_softmax<NP, T::ACC, T::HOLD>, (unsigned)wk * kPair, true, s, j,
                         once<SoftEpi<NP>, T>());
      });
      if (!ok) return SLIM_ERR_CUDA;
    }
    q.acc = ws.acc;
    q.acc_ld = acc_ld(z.D);
    q.first = i == 0;
    q.last = i == pieces - 1;
    int splits[2];
    grad_splits(z, n, splits);
    q.parts[0] = splits[0] > 1 || !q.wide;
    q.parts[1] = splits[1] > 1 || (!q.wide && q.last);
    long long nt[2], cost[2];
    for (int k = 0; k < 2; ++k) {
      q.p[k].splits = splits[k];
      q.part[k] = ws.split_sum[k];
      nt[k] = (long long)q.p[k].tm * q.p[k].tn * splits[k];
      cost[k] = cdiv(q.p[k].kb, splits[k]);
    }
    const int wk = (int)(nt[0] + nt[1] < workers() ? nt[0] + nt[1] : workers());
    deal_tiles(nt, cost, wk, &q.deal);
    prof::Scope sc(prof::K_LOSS_GRAD, s, 2 * fl, ((double)z.N + n) * z.D * 2 * NP + 2 * gb);
    if (!launch<Tile<NP>>(k_loss_grad<NP>, (unsigned)wk * kPair, true, s, q,
                              once<GradEpi<NP>>()))
      return SLIM_ERR_CUDA;
    if (q.parts[0] || q.parts[1]) {
      const long long e = ((q.parts[0] ? n : 0) + (q.parts[1] ? z.N : 0)) * cdiv(z.D, 4);
      prof::Scope sp(prof::K_LOSS_PARTS, s);
      if (!launch_on(k_loss_parts<T>, (unsigned)(cdiv(e, 256) < 152 * 8 ? cdiv(e, 256) : 152 * 8),
                     256, 0, 1, true, s, q))
        return SLIM_ERR_CUDA;
    }
  }
  return SLIM_OK;
}

bool aligned(const void* p, size_t to) {
  return p != nullptr && (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0;
}

}  // namespace
}  // namespace lm
}  // namespace slim

extern "C" slim_status slim_vocab_loss_workspace_size(long long N, int D, int V, slim_dtype dtype,
                                                      int piece, int backward, size_t* bytes) {
  using namespace slim::lm;
  if (!bytes || !sizes_ok(N, D, V, dtype) || (backward && piece < 1)) return SLIM_ERR_INVALID_ARG;
  if (rows_fit(N, D, dtype)) {
    *bytes = rows_workspace((int)N, D, V, backward != 0);
    return SLIM_OK;
  }
  slim::Carver cv(nullptr);
  carve(cv, Sizes{N, D, V, dtype}, piece, backward != 0);
  *bytes = cv.bytes();
  return SLIM_OK;
}

extern "C" slim_status slim_vocab_loss_fwd(const void* x, const void* w, const void* targets,
                                           slim_index itype, long long N, int D, int V,
                                           slim_dtype dtype, long long ignore_index, float* loss,
                                           float* lse, float* total, void* workspace,
                                           size_t workspace_bytes, void* stream) {
  using namespace slim::lm;
  if (!sizes_ok(N, D, V, dtype) || (itype != SLIM_I32 && itype != SLIM_I64))
    return SLIM_ERR_INVALID_ARG;
  if (!aligned(w, 16) || !aligned(total, 4)) return SLIM_ERR_INVALID_ARG;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (N == 0)
    return cudaMemsetAsync(total, 0, 2 * sizeof(float), s) == cudaSuccess ? SLIM_OK : SLIM_ERR_CUDA;
  if (!aligned(x, 16) || !aligned(targets, itype == SLIM_I64 ? 8 : 4) || !aligned(loss, 4) ||
      !aligned(lse, 4))
    return SLIM_ERR_INVALID_ARG;
  size_t need = 0;
  slim_vocab_loss_workspace_size(N, D, V, dtype, 1, 0, &need);
  if (workspace == nullptr || workspace_bytes < need) return SLIM_ERR_WORKSPACE;
  if (!aligned(workspace, 256)) return SLIM_ERR_INVALID_ARG;
  unsigned* rep = nullptr;
  const bool rows = rows_fit(N, D, dtype);
  const slim_status st =
      rows ? slim::report::pending(workspace) : slim::report::begin(workspace, true, &rep);
  if (st != SLIM_OK) return st;
  if (rows)
    return rows_fwd(x, w, targets, itype, (int)N, D, V, dtype, ignore_index, loss, lse, total,
                    workspace, s);
  const Sizes z{N, D, V, dtype};
  slim::Carver cv(workspace);
  const Ws ws = carve(cv, z, 1, false);
  if (dtype == SLIM_BF16)
    return fwd<1>(z, x, w, targets, itype, ignore_index, loss, lse, total, ws, rep, s);
  return fwd<3>(z, x, w, targets, itype, ignore_index, loss, lse, total, ws, rep, s);
}

extern "C" slim_status slim_vocab_loss_bwd(const void* x, const void* w, const void* targets,
                                           slim_index itype, const float* lse, const float* dloss,
                                           int dloss_stride, const float* count, long long N, int D,
                                           int V, slim_dtype dtype, int piece,
                                           long long ignore_index, void* dx, void* dw,
                                           void* workspace, size_t workspace_bytes, void* stream) {
  using namespace slim::lm;
  if (!sizes_ok(N, D, V, dtype) || (itype != SLIM_I32 && itype != SLIM_I64) || piece < 1 ||
      (dloss_stride & ~1))
    return SLIM_ERR_INVALID_ARG;
  if (!aligned(w, 16) || !aligned(dw, 16) || (count && !aligned(count, 4)))
    return SLIM_ERR_INVALID_ARG;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (N == 0) {
    const size_t n = (size_t)V * D * (dtype == SLIM_F32 ? 4 : 2);
    return cudaMemsetAsync(dw, 0, n, s) == cudaSuccess ? SLIM_OK : SLIM_ERR_CUDA;
  }
  if (!aligned(x, 16) || !aligned(targets, itype == SLIM_I64 ? 8 : 4) || !aligned(lse, 4) ||
      !aligned(dloss, 4) || !aligned(dx, 16))
    return SLIM_ERR_INVALID_ARG;
  size_t need = 0;
  slim_vocab_loss_workspace_size(N, D, V, dtype, piece, 1, &need);
  if (workspace == nullptr || workspace_bytes < need) return SLIM_ERR_WORKSPACE;
  if (!aligned(workspace, 256)) return SLIM_ERR_INVALID_ARG;
  unsigned* rep = nullptr;
  const bool rows = rows_fit(N, D, dtype);
  const slim_status st =
      rows ? slim::report::pending(workspace) : slim::report::begin(workspace, true, &rep);
  if (st != SLIM_OK) return st;
  if (rows)
    return rows_bwd(x, w, targets, itype, lse, dloss, dloss_stride, count, (int)N, D, V, dtype,
                    ignore_index, dx, dw, workspace, s);
  const Sizes z{N, D, V, dtype};
  slim::Carver cv(workspace);
  const Ws ws = carve(cv, z, piece, true);
  if (dtype == SLIM_BF16)
    return bwd<1>(z, x, w, targets, itype, ignore_index, lse, dloss, dloss_stride, count,
                       piece, dx, dw, ws, rep, s);
  return bwd<3>(z, x, w, targets, itype, ignore_index, lse, dloss, dloss_stride, count, piece,
                     dx, dw, ws, rep, s);
}
