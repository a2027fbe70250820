// Tile products of the vocabulary loss on the tcgen05 tensor cores: the roles
// of a persistent, warp-specialised kernel that computes D = A B^T tiles with
// an epilogue of its caller's.
//
// A pair of blocks works on a tile, each on half of its rows, and runs three roles
// side by side: a warp of each block copies its operand tiles into a ring of
// shared-memory stages by TMA, a warp of the leading block issues the MMAs on them
// (one lane of either issues), and sixteen warps a block read finished accumulators
// from TMEM and run the epilogue.  Two accumulators alternate, so a tile's epilogue
// runs under the next tile's MMAs.
//
// Operands are planes of bf16 matrices, K-major ([rows][K]) or MN-major
// ([K][rows]); coordinates past an edge read as zero.  NP = 3: a value is the
// sum of its three planes' values, and the product is the sum of the six plane
// products down to 2^-16 of the largest.
//
// The tensor core cuts off the last bits at every step of a sum: measured, a
// sum of 512 bf16 products comes out low by 4e-7 of itself and one of 2048 by
// 1.7e-6 (9e-7 and 5.7e-6 where all have one sign; 6.6e-3 over 2^20 terms).  ACC: a sum is cut into
// chains that the epilogue's registers join in fp32, where that loss would show in
// an fp32 result.
#pragma once
#include "common.cuh"
#include "tc_common.cuh"

namespace slim {
namespace lm {

constexpr int kPair = 2;           // blocks of a tile
constexpr int kTM = 128;           // rows of a block's half of a tile
constexpr int kTN = 256;           // columns of a tile
constexpr int kTK = 64;            // reduction per stage
constexpr int kEpiWarps = 16;      // four per quarter of the rows, 64 columns each
constexpr int kEpiCols = kTN / 4;
constexpr int kGemmThreads = 128 + 32 * kEpiWarps;  // warps: TMA, MMA, TMEM, spare, epilogue

constexpr int kSmemBytes = 227 * 1024 - 1024 - 512;  // after alignment and barriers
// HOLD: a block keeps its rows of a short A (up to kHeld stages, K-major) in
// shared memory while it stays with the same tile row, and the ring carries B
// alone.  Worth it where a worker walks along many columns.
constexpr int kHeld = 8;
template <int NP, bool JOIN = (NP > 1), bool HOLD_A = false>
struct Tile {
  static constexpr int PLANES = NP;
  static constexpr bool ACC = JOIN, HOLD = HOLD_A;
  static_assert(!HOLD || NP == 1, "one plane");
  static constexpr int BROWS = kTN / kPair;    // rows of B that a block holds
  static constexpr int A_BYTES = kTM * kTK * 2, B_BYTES = BROWS * kTK * 2;
  static constexpr int HELD_BYTES = HOLD ? kHeld * A_BYTES : 0;
  static constexpr int STAGE = HOLD ? B_BYTES : A_BYTES + B_BYTES;  // one plane of either operand
  static constexpr int FIT = (kSmemBytes - HELD_BYTES) / STAGE;
  static constexpr int STAGES = FIT < 8 ? FIT : 8;
  // chains of 512 of the reduction, or of 64 with three planes: there only the
  // last four steps, the large planes', work on a large sum
  static constexpr int CHAIN = NP == 1 ? 8 : 1;
  static constexpr size_t smem() { return 1024 + HELD_BYTES + (size_t)STAGES * STAGE; }
  static_assert(STAGES >= 3, "a stage per plane");
};

// One product: D [M, N] = sum over K of A and B.
struct Product {
  CUtensorMap a, b;
  int a_mn, b_mn;  // operand layouts: 0 K-major, 1 MN-major
  int M, N;
  int tm, tn;      // tiles each way (tm in tiles of kTM * kPair rows)
  int kb;          // stages (of kTK) of the reduction
  int splits;      // parts of the reduction, computed as tiles of their own
};

// One tile: stages [k0, k1) of product p's reduction.
struct Work {
  const Product* p;
  int m, n, split, k0, k1;
};
// A contiguous range of a product's tiles, columns and splits fastest.  It is
// walked by counting: a division per tile would hold up every role.
struct TileRange {
  const Product* p;
  int m, n, split;
  int left;
  __device__ __forceinline__ TileRange(const Product* q, long long begin, long long end)
      : p(q), left((int)(end - begin)) {
    const long long tile = begin / q->splits;
    split = (int)(begin - tile * q->splits);
    m = (int)(tile / q->tn);
    n = (int)(tile - (long long)m * q->tn);
  }
  __device__ __forceinline__ bool next(Work& w) {
    if (left <= 0) return false;
    --left;
    w.p = p;
    w.m = m;
    w.n = n;
    w.split = split;
    w.k0 = 0;
    w.k1 = p->kb;
    if (p->splits > 1) {
      w.k0 = (int)((long long)split * p->kb / p->splits);
      w.k1 = (int)((long long)(split + 1) * p->kb / p->splits);
    }
    if (++split == p->splits) {
      split = 0;
      if (++n == p->tn) {
        n = 0;
        ++m;
      }
    }
    return true;
  }
};

struct GemmShared {
  uint64_t full[8], empty[8], tfull[2], tempty[2];
  uint64_t held, unheld;  // HOLD: the rows are there; no MMA reads them any more
  uint32_t tmem;
};

// ------------------------------------------------------------------ cluster
__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ uint32_t map_to_rank(uint32_t addr, uint32_t rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
  return r;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ void arrive_at_leader(uint32_t bar) {
    // what it hands over is TMEM, read by completed tcgen05.ld: nothing in memory
    // has to be made visible to the other block (a release at cluster scope
    // waits for the warp's earlier stores, 0.5 us a tile)
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(map_to_rank(bar, 0))
                 : "memory");
}

// ------------------------------------------------------------------ pair forms
__device__ __forceinline__ void gemm_tmem_alloc(uint32_t dst, uint32_t cols) {
  asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(dst),
               "r"(cols)
               : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void gemm_tmem_free(uint32_t t, uint32_t cols) {
  asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(t), "r"(cols)
               : "memory");
}
__device__ __forceinline__ void gemm_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc,
                                         uint32_t acc) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(acc)
      : "memory");
}
// Arrives on the mbarrier of both blocks once this thread's MMAs so far are done.
__device__ __forceinline__ void gemm_commit(uint32_t bar) {
  asm volatile(
      "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 "
      "[%0], %1;" ::"r"(bar),
      "h"((uint16_t)3)
      : "memory");
}
// One box of a tensor map to shared memory; x is a multiple of 64 elements
// (128 bytes).  The bytes are counted on the leading block's barrier.
__device__ __forceinline__ void gemm_tma(uint32_t dst, const CUtensorMap* map, int x, int y, int z,
                                         uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes "
      "[%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(bar)
      : "memory");
}

// ------------------------------------------------------------------ roles
// Sets the ring up and allocates TMEM; every thread of the block (of the pair).
template <typename T>
__device__ __forceinline__ void gemm_begin(GemmShared& sh) {
  if (threadIdx.x == 0) {
    for (int i = 0; i < T::STAGES; ++i) {
      tc::mbar_init(tc::smem_u32(&sh.full[i]), 1);
      tc::mbar_init(tc::smem_u32(&sh.empty[i]), 1);
    }
    tc::mbar_init(tc::smem_u32(&sh.held), 1);
    tc::mbar_init(tc::smem_u32(&sh.unheld), 1);
    for (int i = 0; i < 2; ++i) {
      tc::mbar_init(tc::smem_u32(&sh.tfull[i]), 1);
      tc::mbar_init(tc::smem_u32(&sh.tempty[i]), kEpiWarps * kPair);
    }
    tc::mbar_fence_init();
  }
  if (threadIdx.x / 32 == 2) gemm_tmem_alloc(tc::smem_u32(&sh.tmem), 2 * kTN);
  tc::tc_fence_before();
  cluster_sync();
  tc::tc_fence_after();
}

template <typename T>
__device__ __forceinline__ void gemm_end(GemmShared& sh, bool failed) {
  // a role that gave up may leave copies in flight: let them land
  if (failed)
    for (int i = 0; i < 1000; ++i) __nanosleep(10000);
  tc::tc_fence_before();
  cluster_sync();
  if (threadIdx.x / 32 == 2) gemm_tmem_free(sh.tmem, 2 * kTN);
}

// A bounded wait of a whole warp: false for all lanes if one of them gave up.
// What follows takes a full warp (tcgen05.ld, the block's and the pair's
// barriers), also when the wait ran out.
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, int* err) {
  return __all_sync(0xffffffffu, tc::mbar_wait(bar, parity, err));
}

// One lane of a converged warp, the same every time.  ptxas knows that a branch
// on it holds one thread, and keeps what the MMAs take in uniform registers.
__device__ __forceinline__ bool elect_one() {
  uint32_t p;
  asm volatile(
      "{\n\t.reg .pred P;\n\t"
      "elect.sync _|P, 0xffffffff;\n\t"
      "selp.u32 %0, 1, 0, P;\n\t}"
      : "=r"(p));
  return p != 0;
}

// A value that all lanes agree on, told to the compiler as such: what an MMA and
// its loop take comes from uniform registers.
template <typename V>
__device__ __forceinline__ V uniform(V x) {
  return __shfl_sync(0xffffffffu, x, 0);
}
__device__ __forceinline__ const CUtensorMap* uniform(const CUtensorMap* x) {
  return reinterpret_cast<const CUtensorMap*>(
      __shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(x), 0));
}

// The copying warp.  `next(work)` yields this worker's tiles in order: the same
// sequence in every role.  All lanes walk the loop and one of them issues, as for
// the MMAs: a lone thread with its operands in ordinary registers took 600
// cycles for a stage's four copies, more than the stage's MMAs.  False if a wait
// gave up.
template <typename T, typename Next>
__device__ bool gemm_copy(GemmShared& sh, uint8_t* stages, Next next, int* err) {
  constexpr int NP = T::PLANES;
  const int rank = uniform((int)cluster_rank());
  const uint32_t full0 = tc::smem_u32(&sh.full[0]), empty0 = tc::smem_u32(&sh.empty[0]);
  const uint32_t count0 = map_to_rank(full0, 0);  // the leading block's
  const uint32_t smem = tc::smem_u32(stages);
  uint32_t st = 0, phase = 1, held_phase = 0;
  int held_row = -1;
  auto step_on = [&] {
    if (++st == T::STAGES) {
      st = 0;
      phase ^= 1;
    }
  };
  auto free = [&] { return warp_wait(empty0 + 8 * st, phase, err); };
  Work w;
  while (next(w)) {
    const CUtensorMap* map_a = uniform(&w.p->a);
    const CUtensorMap* map_b = uniform(&w.p->b);
    const int a_mn = uniform(w.p->a_mn), b_mn = uniform(w.p->b_mn);
    const int row = uniform((w.m * kPair + rank) * kTM), col = uniform(w.n * kTN + rank * T::BROWS);
    const int k0 = uniform(w.k0) * kTK, k1 = uniform(w.k1) * kTK;
    if (T::HOLD && row != held_row) {
      if (held_row >= 0) {
        if (!warp_wait(tc::smem_u32(&sh.unheld), held_phase, err)) return false;
        held_phase ^= 1;
      }
      held_row = row;
      if (elect_one()) {
        const uint32_t held = tc::smem_u32(&sh.held);
        if (rank == 0) tc::mbar_expect_tx(held, kPair * (k1 - k0) / kTK * T::A_BYTES);
        const uint32_t bar = map_to_rank(held, 0);
        for (int k = k0; k < k1; k += kTK)
          gemm_tma(smem + (k - k0) / kTK * T::A_BYTES, map_a, k, row, 0, bar);
      }
      __syncwarp();
    }
    for (int k = k0; k < k1; k += kTK) {
#pragma unroll 1
      for (int q = 0; q < NP; ++q) {
        if (!free()) return false;
        if (elect_one()) {
          if (rank == 0) tc::mbar_expect_tx(full0 + 8 * st, kPair * T::STAGE);
          const uint32_t full = count0 + 8 * st;
          const uint32_t sa = smem + T::HELD_BYTES + st * T::STAGE;
          const uint32_t sb = T::HOLD ? sa : sa + T::A_BYTES;
          if (T::HOLD) {
            // the rows are held
          } else if (a_mn) {
#pragma unroll
            for (int j = 0; j < kTM / 64; ++j)
              gemm_tma(sa + j * 8192, map_a, row + 64 * j, k, q, full);
          } else {
            gemm_tma(sa, map_a, k, row, q, full);
          }
          if (b_mn) {
#pragma unroll
            for (int j = 0; j < T::BROWS / 64; ++j)
              gemm_tma(sb + j * 8192, map_b, col + 64 * j, k, q, full);
          } else {
            gemm_tma(sb, map_b, k, col, q, full);
          }
        }
        __syncwarp();
        step_on();
      }
    }
  }
  // every stage handed back: no arrival is on its way when the block leaves
  for (int i = 0; i < T::STAGES; ++i) {
    if (!free()) return false;
    step_on();
  }
  return true;
}

// The warp that issues MMAs (of the leading block of a pair).  All lanes walk
// the loop; one of them issues.
template <typename T, typename Next>
__device__ bool gemm_multiply(GemmShared& sh, uint8_t* stages, Next next, int* err) {
  Work w;
  const uint32_t full0 = tc::smem_u32(&sh.full[0]), empty0 = tc::smem_u32(&sh.empty[0]);
  const uint32_t tmem = sh.tmem;
  uint32_t st = 0, phase = 0, acc = 0, held_phase = 0;
  int held_m = -1;
  auto step_on = [&](uint32_t& s, uint32_t& ph) {
    if (++s == T::STAGES) {
      s = 0;
      ph ^= 1;
    }
  };
  auto wait = [&](uint32_t bar, uint32_t parity) {
    const bool ok = warp_wait(bar, parity, err);
    tc::tc_fence_after();
    return ok;
  };
  while (next(w)) {
    const int a_mn = uniform(w.p->a_mn), b_mn = uniform(w.p->b_mn);
    const int first = uniform(w.k0), last = uniform(w.k1);
    const uint32_t idesc = tc::idesc_bf16(kTM * kPair, kTN, a_mn, b_mn);
    const uint32_t a_step = a_mn ? 128 : 2, b_step = b_mn ? 128 : 2;
    const uint32_t ring = tc::smem_u32(stages) + T::HELD_BYTES;
    const uint64_t a0 = tc::sdesc(tc::smem_u32(stages), a_mn ? 8192 : 16, 1024);
    const uint64_t b0 = tc::sdesc(T::HOLD ? ring : ring + T::A_BYTES, b_mn ? 8192 : 16, 1024);
    if (T::HOLD && uniform(w.m) != held_m) {
      if (held_m >= 0 && elect_one()) gemm_commit(tc::smem_u32(&sh.unheld));
      __syncwarp();
      held_m = uniform(w.m);
      if (!wait(tc::smem_u32(&sh.held), held_phase)) return false;
      held_phase ^= 1;
    }
    const int step = T::ACC ? T::CHAIN : last - first;
    for (int k0 = first; k0 < last; k0 += step, ++acc) {
      const uint32_t buf = acc & 1;
      if (!wait(tc::smem_u32(&sh.tempty[buf]), ((acc >> 1) & 1) ^ 1)) return false;
      const uint32_t d = tmem + buf * kTN;
      uint32_t more = 0;
      // by the issuing lane
      auto product = [&](uint32_t ia, uint32_t ib) {
        const uint64_t da = a0 + ia * ((T::HOLD ? T::A_BYTES : T::STAGE) >> 4);
        const uint64_t db = b0 + ib * (T::STAGE >> 4);
#pragma unroll
        for (int j = 0; j < kTK / 16; ++j)
          gemm_mma(d, da + j * a_step, db + j * b_step, idesc, j == 0 ? more : 1u);
      };
      auto done = [&](uint32_t i) { gemm_commit(empty0 + 8 * i); };
      const int k1 = min(k0 + step, last);
      for (int k = k0; k < k1; ++k) {
        uint32_t s[3];
#pragma unroll
        for (int q = 0; q < T::PLANES; ++q) {
          s[q] = st;
          if (!wait(full0 + 8 * st, phase)) return false;
          step_on(st, phase);
        }
        if (elect_one()) {
          if (T::PLANES > 1) {
            // smallest products first: what each step cuts off is in
            // proportion to the sum so far
            product(s[0], s[2]);
            more = 1;
            product(s[2], s[0]);
            done(s[2]);
            product(s[1], s[1]);
            product(s[0], s[1]);
            product(s[1], s[0]);
            done(s[1]);
          }
          product(T::HOLD ? k - first : s[0], s[0]);
          done(s[0]);
        }
        more = 1;
        __syncwarp();
      }
      if (elect_one()) gemm_commit(tc::smem_u32(&sh.tfull[buf]));
      __syncwarp();
    }
  }
  return true;
}

// An epilogue warp.  For every tile, epi.begin(work, row, col0) once, then
// epi.chunk(c, v) for each 32 columns col0 + c .. of row `row` (of this thread)
// that begin inside the product (v is the epilogue's to change).  Reads past the
// product's rows still run (their values are zero sums); the epilogue drops them.
template <typename T, typename Next, typename Epi>
__device__ bool gemm_finish(GemmShared& sh, Next next, Epi& epi, int* err) {
  const uint32_t rank = cluster_rank();
  const int warp = threadIdx.x / 32 - 4, lane = threadIdx.x & 31;
  const int quarter = warp & 3, part = warp >> 2;
  Work w;
  uint32_t acc = 0;
  while (next(w)) {
    const Product* p = w.p;
    const int row = (w.m * kPair + (int)rank) * kTM + quarter * 32 + lane;
    const int col = w.n * kTN + part * kEpiCols;
    const int step = T::ACC ? T::CHAIN : w.k1 - w.k0;
    float sum[T::ACC ? kEpiCols : 1];
    if (T::ACC) {
#pragma unroll
      for (int c = 0; c < kEpiCols; ++c) sum[c] = 0.0f;
    }
    epi.begin(w, row, col);
    for (int k0 = w.k0; k0 < w.k1; k0 += step, ++acc) {
      const int buf = acc & 1;
      if (!warp_wait(tc::smem_u32(&sh.tfull[buf]), (acc >> 1) & 1, err)) return false;
      tc::tc_fence_after();
      const uint32_t t =
          sh.tmem + buf * kTN + part * kEpiCols + ((uint32_t)(quarter * 32) << 16);
      if (T::ACC) {
#pragma unroll
        for (int c = 0; c < kEpiCols; c += 16) {
          float v[16];
          tc::tmem_ld16(t + c, v);
#pragma unroll
          for (int i = 0; i < 16; ++i) sum[c + i] += v[i];
        }
      } else {
#pragma unroll 1
        for (int c = 0; c < kEpiCols && col + c < p->N; c += 32) {
          float v[32];
          __syncwarp();
          tc::tmem_ld32(t + c, v);
          epi.chunk(c, v);
        }
      }
      tc::tc_fence_before();
      __syncwarp();
      if (lane == 0) arrive_at_leader(tc::smem_u32(&sh.tempty[buf]));
    }
    if (T::ACC) {
#pragma unroll
      for (int c = 0; c < kEpiCols; c += 32)
        if (col + c < p->N) epi.chunk(c, &sum[c]);
    }
  }
  return true;
}

// All roles of a kernel's block.  Epi is made by the caller; workers iterate with
// `next`.
template <typename T, typename Next, typename Epi>
__device__ __forceinline__ void gemm_roles(GemmShared& sh, uint8_t* stages, const Next& next,
                                           Epi& epi, int* err) {
  gemm_begin<T>(sh);
  tc::grid_dependency_wait();  // set up under the previous kernel's end
  const int warp = uniform((int)threadIdx.x / 32);
  bool ok = true;
  // With ACC the epilogue holds 64 sums a thread: the first warpgroup hands its
  // registers over.  A block starts with 640 x 96 = 61440; 128 x 32 + 512 x 112 are
  // as many after the split.
  if (warp < 4) {
    if (T::ACC) asm volatile("setmaxnreg.dec.sync.aligned.u32 32;");
    if (warp == 0)
      ok = gemm_copy<T>(sh, stages, next, err);
    else if (warp == 1 && (cluster_rank() == 0))
      ok = gemm_multiply<T>(sh, stages, next, err);
  } else {
    if (T::ACC) asm volatile("setmaxnreg.inc.sync.aligned.u32 112;");
    ok = gemm_finish<T>(sh, next, epi, err);
  }
  __syncwarp();
  gemm_end<T>(sh, !ok);
}

// ------------------------------------------------------------------ rows to memory
// A lane holds 32 columns of its own row.  It moves them in whole 32-byte
// sectors: a 256 x 256 tile of bf16 took 5.6 k cycles this way under the next
// tile's MMAs (5.1 k without a store), 7.9 k with 16-byte stores, and 6.5 k
// through shared memory and TMA, which compete with the MMAs' operands.  Past
// L1, whose lines are the same memory: 6 % of the softmax kernel.
__device__ __forceinline__ void store32(void* p, const uint32_t* u) {
  asm volatile("st.global.L1::no_allocate.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(u[0]),
               "r"(u[1]), "r"(u[2]), "r"(u[3]), "r"(u[4]), "r"(u[5]), "r"(u[6]), "r"(u[7])
               : "memory");
}
__device__ __forceinline__ void load32(const void* p, uint32_t* u) {
  asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]),
                 "=r"(u[7])
               : "l"(p)
               : "memory");
}

}  // namespace lm
}  // namespace slim
