// Embedding lookup with scaling, and the gradient of its table by sorted
// tokens.  Contract: include/slim_lm.h.
//
// Forward: out_i = scale * table[ids_i].  One read and one write per element
// and no reuse, so HBM bounds it; a group of threads copies a row in the widest
// vectors its width allows.
//
// Gradient: dtable_v = scale * sum_{i: ids_i = v} dout_i.  The tokens are
// sorted by id with a stable radix sort (8-bit digits, only the bits that V
// needs), which turns the scatter into sums over runs of equal ids in order of
// position.  The sorted list is cut into chunks of equal length, whatever the
// ids: a frequent token's run is spread over many chunks and a rare token's
// shares one, so the work is even.  A run inside one chunk is summed in
// registers and written once; a run that crosses chunks leaves a partial row
// per chunk, which a last kernel adds in order.  Every sum has a fixed order.
#include <stdint.h>

#include "../../include/slim_lm.h"
#include "common.cuh"
#include "profiler.h"

namespace slim {
namespace lm {
namespace {

constexpr int kSMs = 152;

// ------------------------------------------------------------------ vectors
// VB bytes of T, as EPV fp32 values.
template <int VB> struct Raw;
template <> struct Raw<16> { using type = uint4; };
template <> struct Raw<8> { using type = uint2; };
template <> struct Raw<4> { using type = uint32_t; };
template <> struct Raw<2> { using type = uint16_t; };

template <typename T, int VB>
struct Vec {
  static constexpr int n = VB / (int)sizeof(T);
  union {
    typename Raw<VB>::type raw;
    T e[n];
  };
  __device__ __forceinline__ Vec() {}
  __device__ __forceinline__ void load(const T* p) {
    raw = *reinterpret_cast<const typename Raw<VB>::type*>(p);
  }
  __device__ __forceinline__ void store(T* p) const {
    *reinterpret_cast<typename Raw<VB>::type*>(p) = raw;
  }
  __device__ __forceinline__ float get(int i) const { return Io<T>::load(e, i); }
  __device__ __forceinline__ void set(int i, float x) { Io<T>::store(e, i, x); }
};

// The widest vector (bytes) that divides a row of D elements.
int vec_bytes(int D, int es) {
  const long long row = (long long)D * es;
  for (int vb = 16; vb > es; vb >>= 1)
    if (row % vb == 0) return vb;
  return es;
}

// Threads of a group that shares one row of U vectors: a power of two, at most
// 256, at least enough for `per` vectors a thread.
int group_log2(long long U, int per) {
  int l = 0;
  while (l < 8 && ((long long)per << l) < U) ++l;
  return l;
}

__device__ __forceinline__ long long load_id(const void* ids, int i64, long long i) {
  return i64 ? static_cast<const long long*>(ids)[i] : static_cast<const int*>(ids)[i];
}

// ------------------------------------------------------------------ forward
constexpr int kFwdItems = 4;

template <typename T, int VB>
__global__ void __launch_bounds__(256) k_embed_fwd(const void* ids, int i64, const T* table,
                                                   long long N, int D, int V, int U, int gl,
                                                   float scale, T* out) {
  constexpr int n = Vec<T, VB>::n;
  const int g = 1 << gl, lane = threadIdx.x & (g - 1);
  const long long row = (long long)blockIdx.x * (256 >> gl) + (threadIdx.x >> gl);
  if (row >= N) return;
  const long long id = load_id(ids, i64, row);
  const bool in = id >= 0 && id < V;
  const T* src = table + (size_t)(in ? id : 0) * D;
  T* dst = out + (size_t)row * D;
  for (int u0 = lane; u0 < U; u0 += g * kFwdItems) {
    Vec<T, VB> v[kFwdItems];
#pragma unroll
    for (int j = 0; j < kFwdItems; ++j)
      if (u0 + j * g < U && in) v[j].load(src + (size_t)(u0 + j * g) * n);
#pragma unroll
    for (int j = 0; j < kFwdItems; ++j) {
      if (u0 + j * g >= U) break;
#pragma unroll
      for (int e = 0; e < n; ++e) v[j].set(e, in ? v[j].get(e) * scale : 0.0f);
      v[j].store(dst + (size_t)(u0 + j * g) * n);
    }
  }
}

// ------------------------------------------------------------------ sort
// Keys are ids, with every id outside the table mapped to V, so that padding
// sorts behind all rows.
constexpr int kRadixBits = 8, kRadix = 1 << kRadixBits;
constexpr int kSortThreads = 1024, kSortWarps = kSortThreads / 32;

struct SortSrc {
  const void* ids;  // first pass: the caller's ids; later passes: null
  int i64, V;
  const uint32_t *key, *pos;
  __device__ __forceinline__ uint32_t key_at(long long i) const {
    if (!ids) return key[i];
    const long long id = load_id(ids, i64, i);
    return id >= 0 && id < V ? (uint32_t)id : (uint32_t)V;
  }
  __device__ __forceinline__ uint32_t pos_at(long long i) const {
    return ids ? (uint32_t)i : pos[i];
  }
};

// Digit counts of [a, e) added to hist[kRadix] (shared memory), one atomic per
// distinct digit of a warp.
__device__ void count_digits(const SortSrc& s, long long a, long long e, int shift,
                             uint32_t* hist) {
  for (long long i0 = a; i0 < e; i0 += kSortThreads) {
    const long long i = i0 + threadIdx.x;
    const uint32_t d = i < e ? (s.key_at(i) >> shift) & (kRadix - 1) : kRadix;
    const unsigned peers = __match_any_sync(0xffffffffu, d);
    if (d < kRadix && (peers & ((1u << (threadIdx.x & 31)) - 1)) == 0)
      atomicAdd(&hist[d], (uint32_t)__popc(peers));
  }
}

// Exclusive prefix sum of x[kRadix] (shared memory) in place, by all threads.
__device__ void scan_digits(uint32_t* x, uint32_t* warp_sum) {
  const int t = threadIdx.x, lane = t & 31, w = t >> 5;
  uint32_t v = 0, inc = 0;
  if (t < kRadix) {
    v = inc = x[t];
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t y = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += y;
    }
    if (lane == 31) warp_sum[w] = inc;
  }
  __syncthreads();
  if (t < kRadix) {
    uint32_t before = 0;
    for (int i = 0; i < w; ++i) before += warp_sum[i];
    x[t] = before + inc - v;
  }
  __syncthreads();
}

// Scatters [a, e) stably by digit; base[d] is where this range's first item
// with digit d goes, and is advanced.
__device__ void scatter_range(const SortSrc& s, long long a, long long e, int shift,
                              uint32_t (*wh)[kRadix], uint32_t* base, uint32_t* key_out,
                              uint32_t* pos_out) {
  const int t = threadIdx.x, lane = t & 31, w = t >> 5;
  for (long long i0 = a; i0 < e; i0 += kSortThreads) {
    for (int x = t; x < kSortWarps * kRadix; x += kSortThreads) (&wh[0][0])[x] = 0;
    __syncthreads();
    const long long i = i0 + t;
    const bool on = i < e;
    uint32_t key = 0, pos = 0, d = kRadix;
    if (on) {
      key = s.key_at(i);
      pos = s.pos_at(i);
      d = (key >> shift) & (kRadix - 1);
    }
    const unsigned peers = __match_any_sync(0xffffffffu, d);
    const uint32_t rank = __popc(peers & ((1u << lane) - 1));
    if (on && rank == 0) wh[w][d] = __popc(peers);
    __syncthreads();
    if (t < kRadix) {  // counts of the warps -> first place of each warp's items
      uint32_t run = base[t];
      for (int x = 0; x < kSortWarps; ++x) {
        const uint32_t c = wh[x][t];
        wh[x][t] = run;
        run += c;
      }
      base[t] = run;
    }
    __syncthreads();
    if (on) {
      const uint32_t at = wh[w][d] + rank;
      key_out[at] = key;
      pos_out[at] = pos;
    }
    __syncthreads();
  }
}

__global__ void __launch_bounds__(kSortThreads) k_sort_count(SortSrc s, long long N, int tile,
                                                             int shift, uint32_t* cnt,
                                                             int* header) {
  __shared__ uint32_t hist[kRadix];
  if (blockIdx.x == 0 && threadIdx.x < 4) header[threadIdx.x] = 0;
  if (threadIdx.x < kRadix) hist[threadIdx.x] = 0;
  __syncthreads();
  const long long a = (long long)blockIdx.x * tile, e = a + tile < N ? a + tile : N;
  count_digits(s, a, e, shift, hist);
  __syncthreads();
  if (threadIdx.x < kRadix) cnt[blockIdx.x * kRadix + threadIdx.x] = hist[threadIdx.x];
}

__global__ void __launch_bounds__(kSortThreads) k_sort_scatter(SortSrc s, long long N, int tile,
                                                               int shift, const uint32_t* cnt,
                                                               uint32_t* key_out,
                                                               uint32_t* pos_out) {
  __shared__ uint32_t wh[kSortWarps][kRadix];
  __shared__ uint32_t base[kRadix], before[kRadix], sums[kRadix / 32];
  const int t = threadIdx.x, d = t & (kRadix - 1);
  // every tile's counts: the total of each digit, and that of the tiles before
  constexpr int kQ = kSortThreads / kRadix;
  uint32_t total = 0, prior = 0;
  for (int x = t / kRadix; x < (int)gridDim.x; x += kQ) {
    const uint32_t c = cnt[x * kRadix + d];
    total += c;
    if (x < (int)blockIdx.x) prior += c;
  }
  wh[t / kRadix][d] = total;
  wh[kQ + t / kRadix][d] = prior;
  __syncthreads();
  if (t < kRadix) {
    uint32_t a = 0, b = 0;
    for (int q = 0; q < kQ; ++q) {
      a += wh[q][t];
      b += wh[kQ + q][t];
    }
    base[t] = a;
    before[t] = b;
  }
  __syncthreads();
  scan_digits(base, sums);
  if (t < kRadix) base[t] += before[t];
  __syncthreads();
  const long long a = (long long)blockIdx.x * tile, e = a + tile < N ? a + tile : N;
  scatter_range(s, a, e, shift, wh, base, key_out, pos_out);
}

// The whole sort of a short list by one block, all passes in one launch.
__global__ void __launch_bounds__(kSortThreads) k_sort_one(SortSrc s, long long N, int passes,
                                                           uint32_t* k0, uint32_t* p0,
                                                           uint32_t* k1, uint32_t* p1,
                                                           int* header) {
  if (threadIdx.x < 4) header[threadIdx.x] = 0;
  __shared__ uint32_t wh[kSortWarps][kRadix];
  __shared__ uint32_t base[kRadix], sums[kRadix / 32];
  for (int p = 0; p < passes; ++p) {
    if (threadIdx.x < kRadix) base[threadIdx.x] = 0;
    __syncthreads();
    count_digits(s, 0, N, p * kRadixBits, base);
    __syncthreads();
    scan_digits(base, sums);
    uint32_t *ko = p & 1 ? k1 : k0, *po = p & 1 ? p1 : p0;
    scatter_range(s, 0, N, p * kRadixBits, wh, base, ko, po);
    s.ids = nullptr;
    s.key = ko;
    s.pos = po;
  }
}

// ------------------------------------------------------------------ sums
struct SumJob {
  const uint32_t *key, *pos;  // sorted
  long long N;
  int D, V, U, gl;            // U vectors a row, 2^gl threads a group
  int chunk;                  // sorted tokens per chunk
  long long chunks;
  float scale;
  int accumulate;
  float* part;                // [chunks][2][D]: a run that came in, one that goes on
};

template <typename T, int VB>
__device__ __forceinline__ void finish_row(const SumJob& j, const float* acc, T* dst) {
  Vec<T, VB> o;
  if (j.accumulate) {
    o.load(dst);
#pragma unroll
    for (int e = 0; e < Vec<T, VB>::n; ++e) o.set(e, fmaf(j.scale, acc[e], o.get(e)));
  } else {
#pragma unroll
    for (int e = 0; e < Vec<T, VB>::n; ++e) o.set(e, j.scale * acc[e]);
  }
  o.store(dst);
}

// Whether `row` is among the sorted keys.
__device__ __forceinline__ bool has_key(const uint32_t* key, long long N, uint32_t row) {
  long long lo = 0, hi = N;
  while (lo < hi) {
    const long long mid = (lo + hi) >> 1;
    if (key[mid] < row)
      lo = mid + 1;
    else
      hi = mid;
  }
  return lo < N && key[lo] == row;
}

constexpr int kSumAhead = 8;  // rows in flight per thread

// Blocks [0, sum_blocks): one group of threads per (chunk, columns).  Blocks
// from sum_blocks on write the rows that no token names as zero, 32 rows a
// warp.
template <typename T, int VB>
__global__ void __launch_bounds__(256) k_embed_sum(SumJob j, const T* dout, T* dtable,
                                                   unsigned sum_blocks) {
  constexpr int n = Vec<T, VB>::n;
  if (blockIdx.x >= sum_blocks) {
    const int lane = threadIdx.x & 31;
    const long long r0 =
        ((long long)(blockIdx.x - sum_blocks) * 8 + (threadIdx.x >> 5)) * 32;
    const bool empty = r0 + lane < j.V && !has_key(j.key, j.N, (uint32_t)(r0 + lane));
    unsigned rows = __ballot_sync(0xffffffffu, empty);
    Vec<T, VB> z;
#pragma unroll
    for (int e = 0; e < n; ++e) z.set(e, 0.0f);
    while (rows) {
      const int r = __ffs(rows) - 1;
      rows &= rows - 1;
      T* dst = dtable + (size_t)(r0 + r) * j.D;
      for (int u = lane; u < j.U; u += 32) z.store(dst + (size_t)u * n);
    }
    return;
  }
  const int g = 1 << j.gl;
  const long long groups = (long long)blockIdx.x * (256 >> j.gl) + (threadIdx.x >> j.gl);
  const int colblocks = (j.U + g - 1) >> j.gl;
  const long long c = groups / colblocks;
  const int u = (int)(groups % colblocks) * g + (threadIdx.x & (g - 1));
  if (c >= j.chunks || u >= j.U) return;
  const long long a = c * j.chunk, e = a + j.chunk < j.N ? a + j.chunk : j.N;
  const uint32_t V = (uint32_t)j.V;
  const bool came = a > 0 && j.key[a - 1] == j.key[a];    // the first run started earlier
  const bool goes = e < j.N && j.key[e - 1] == j.key[e];  // the last run goes on
  float acc[n];
#pragma unroll
  for (int x = 0; x < n; ++x) acc[x] = 0.0f;
  uint32_t cur = j.key[a];
  bool first = true;
  auto flush = [&](bool last) {
    if (cur < V) {
      float* p = nullptr;
      if (first && came)
        p = j.part + ((size_t)c * 2) * j.D;
      else if (last && goes)
        p = j.part + ((size_t)c * 2 + 1) * j.D;
      if (p) {
#pragma unroll
        for (int x = 0; x < n; ++x) p[(size_t)u * n + x] = acc[x];
      } else {
        finish_row<T, VB>(j, acc, dtable + (size_t)cur * j.D + (size_t)u * n);
      }
    }
    first = false;
#pragma unroll
    for (int x = 0; x < n; ++x) acc[x] = 0.0f;
  };
  for (long long i = a; i < e; i += kSumAhead) {
    uint32_t k[kSumAhead];
    Vec<T, VB> v[kSumAhead];
#pragma unroll
    for (int x = 0; x < kSumAhead; ++x) {
      k[x] = i + x < e ? j.key[i + x] : V;
      if (k[x] < V) v[x].load(dout + (size_t)j.pos[i + x] * j.D + (size_t)u * n);
    }
#pragma unroll
    for (int x = 0; x < kSumAhead; ++x) {
      if (i + x >= e) break;
      if (k[x] != cur) {
        flush(false);
        cur = k[x];
      }
      if (cur < V) {
#pragma unroll
        for (int y = 0; y < n; ++y) acc[y] += v[x].get(y);
      }
    }
  }
  flush(true);
}

// Joins the runs that cross chunks.  A block looks at one chunk; if a run
// starts in it and goes on, its groups of threads add the later chunks'
// partial rows (each group a contiguous share of them, in order), and the
// groups' sums are added in order.
constexpr int kJoinThreads = 512;
template <typename T, int VB>
__global__ void __launch_bounds__(kJoinThreads) k_embed_join(SumJob j, T* dtable) {
  constexpr int n = Vec<T, VB>::n;
  __shared__ float sh[kJoinThreads * n];
  const long long c = blockIdx.x;
  const long long a = c * j.chunk, e = a + j.chunk;
  if (e >= j.N) return;
  const uint32_t key = j.key[e - 1];
  if (key != j.key[e] || key >= (uint32_t)j.V) return;
  // the run came into this chunk from an earlier one, which joins it
  if (a > 0 && j.key[a] == key && j.key[a - 1] == key) return;
  // the run's last token, then the last chunk that holds some of it
  long long lo = e, hi = j.N;  // key[lo] == key, key[hi] != key
  while (hi - lo > 1) {
    const long long mid = (lo + hi) >> 1;
    if (j.key[mid] == key)
      lo = mid;
    else
      hi = mid;
  }
  const long long more = lo / j.chunk - c;  // chunks c+1 .. c+more, in their slot 0
  const int g = 1 << j.gl, lane = threadIdx.x & (g - 1), grp = threadIdx.x >> j.gl;
  const int groups = kJoinThreads >> j.gl;
  const long long share = (more + groups - 1) / groups;
  const long long b0 = grp * share < more ? grp * share : more;
  const long long b1 = b0 + share < more ? b0 + share : more;
  for (int u0 = 0; u0 < j.U; u0 += g) {
    const int u = u0 + lane;
    const bool on = u < j.U;
    float acc[n];
#pragma unroll
    for (int x = 0; x < n; ++x)
      acc[x] = on && grp == 0 ? j.part[((size_t)c * 2 + 1) * j.D + (size_t)u * n + x] : 0.0f;
    if (on) {
#pragma unroll 4
      for (long long b = b0; b < b1; ++b) {
        const float* p = j.part + ((size_t)(c + 1 + b) * 2) * j.D + (size_t)u * n;
#pragma unroll
        for (int x = 0; x < n; ++x) acc[x] += p[x];
      }
    }
#pragma unroll
    for (int x = 0; x < n; ++x) sh[x * kJoinThreads + threadIdx.x] = acc[x];
    __syncthreads();
    if (grp == 0 && on) {
      for (int q = 1; q < groups; ++q)
#pragma unroll
        for (int x = 0; x < n; ++x) acc[x] += sh[x * kJoinThreads + (q << j.gl) + lane];
      finish_row<T, VB>(j, acc, dtable + (size_t)key * j.D + (size_t)u * n);
    }
    __syncthreads();
  }
}

// ------------------------------------------------------------------ host
bool sizes_ok(long long N, int D, int V, slim_dtype dtype, slim_index itype) {
  if (N < 0 || N >= (1LL << 31) || D < 1 || V < 1) return false;
  if (dtype != SLIM_F32 && dtype != SLIM_BF16) return false;
  if (itype != SLIM_I32 && itype != SLIM_I64) return false;
  // element counts stay far inside 64 bits
  return (long long)D <= (1LL << 42) / (N > 0 ? N : 1) && (long long)D <= (1LL << 42) / V;
}

bool aligned(const void* p, size_t to) {
  return p != nullptr && (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0;
}

constexpr long long kOneBlock = 4096;  // longest list one block sorts alone

struct Plan {
  int passes, tiles, tile;
  int chunk;
  long long chunks;
};
Plan plan(long long N, int V) {
  Plan p;
  int bits = 1;
  while ((1LL << bits) < (long long)V + 1) ++bits;
  p.passes = (bits + kRadixBits - 1) / kRadixBits;
  const long long want = (N + 2047) / 2048;
  p.tiles = (int)(want < kSMs ? (want > 0 ? want : 1) : kSMs);
  p.tile = (int)((N + p.tiles - 1) / p.tiles);
  long long k = (N + 1023) / 1024;
  p.chunk = (int)(k < 16 ? 16 : k > 64 ? 64 : k);
  p.chunks = (N + p.chunk - 1) / p.chunk;
  return p;
}

struct Ws {
  int* header;  // the call's error word (no kernel here waits)
  uint32_t *k0, *p0, *k1, *p1, *cnt;
  float* part;
};
Ws carve(Carver& cv, long long N, int D, const Plan& p) {
  Ws w;
  w.header = cv.take<int>(4);
  w.k0 = cv.take<uint32_t>(N);
  w.p0 = cv.take<uint32_t>(N);
  w.k1 = cv.take<uint32_t>(p.passes > 1 ? N : 0);
  w.p1 = cv.take<uint32_t>(p.passes > 1 ? N : 0);
  w.cnt = cv.take<uint32_t>((size_t)p.tiles * kRadix);
  w.part = cv.take<float>((size_t)p.chunks * 2 * D);
  return w;
}

bool launched() { return cudaGetLastError() == cudaSuccess; }

template <typename T, int VB>
slim_status fwd(const void* ids, slim_index itype, const void* table, long long N, int D, int V,
                float scale, void* out, cudaStream_t s) {
  const int U = D / Vec<T, VB>::n, gl = group_log2(U, kFwdItems);
  const long long blocks = (N + (256 >> gl) - 1) / (256 >> gl);
  prof::Scope ps(prof::K_EMBED_FWD, s, 0.0, 2.0 * N * D * sizeof(T));
  k_embed_fwd<T, VB><<<(unsigned)blocks, 256, 0, s>>>(ids, itype == SLIM_I64, (const T*)table, N,
                                                      D, V, U, gl, scale, (T*)out);
  return launched() ? SLIM_OK : SLIM_ERR_CUDA;
}

slim_status sort(const void* ids, slim_index itype, long long N, int V, const Plan& p, const Ws& w,
                 cudaStream_t s, const uint32_t** key, const uint32_t** pos) {
  SortSrc src{ids, itype == SLIM_I64, V, nullptr, nullptr};
  if (N <= kOneBlock) {
    prof::Scope ps(prof::K_EMBED_SORT, s);
    k_sort_one<<<1, kSortThreads, 0, s>>>(src, N, p.passes, w.k0, w.p0, w.k1, w.p1,
                                       w.header);
    if (!launched()) return SLIM_ERR_CUDA;
  } else {
    for (int i = 0; i < p.passes; ++i) {
      {
        prof::Scope ps(prof::K_EMBED_SORT, s);
        k_sort_count<<<p.tiles, kSortThreads, 0, s>>>(src, N, p.tile, i * kRadixBits, w.cnt,
                                                     w.header);
        if (!launched()) return SLIM_ERR_CUDA;
      }
      uint32_t *ko = i & 1 ? w.k1 : w.k0, *po = i & 1 ? w.p1 : w.p0;
      prof::Scope ps(prof::K_EMBED_SORT, s);
      k_sort_scatter<<<p.tiles, kSortThreads, 0, s>>>(src, N, p.tile, i * kRadixBits, w.cnt, ko,
                                                      po);
      if (!launched()) return SLIM_ERR_CUDA;
      src = SortSrc{nullptr, 0, V, ko, po};
    }
  }
  *key = p.passes & 1 ? w.k0 : w.k1;
  *pos = p.passes & 1 ? w.p0 : w.p1;
  return SLIM_OK;
}

template <typename T, int VB>
slim_status bwd(const void* ids, slim_index itype, const void* dout, long long N, int D, int V,
                float scale, int accumulate, void* dtable, void* ws, cudaStream_t s) {
  const Plan p = plan(N, V);
  Carver cv(ws);
  const Ws w = carve(cv, N, D, p);
  SumJob j{};
  const slim_status st = sort(ids, itype, N, V, p, w, s, &j.key, &j.pos);
  if (st != SLIM_OK) return st;
  j.N = N;
  j.D = D;
  j.V = V;
  j.U = D / Vec<T, VB>::n;
  j.gl = group_log2(j.U, 1);
  j.chunk = p.chunk;
  j.chunks = p.chunks;
  j.scale = scale;
  j.accumulate = accumulate;
  j.part = w.part;
  const long long colblocks = (j.U + (1 << j.gl) - 1) >> j.gl;
  const long long per = 256 >> j.gl;
  const long long sum_blocks = (p.chunks * colblocks + per - 1) / per;
  const long long zero_blocks = accumulate ? 0 : ((long long)V + 255) / 256;
  if (sum_blocks + zero_blocks >= (1LL << 31)) return SLIM_ERR_UNSUPPORTED;
  {
    prof::Scope ps(prof::K_EMBED_SUM, s, 0.0, ((double)N + V) * D * sizeof(T));
    k_embed_sum<T, VB><<<(unsigned)(sum_blocks + zero_blocks), 256, 0, s>>>(
        j, (const T*)dout, (T*)dtable, (unsigned)sum_blocks);
    if (!launched()) return SLIM_ERR_CUDA;
  }
  if (p.chunks > 1) {
    prof::Scope ps(prof::K_EMBED_SUM, s);
    k_embed_join<T, VB><<<(unsigned)(p.chunks - 1), kJoinThreads, 0, s>>>(j, (T*)dtable);
    if (!launched()) return SLIM_ERR_CUDA;
  }
  return SLIM_OK;
}

#define EMBED_DISPATCH(FN, ...)                                \
  do {                                                         \
    if (dtype == SLIM_F32) {                                   \
      switch (vec_bytes(D, 4)) {                               \
        case 16: return FN<float, 16>(__VA_ARGS__);            \
        case 8: return FN<float, 8>(__VA_ARGS__);              \
        default: return FN<float, 4>(__VA_ARGS__);             \
      }                                                        \
    }                                                          \
    switch (vec_bytes(D, 2)) {                                 \
      case 16: return FN<__nv_bfloat16, 16>(__VA_ARGS__);      \
      case 8: return FN<__nv_bfloat16, 8>(__VA_ARGS__);        \
      case 4: return FN<__nv_bfloat16, 4>(__VA_ARGS__);        \
      default: return FN<__nv_bfloat16, 2>(__VA_ARGS__);       \
    }                                                          \
  } while (0)

}  // namespace
}  // namespace lm
}  // namespace slim

extern "C" slim_status slim_embed_fwd(const void* ids, slim_index itype, const void* table,
                                      long long N, int D, int V, slim_dtype dtype, float scale,
                                      void* out, void* stream) {
  using namespace slim::lm;
  if (!sizes_ok(N, D, V, dtype, itype)) return SLIM_ERR_INVALID_ARG;
  if (!aligned(table, 16)) return SLIM_ERR_INVALID_ARG;
  if (N == 0) return SLIM_OK;
  if (!aligned(ids, itype == SLIM_I64 ? 8 : 4) || !aligned(out, 16)) return SLIM_ERR_INVALID_ARG;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  EMBED_DISPATCH(fwd, ids, itype, table, N, D, V, scale, out, s);
}

extern "C" slim_status slim_embed_bwd_workspace_size(long long N, int D, int V, slim_dtype dtype,
                                                     size_t* bytes) {
  using namespace slim::lm;
  if (!bytes || !sizes_ok(N, D, V, dtype, SLIM_I64)) return SLIM_ERR_INVALID_ARG;
  slim::Carver cv(nullptr);
  carve(cv, N, D, plan(N, V));
  *bytes = cv.bytes();
  return SLIM_OK;
}

extern "C" slim_status slim_embed_bwd(const void* ids, slim_index itype, const void* dout,
                                      long long N, int D, int V, slim_dtype dtype, float scale,
                                      int accumulate, void* dtable, void* workspace,
                                      size_t workspace_bytes, void* stream) {
  using namespace slim::lm;
  if (!sizes_ok(N, D, V, dtype, itype) || (accumulate & ~1)) return SLIM_ERR_INVALID_ARG;
  if (!aligned(dtable, 16)) return SLIM_ERR_INVALID_ARG;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (N == 0) {
    const size_t n = (size_t)V * D * (dtype == SLIM_F32 ? 4 : 2);
    if (!accumulate && cudaMemsetAsync(dtable, 0, n, s) != cudaSuccess) return SLIM_ERR_CUDA;
    return SLIM_OK;
  }
  if (!aligned(ids, itype == SLIM_I64 ? 8 : 4) || !aligned(dout, 16)) return SLIM_ERR_INVALID_ARG;
  size_t need = 0;
  slim_embed_bwd_workspace_size(N, D, V, dtype, &need);
  if (workspace == nullptr || workspace_bytes < need) return SLIM_ERR_WORKSPACE;
  if (!aligned(workspace, 256)) return SLIM_ERR_INVALID_ARG;
  EMBED_DISPATCH(bwd, ids, itype, dout, N, D, V, scale, accumulate, dtable, workspace, s);
}
