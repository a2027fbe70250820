// Embedding lookup with scaling, and the gradient of its table by sorted
// tokens.  Contract: include/slim_lm.h.
//
// Forward: out_i = scale * table[ids_i].  One read and one write per element
// and no reuse, so HBM bounds it; a group of threads copies a row in the widest
// vectors its width allows.  65536 rows of 768 fp32 from a table of 50021: 49 us,
// 5.9 TB/s of rows read and written.
//
// Gradient: dtable_v = scale * sum_{i: ids_i = v} dout_i.  The tokens are
// sorted by id with a stable radix sort (8-bit digits, only the bits that V
// needs), which turns the scatter into sums over runs of equal ids in order of
// position.  The sorted list is cut into chunks of equal length, whatever the
// ids: a frequent token's run is spread over many chunks and a rare token's
// shares one, so the work is even.  A run inside one chunk is summed in
// registers and written once; a run that crosses chunks leaves a partial row
// per chunk, which a last kernel adds in order.  Every sum has a fixed order.
// 65536 x 768 fp32 tokens on 32768 rows: 75 us, of which the sums 54 (5.6 TB/s,
// HBM) and the sort about 15 (four launches of a few us each, latency); 32768 x
// 512 bf16 on 256 rows 25 us, where the chain of four launches bounds it.
#include <stdint.h>

#include "../../include/slim_lm.h"
#include "common.cuh"
#include "launch.h"
#include "profiler.h"
#include "tc_common.cuh"

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
  // What is read or written once gives way in L2 to what is not: the rows of a
  // table (lookup 50.8 -> 48.6 us) and the partial rows (gradient 79 -> 75 us; at
  // 65536 x 768 fp32, tables of 50021 and 32768 rows).
  __device__ __forceinline__ void load_once(const T* p) {
    raw = __ldcs(reinterpret_cast<const typename Raw<VB>::type*>(p));
  }
  __device__ __forceinline__ void store_once(T* p) const {
    __stcs(reinterpret_cast<typename Raw<VB>::type*>(p), raw);
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
      v[j].store_once(dst + (size_t)(u0 + j * g) * n);
    }
  }
}

// ------------------------------------------------------------------ sort
// Keys are ids.  The first pass reads the caller's ids and drops those outside
// the table, so the key takes only the bits that V - 1 has; the number that
// remains stays on the device (`count`).
constexpr int kRadixBits = 8, kRadix = 1 << kRadixBits;
constexpr int kSortThreads = 1024, kSortWarps = kSortThreads / 32;
constexpr uint32_t kNoKey = 0xffffffffu;

struct SortSrc {
  const void* ids;  // first pass: the caller's ids; later passes: null
  int i64, V;
  const uint32_t *key, *pos;
  const int* count;  // of the later passes' items
  __device__ __forceinline__ long long items(long long N) const {
    return ids ? N : (long long)*count;
  }
  __device__ __forceinline__ uint32_t key_at(long long i) const {
    if (!ids) return key[i];
    const long long id = load_id(ids, i64, i);
    return id >= 0 && id < V ? (uint32_t)id : kNoKey;
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
    const uint32_t key = i < e ? s.key_at(i) : kNoKey;
    const uint32_t d = key == kNoKey ? kRadix : (key >> shift) & (kRadix - 1);
    const unsigned peers = __match_any_sync(0xffffffffu, d);
    if (d < kRadix && (peers & ((1u << (threadIdx.x & 31)) - 1)) == 0)
      atomicAdd(&hist[d], (uint32_t)__popc(peers));
  }
}

// Exclusive prefix sum of x[kRadix] (shared memory) in place, by all threads;
// returns the total to thread kRadix - 1.
__device__ uint32_t scan_digits(uint32_t* x, uint32_t* warp_sum) {
  const int t = threadIdx.x, lane = t & 31, w = t >> 5;
  uint32_t v = 0, inc = 0, before = 0;
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
    for (int i = 0; i < w; ++i) before += warp_sum[i];
    x[t] = before + inc - v;
  }
  __syncthreads();
  return before + inc;
}

// Scatters [a, e) stably by digit; base[d] is where this range's first item
// with digit d goes, and is advanced.
__device__ void scatter_range(const SortSrc& s, long long a, long long e, int shift,
                              uint32_t (*wh)[kRadix], uint32_t* base, uint32_t* key_out,
                              uint32_t* pos_out) {
  const int t = threadIdx.x, lane = t & 31, w = t >> 5;
  for (long long i0 = a; i0 < e; i0 += kSortThreads) {
    for (int x = t; x < kSortWarps * kRadix; x += kSortThreads) (&wh[0][0])[x] = 0;
    const long long i = i0 + t;
    uint32_t key = kNoKey, pos = 0, d = kRadix;
    if (i < e) {
      key = s.key_at(i);
      pos = s.pos_at(i);
      if (key != kNoKey) d = (key >> shift) & (kRadix - 1);
    }
    __syncthreads();
    const unsigned peers = __match_any_sync(0xffffffffu, d);
    const uint32_t rank = __popc(peers & ((1u << lane) - 1));
    if (d < kRadix && rank == 0) wh[w][d] = __popc(peers);
    __syncthreads();
    if (t < kRadix) {  // counts of the warps -> first place of each warp's items
      uint32_t run = base[t];
#pragma unroll 8
      for (int x = 0; x < kSortWarps; ++x) {
        const uint32_t c = wh[x][t];
        wh[x][t] = run;
        run += c;
      }
      base[t] = run;
    }
    __syncthreads();
    if (d < kRadix) {
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
  if (threadIdx.x < kRadix) hist[threadIdx.x] = 0;
  tc::grid_dependency_wait();
  if (s.ids && blockIdx.x == 0 && threadIdx.x < 4) header[threadIdx.x] = 0;
  __syncthreads();
  const long long n = s.items(N);
  const long long a = (long long)blockIdx.x * tile, e = a + tile < n ? a + tile : n;
  count_digits(s, a, e, shift, hist);
  __syncthreads();
  if (threadIdx.x < kRadix) cnt[blockIdx.x * kRadix + threadIdx.x] = hist[threadIdx.x];
}

__global__ void __launch_bounds__(kSortThreads) k_sort_scatter(SortSrc s, long long N, int tile,
                                                               int shift, const uint32_t* cnt,
                                                               uint32_t* key_out,
                                                               uint32_t* pos_out, int* count) {
  __shared__ uint32_t wh[kSortWarps][kRadix];
  __shared__ uint32_t base[kRadix], before[kRadix], sums[kRadix / 32];
  const int t = threadIdx.x, d = t & (kRadix - 1);
  tc::grid_dependency_wait();
  // every tile's counts: the total of each digit, and that of the tiles before
  constexpr int kQ = kSortThreads / kRadix;
  uint32_t total = 0, prior = 0;
#pragma unroll 8
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
  const uint32_t all = scan_digits(base, sums);
  if (s.ids && blockIdx.x == 0 && t == kRadix - 1) *count = (int)all;
  if (t < kRadix) base[t] += before[t];
  __syncthreads();
  const long long n = s.items(N);
  const long long a = (long long)blockIdx.x * tile, e = a + tile < n ? a + tile : n;
  scatter_range(s, a, e, shift, wh, base, key_out, pos_out);
}

// The whole sort of a short list by one block, all passes in one launch.
__global__ void __launch_bounds__(kSortThreads) k_sort_one(SortSrc s, long long N, int passes,
                                                           uint32_t* k0, uint32_t* p0,
                                                           uint32_t* k1, uint32_t* p1, int* count,
                                                           int* header) {
  __shared__ uint32_t wh[kSortWarps][kRadix];
  __shared__ uint32_t base[kRadix], sums[kRadix / 32];
  __shared__ uint32_t left;
  tc::grid_dependency_wait();  // (of nothing) lets the next kernel set up meanwhile
  if (threadIdx.x < 4) header[threadIdx.x] = 0;
  for (int p = 0; p < passes; ++p) {
    if (threadIdx.x < kRadix) base[threadIdx.x] = 0;
    __syncthreads();
    const long long n = p == 0 ? N : left;
    count_digits(s, 0, n, p * kRadixBits, base);
    __syncthreads();
    const uint32_t all = scan_digits(base, sums);
    if (threadIdx.x == kRadix - 1) {
      left = all;
      *count = (int)all;
    }
    uint32_t *ko = p & 1 ? k1 : k0, *po = p & 1 ? p1 : p0;
    scatter_range(s, 0, n, p * kRadixBits, wh, base, ko, po);
    s.ids = nullptr;
    s.key = ko;
    s.pos = po;
    __syncthreads();
  }
}

// ------------------------------------------------------------------ sums
constexpr int kMaxChunk = 64;
struct SumJob {
  const uint32_t *key, *pos;  // sorted
  const int* count;           // of them
  int D, V, U, gl;            // U vectors a row, 2^gl threads a group
  int colblocks;              // groups that share a chunk's columns
  int chunk;                  // sorted tokens per chunk
  long long chunks;
  float scale;
  int accumulate;
  float* part;                // [chunks][2][ld]: a run that came in, one that goes on
  long long ld;               // a multiple of 4
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
  o.store_once(dst);
}

// n floats of a partial row.
template <int n>
__device__ __forceinline__ void part_store(float* p, const float* f) {
  if constexpr (n % 4 == 0) {
#pragma unroll
    for (int i = 0; i < n; i += 4)
      *reinterpret_cast<float4*>(p + i) = make_float4(f[i], f[i + 1], f[i + 2], f[i + 3]);
  } else {
#pragma unroll
    for (int i = 0; i < n; ++i) p[i] = f[i];
  }
}
template <int n>
__device__ __forceinline__ void part_add(const float* p, float* f) {
  if constexpr (n % 4 == 0) {
#pragma unroll
    for (int i = 0; i < n; i += 4) {
      const float4 x = *reinterpret_cast<const float4*>(p + i);
      f[i] += x.x;
      f[i + 1] += x.y;
      f[i + 2] += x.z;
      f[i + 3] += x.w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < n; ++i) f[i] += p[i];
  }
}

// Whether `row` is among the sorted keys.
__device__ __forceinline__ bool has_key(const uint32_t* key, int N, uint32_t row) {
  int lo = 0, hi = N;
  while (lo < hi) {
    const int mid = (int)(((unsigned)lo + (unsigned)hi) >> 1);
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
__global__ void __launch_bounds__(256, 4) k_embed_sum(SumJob j, const T* dout, T* dtable,
                                                   unsigned sum_blocks) {
  constexpr int n = Vec<T, VB>::n;
  // a chunk's tokens, fetched once: the rows' loads then wait for no index
  __shared__ uint32_t sk[256], sp[256];
  tc::grid_dependency_wait();
  const int N = *j.count;
  if (blockIdx.x >= sum_blocks) {
    const int lane = threadIdx.x & 31;
    const long long r0 =
        ((long long)(blockIdx.x - sum_blocks) * 8 + (threadIdx.x >> 5)) * 32;
    const bool empty = r0 + lane < j.V && !has_key(j.key, N, (uint32_t)(r0 + lane));
    unsigned rows = __ballot_sync(0xffffffffu, empty);
    Vec<T, VB> z;
#pragma unroll
    for (int e = 0; e < n; ++e) z.set(e, 0.0f);
    while (rows) {
      const int r = __ffs(rows) - 1;
      rows &= rows - 1;
      T* dst = dtable + (size_t)(r0 + r) * j.D;
      for (int u = lane; u < j.U; u += 32) z.store_once(dst + (size_t)u * n);
    }
    return;
  }
  const int g = 1 << j.gl, lane = threadIdx.x & (g - 1);
  const long long group = (long long)blockIdx.x * (256 >> j.gl) + (threadIdx.x >> j.gl);
  const long long c = group / j.colblocks;
  const int u = (int)(group - c * j.colblocks) * g + lane;
  const long long a = c * j.chunk;
  const int len = c < j.chunks && a < N ? (int)(a + j.chunk < N ? j.chunk : N - a) : 0;
  // (a group keeps them at its own threads' places; narrower groups than a chunk
  // read them where they are)
  const bool staged = g >= j.chunk;
  if (staged && lane < len) {
    sk[threadIdx.x] = j.key[a + lane];
    sp[threadIdx.x] = j.pos[a + lane];
  }
  __syncthreads();
  if (len == 0 || u >= j.U) return;
  const uint32_t* key = staged ? sk + (threadIdx.x - lane) : j.key + a;
  const uint32_t* pos = staged ? sp + (threadIdx.x - lane) : j.pos + a;
  uint32_t cur = key[0];
  const bool came = a > 0 && j.key[a - 1] == cur;                  // its run started earlier
  const bool goes = a + len < N && j.key[a + len] == key[len - 1];  // the last run goes on
  float acc[n];
#pragma unroll
  for (int x = 0; x < n; ++x) acc[x] = 0.0f;
  bool first = true;
  float* part = j.part + (size_t)c * 2 * j.ld + (size_t)u * n;
  const T* rows = dout + (size_t)u * n;
  auto flush = [&](bool last) {
    if (first && came)
      part_store<n>(part, acc);
    else if (last && goes)
      part_store<n>(part + j.ld, acc);
    else
      finish_row<T, VB>(j, acc, dtable + (size_t)cur * j.D + (size_t)u * n);
    first = false;
#pragma unroll
    for (int x = 0; x < n; ++x) acc[x] = 0.0f;
  };
  for (int i = 0; i < len; i += kSumAhead) {
    Vec<T, VB> v[kSumAhead];
#pragma unroll
    for (int x = 0; x < kSumAhead; ++x)
      if (i + x < len) v[x].load_once(rows + (size_t)pos[i + x] * j.D);
#pragma unroll
    for (int x = 0; x < kSumAhead; ++x) {
      if (i + x >= len) break;
      const uint32_t k = key[i + x];
      if (k != cur) {
        flush(false);
        cur = k;
      }
#pragma unroll
      for (int y = 0; y < n; ++y) acc[y] += v[x].get(y);
    }
  }
  flush(true);
}

// Joins the runs that cross chunks.  A block looks at one chunk; if a run
// starts in it and goes on, it adds the later chunks' partial rows in order.
// Most such runs reach one chunk further, and all threads go side by side along
// the columns.  A long run (a frequent token) is cut into 16 shares, a warp each,
// whose sums are added in order; a warp goes along 64 vectors of the columns at a
// time.
constexpr int kJoinThreads = 512, kJoinGroups = kJoinThreads / 32, kJoinCols = 2;
template <typename T, int VB>
__global__ void __launch_bounds__(kJoinThreads) k_embed_join(SumJob j, T* dtable) {
  constexpr int n = Vec<T, VB>::n;
  __shared__ float sh[kJoinGroups][kJoinCols][n][32];
  tc::grid_dependency_wait();
  const long long c = blockIdx.x;
  const long long a = c * j.chunk, e = a + j.chunk;  // inside the list as the host knows it
  // (read beside the count, which says whether they mean anything)
  const uint32_t key = j.key[e - 1], next = j.key[e], head = j.key[a],
                 before = a > 0 ? j.key[a - 1] : kNoKey;
  const int N = *j.count;
  if (e >= N || key != next) return;
  // the run came into this chunk from an earlier one, which joins it
  if (head == key && before == key) return;
  const int lane = threadIdx.x & 31, grp = threadIdx.x >> 5;
  // chunks c+1 .. c+more begin inside the run (and are in their slot 0)
  int more = 0;
  for (;;) {
    const long long at = e + (long long)(more + (int)threadIdx.x) * j.chunk;
    const int in = __syncthreads_count(at < N && j.key[at] == key);
    more += in;  // a run is contiguous: the threads in it are the first ones
    if (in < kJoinThreads) break;
  }
  const float* first = j.part + ((size_t)c * 2 + 1) * j.ld;
  const float* rest = j.part + (size_t)(c + 1) * 2 * j.ld;
  T* out = dtable + (size_t)key * j.D;
  if (more < kJoinGroups) {
    for (int u = threadIdx.x; u < j.U; u += kJoinThreads) {
      float acc[n];
#pragma unroll
      for (int x = 0; x < n; ++x) acc[x] = 0.0f;
      part_add<n>(first + (size_t)u * n, acc);
#pragma unroll 4
      for (int b = 0; b < more; ++b) part_add<n>(rest + (size_t)b * 2 * j.ld + (size_t)u * n, acc);
      finish_row<T, VB>(j, acc, out + (size_t)u * n);
    }
    return;
  }
  const int share = (more + kJoinGroups - 1) / kJoinGroups;
  const int b0 = min(grp * share, more), b1 = min(b0 + share, more);
  for (int u0 = 0; u0 < j.U; u0 += 32 * kJoinCols) {
    float acc[kJoinCols][n];
#pragma unroll
    for (int k = 0; k < kJoinCols; ++k)
#pragma unroll
      for (int x = 0; x < n; ++x) acc[k][x] = 0.0f;
    auto add = [&](const float* row) {
#pragma unroll
      for (int k = 0; k < kJoinCols; ++k) {
        const int u = u0 + 32 * k + lane;
        if (u < j.U) part_add<n>(row + (size_t)u * n, acc[k]);
      }
    };
    if (grp == 0) add(first);
#pragma unroll 4
    for (int b = b0; b < b1; ++b) add(rest + (size_t)b * 2 * j.ld);
#pragma unroll
    for (int k = 0; k < kJoinCols; ++k)
#pragma unroll
      for (int x = 0; x < n; ++x) sh[grp][k][x][lane] = acc[k][x];
    __syncthreads();
    if (grp < kJoinCols) {  // one warp per block of 32 vectors
      const int u = u0 + 32 * grp + lane;
      float sum[n];
#pragma unroll
      for (int x = 0; x < n; ++x) sum[x] = sh[0][grp][x][lane];
      for (int q = 1; q < kJoinGroups; ++q)
#pragma unroll
        for (int x = 0; x < n; ++x) sum[x] += sh[q][grp][x][lane];
      if (u < j.U) finish_row<T, VB>(j, sum, out + (size_t)u * n);
    }
    __syncthreads();
  }
}

// ------------------------------------------------------------------ host
bool sizes_ok(long long N, int D, int V, slim_dtype dtype, slim_index itype) {
  if (N < 0 || N >= (1LL << 31) || D < 1 || V < 1) return false;
  if (D > (1 << 30)) return false;  // a row's 32-bit column indices step past its end
  if (dtype != SLIM_F32 && dtype != SLIM_BF16) return false;
  if (itype != SLIM_I32 && itype != SLIM_I64) return false;
  // element counts stay far inside 64 bits
  return (long long)D <= (1LL << 42) / (N > 0 ? N : 1) && (long long)D <= (1LL << 42) / V;
}

bool aligned(const void* p, size_t to) {
  return p != nullptr && (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0;
}

// Longest list that one block sorts alone: 9 us for 1000 ids in two passes; at 4096
// ids four launches are 8 us faster.
constexpr long long kOneBlock = 1024;

struct Plan {
  int passes, tiles, tile;
  int chunk;
  long long chunks;
};
Plan plan(long long N, int V) {
  Plan p;
  int bits = 1;
  while ((1LL << bits) < (long long)V) ++bits;
  p.passes = (bits + kRadixBits - 1) / kRadixBits;
  const long long want = (N + kSortThreads - 1) / kSortThreads;  // one round of a block's threads
  p.tiles = (int)(want < kSMs ? (want > 0 ? want : 1) : kSMs);
  p.tile = (int)((N + p.tiles - 1) / p.tiles);
  // chunks short enough for some waves of blocks, long enough that their
  // partial rows (two each) stay small beside the rows they sum: 65536 x 768
  // fp32 in chunks of 16, 32, 64 takes 87, 82, 75 us
  const long long k = N / 1024;
  p.chunk = (int)(k < 16 ? 16 : k > kMaxChunk ? kMaxChunk : k);
  p.chunks = (N + p.chunk - 1) / p.chunk;
  return p;
}

struct Ws {
  int* header;  // the call's error word (no kernel here waits)
  uint32_t *k0, *p0, *k1, *p1, *cnt;
  int* count;
  float* part;
};
long long part_ld(int D) { return (D + 3) / 4 * 4; }
Ws carve(Carver& cv, long long N, int D, const Plan& p) {
  Ws w;
  w.header = cv.take<int>(4);
  w.k0 = cv.take<uint32_t>(N);
  w.p0 = cv.take<uint32_t>(N);
  w.k1 = cv.take<uint32_t>(p.passes > 1 ? N : 0);
  w.p1 = cv.take<uint32_t>(p.passes > 1 ? N : 0);
  w.cnt = cv.take<uint32_t>((size_t)p.tiles * kRadix);
  w.count = cv.take<int>(1);
  w.part = cv.take<float>((size_t)p.chunks * 2 * part_ld(D));
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
  SortSrc src{ids, itype == SLIM_I64, V, nullptr, nullptr, w.count};
  if (N <= kOneBlock) {
    prof::Scope ps(prof::K_EMBED_SORT, s);
    k_sort_one<<<1, kSortThreads, 0, s>>>(src, N, p.passes, w.k0, w.p0, w.k1, w.p1, w.count,
                                          w.header);
    if (!launched()) return SLIM_ERR_CUDA;
  } else {
    for (int i = 0; i < p.passes; ++i) {
      const int shift = i * kRadixBits;
      {
        prof::Scope ps(prof::K_EMBED_SORT, s);
        if (!launch_on<SortSrc, long long, int, int, uint32_t*, int*>(
                k_sort_count, p.tiles, kSortThreads, 0, 1, i > 0, s, src, N, p.tile, shift, w.cnt,
                w.header))
          return SLIM_ERR_CUDA;
      }
      uint32_t *ko = i & 1 ? w.k1 : w.k0, *po = i & 1 ? w.p1 : w.p0;
      prof::Scope ps(prof::K_EMBED_SORT, s);
      if (!launch_on<SortSrc, long long, int, int, const uint32_t*, uint32_t*, uint32_t*, int*>(
              k_sort_scatter, p.tiles, kSortThreads, 0, 1, true, s, src, N, p.tile, shift, w.cnt,
              ko, po, w.count))
        return SLIM_ERR_CUDA;
      src = SortSrc{nullptr, 0, V, ko, po, w.count};
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
  j.U = D / Vec<T, VB>::n;
  j.gl = group_log2(j.U, 1);
  j.colblocks = (j.U + (1 << j.gl) - 1) >> j.gl;
  const long long per = 256 >> j.gl;
  const long long sum_blocks = (p.chunks * j.colblocks + per - 1) / per;
  const long long zero_blocks = accumulate ? 0 : ((long long)V + 255) / 256;
  if (sum_blocks + zero_blocks >= (1LL << 31)) return SLIM_ERR_UNSUPPORTED;
  const slim_status st = sort(ids, itype, N, V, p, w, s, &j.key, &j.pos);
  if (st != SLIM_OK) return st;
  j.count = w.count;
  j.D = D;
  j.V = V;
  j.chunk = p.chunk;
  j.chunks = p.chunks;
  j.scale = scale;
  j.accumulate = accumulate;
  j.part = w.part;
  j.ld = part_ld(D);
  {
    prof::Scope ps(prof::K_EMBED_SUM, s, 0.0, ((double)N + V) * D * sizeof(T));
    if (!launch_on<SumJob, const T*, T*, unsigned>(
            k_embed_sum<T, VB>, (unsigned)(sum_blocks + zero_blocks), 256, 0, 1, true, s, j,
            (const T*)dout, (T*)dtable, (unsigned)sum_blocks))
      return SLIM_ERR_CUDA;
  }
  if (p.chunks > 1) {
    prof::Scope ps(prof::K_EMBED_JOIN, s);
    if (!launch_on<SumJob, T*>(k_embed_join<T, VB>, (unsigned)(p.chunks - 1), kJoinThreads, 0, 1,
                               true, s, j, (T*)dtable))
      return SLIM_ERR_CUDA;
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
