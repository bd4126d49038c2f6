// Pages of the paged K/V cache: extend, fork, unshare, free, copy, compact.
//
// refs is the only record of what is free (0), so a free page is found by a scan,
// and which one a call takes depends on the cache's state alone: the lowest ids.
// One workgroup plans a call: it checks the arguments, counts the pages wanted and
// looks through refs for that many before anything is changed, so that a call does
// all or nothing without the host. A second launch moves the bytes with the whole
// device. Counts change by integer additions, so no result depends on an order.
// Planning is bound by latency (a few passes over LDS and refs), copies by HBM.
#include "cache.h"

namespace daf {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

constexpr int kPlan = 1024;               // threads of a planning workgroup
constexpr int kPer = kMaxPageSeqs / kPlan;  // sequences per thread
constexpr int kHash = 2 * kMaxPageSeqs;   // slots of the set of sequences
constexpr int kCopyThreads = 256;
constexpr int kPiece = 4 * kCopyThreads * 16;  // bytes a workgroup moves at a time

// Exclusive prefix sums over the workgroup's threads, in 64 bits (a sum may pass 32
// on its way to being refused); *total gets the sum. sh: 17 words.
__device__ __forceinline__ int64_t block_scan(int64_t x, int64_t *sh, int64_t *total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int64_t s = x;
#pragma unroll
  for (int k = 1; k < 64; k <<= 1) {
    const int64_t y = __shfl_up(s, k);
    if (lane >= k) s += y;
  }
  __syncthreads();  // sh may still be read from the scan before
  if (lane == 63) sh[wave] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    int64_t sum = 0;
    for (int w = 0; w < kPlan / 64; ++w) {
      const int64_t y = sh[w];
      sh[w] = sum;
      sum += y;
    }
    sh[kPlan / 64] = sum;
  }
  __syncthreads();
  *total = sh[kPlan / 64];
  return sh[wave] + s - x;
}

// A set of sequence numbers: open addressing over kHash slots, at most half full.
__device__ __forceinline__ unsigned hash_of(int key) { return (unsigned)key * 2654435761u >> 19; }
static_assert(kHash == 1 << 13, "hash_of gives 13 bits");
// false if the key was there already
__device__ __forceinline__ bool set_add(int *set, int key) {
  for (unsigned i = hash_of(key);; i = (i + 1) & (kHash - 1)) {
    const int old = atomicCAS(&set[i], -1, key);
    if (old == -1) return true;
    if (old == key) return false;
  }
}
__device__ __forceinline__ bool set_has(const int *set, int key) {
  for (unsigned i = hash_of(key);; i = (i + 1) & (kHash - 1)) {
    if (set[i] == key) return true;
    if (set[i] == -1) return false;
  }
}

// Walks the free pages in order of their ids, 4 per thread and step, until `want`
// of them were seen: f(rank, id) for each. Returns how many there were (<= want).
template <typename F>
__device__ __forceinline__ int64_t walk_free(const int32_t *refs, int n_pages, int64_t want, int64_t *sh, F f) {
  int64_t seen = 0;
  for (int64_t base = 0; base < n_pages && seen < want; base += kPlan * 4) {
    const int64_t at = base + threadIdx.x * 4;
    int r[4];
    if (at + 4 <= n_pages) {
      const i32x4 v = *reinterpret_cast<const i32x4 *>(refs + at);
#pragma unroll
      for (int k = 0; k < 4; ++k) r[k] = v[k];
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k) r[k] = at + k < n_pages ? refs[at + k] : 1;
    }
    int64_t mine = 0, total;
#pragma unroll
    for (int k = 0; k < 4; ++k) mine += r[k] <= 0;
    int64_t rank = seen + block_scan(mine, sh, &total);
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (r[k] <= 0) {
        if (rank < want) f((int)rank, (int)(at + k));
        ++rank;
      }
    seen += total;
  }
  return seen < want ? seen : want;
}

__device__ __forceinline__ int pages_of(int tokens) { return (tokens + kPage - 1) / kPage; }
__device__ __forceinline__ bool in_range(int x, int n) { return (unsigned)x < (unsigned)n; }

__global__ __launch_bounds__(kPlan) void pages_extend_kernel(const PoolView c, int n, const int32_t *seq,
                                                             const int32_t *n_new, int32_t *status) {
  __shared__ int set[kHash];
  __shared__ int off[kMaxPageSeqs];
  __shared__ int64_t sh[kPlan / 64 + 1];
  __shared__ int bad;
  const int t = threadIdx.x;
  for (int i = t; i < kHash; i += kPlan) set[i] = -1;
  if (t == 0) bad = 0;
  __syncthreads();
  int have[kPer], add[kPer], need[kPer];
  int64_t mine = 0;
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const int i = t * kPer + k;
    have[k] = add[k] = need[k] = 0;
    if (i >= n) continue;
    const int s = seq ? seq[i] : i;
    add[k] = n_new ? n_new[i] : 1;
    if (!in_range(s, c.n_seqs) || add[k] < 0 || !set_add(set, s)) {
      bad = 1;
      continue;
    }
    have[k] = seq_len(c.len, c.n_seqs, c.max_seq_pages, s);
    if ((int64_t)have[k] + add[k] > (int64_t)c.max_seq_pages * kPage) {
      bad = 1;
      continue;
    }
    need[k] = pages_of(have[k] + add[k]) - pages_of(have[k]);
    mine += need[k];
  }
  int64_t want;
  int64_t at = block_scan(mine, sh, &want);  // a barrier: `bad` is final
  if (bad) {
    if (t == 0) *status = -1;
    return;
  }
  int64_t found = walk_free(c.refs, c.n_pages, want, sh, [](int, int) {});
  if (found < want) {
    if (t == 0) *status = (int)min(want - found, (int64_t)INT32_MAX);
    return;
  }
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    off[t * kPer + k] = (int)at;  // want <= n_pages here
    at += need[k];
  }
  __syncthreads();
  walk_free(c.refs, c.n_pages, want, sh, [&](int rank, int id) {
    int i = 0;  // the last request whose pages start at or below the rank
    for (int step = kMaxPageSeqs / 2; step; step >>= 1)
      if (off[i + step] <= rank) i += step;
    const int s = seq ? seq[i] : i;
    const int first = pages_of(seq_len(c.len, c.n_seqs, c.max_seq_pages, s));
    c.table[(int64_t)s * c.max_seq_pages + first + rank - off[i]] = id;
    c.refs[id] = 1;
  });
  __syncthreads();  // lengths are read above
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const int i = t * kPer + k;
    if (i < n) c.len[seq ? seq[i] : i] = have[k] + add[k];
  }
  if (t == 0) *status = 0;
}

__global__ __launch_bounds__(kPlan) void pages_fork_kernel(const PoolView c, const PageWork w, int n,
                                                           const int32_t *src, const int32_t *dst, int32_t *status) {
  __shared__ int set[kHash];
  __shared__ int64_t sh[kPlan / 64 + 1];
  __shared__ int bad;
  const int t = threadIdx.x;
  for (int i = t; i < kHash; i += kPlan) set[i] = -1;
  if (t == 0) bad = 0, w.count[0] = 0, w.count[1] = 0;
  __syncthreads();
  int s[kPer], d[kPer], L[kPer];
  int64_t mine = 0;
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const int i = t * kPer + k;
    s[k] = d[k] = -1;
    L[k] = 0;
    if (i >= n) continue;
    s[k] = src[i];
    d[k] = dst[i];
    if (!in_range(s[k], c.n_seqs) || !in_range(d[k], c.n_seqs) || c.len[d[k]] > 0 || !set_add(set, d[k])) {
      bad = 1;
      continue;
    }
    L[k] = seq_len(c.len, c.n_seqs, c.max_seq_pages, s[k]);
    mine += L[k] % kPage > 0;
  }
  int64_t want;
  int64_t rank = block_scan(mine, sh, &want);
#pragma unroll
  for (int k = 0; k < kPer; ++k)
    if (s[k] >= 0 && set_has(set, s[k])) bad = 1;
  __syncthreads();
  if (bad) {
    if (t == 0) *status = -1;
    return;
  }
  const int64_t found = walk_free(c.refs, c.n_pages, want, sh, [](int, int) {});
  if (found < want) {
    if (t == 0) *status = (int)(want - found);
    return;
  }
  walk_free(c.refs, c.n_pages, want, sh, [&](int r, int id) {
    w.dst[r] = id;
    c.refs[id] = 1;
  });
  __syncthreads();
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    if (d[k] < 0) continue;
    if (L[k] % kPage) {
      const int full = L[k] / kPage;
      w.src[rank] = c.table[(int64_t)s[k] * c.max_seq_pages + full];
      c.table[(int64_t)d[k] * c.max_seq_pages + full] = w.dst[rank];
      ++rank;
    }
    c.len[d[k]] = L[k];
  }
  if (t == 0) {
    w.count[0] = (int)want;
    w.count[1] = 1;  // shared pages may follow
    *status = 0;
  }
}

// Rows of the launch in tiles of kPlan; a row that is its page's first in its
// request stands for the page. The pages that are shared are listed in order.
__global__ __launch_bounds__(kPlan) void pages_unshare_kernel(const UnshareLaunch p) {
  __shared__ int set[kHash];
  __shared__ int64_t sh[kPlan / 64 + 1];
  __shared__ int bad;
  const PoolView &c = p.c;
  const int t = threadIdx.x;
  for (int i = t; i < kHash; i += kPlan) set[i] = -1;
  if (t == 0) bad = 0, p.w.count[0] = 0, p.w.count[1] = 0;
  __syncthreads();
  if (t < p.n_req) {
    const int s = p.seq ? p.seq[t] : t;
    if (!in_range(s, c.n_seqs) || !set_add(set, s)) bad = 1;
  }
  __syncthreads();
  if (bad) {
    if (t == 0) *p.status = -1;
    return;
  }
  const int rows = p.cu[p.n_req];
  int64_t want = 0;
  for (int64_t base = 0; base < rows; base += kPlan) {
    const int64_t i = base + t;
    bool take = false;
    int64_t slot = 0;
    int page = -1;
    if (i < rows) {
      int b = 0;
      for (int step = kMaxCacheReqs / 2; step; step >>= 1)
        if (b + step < p.n_req && p.cu[b + step] <= i) b += step;
      const int s = p.seq ? p.seq[b] : b;
      const int L = seq_len(c.len, c.n_seqs, c.max_seq_pages, s);
      const int j = (int)i - p.cu[b];
      const int shift = L - (p.cu[b + 1] - p.cu[b]);
      const int at = p.pos ? p.pos[i] : shift + j;
      const int before = j == 0 ? -1 : p.pos ? p.pos[i - 1] : at - 1;
      if (p.pos && j > 0 && before >= at) bad = 1;  // a page would be listed twice
      if (at >= 0 && at < L && (before < 0 || before / kPage != at / kPage)) {
        slot = (int64_t)s * c.max_seq_pages + at / kPage;
        page = c.table[slot];
        take = in_range(page, c.n_pages) && c.refs[page] > 1;
      }
    }
    int64_t total;
    const int64_t rank = want + block_scan(take, sh, &total);
    if (take && rank < c.n_pages) {
      p.w.src[rank] = page;
      // the table entry, in two words (dst is not needed yet)
      p.w.aux[rank] = (int)(slot % c.max_seq_pages);
      p.w.dst[rank] = (int)(slot / c.max_seq_pages);
    }
    want += total;
  }
  if (bad) {  // final since the last scan's barriers
    if (t == 0) *p.status = -1;
    return;
  }
  const int64_t found = walk_free(c.refs, c.n_pages, want, sh, [](int, int) {});
  if (found < want) {
    if (t == 0) *p.status = (int)min(want - found, (int64_t)INT32_MAX);
    return;
  }
  __syncthreads();
  // free ids are found before any count changes: none of the old pages is among them
  walk_free(c.refs, c.n_pages, want, sh, [&](int r, int id) {
    c.table[(int64_t)p.w.dst[r] * c.max_seq_pages + p.w.aux[r]] = id;
    p.w.dst[r] = id;
    c.refs[id] = 1;
  });
  __syncthreads();
  for (int64_t r = t; r < want; r += kPlan) atomicAdd(&c.refs[p.w.src[r]], -1);
  if (t == 0) {
    p.w.count[0] = (int)want;
    *p.status = 0;
  }
}

__global__ __launch_bounds__(kCopyThreads) void pages_free_kernel(const PoolView c, int n, const int32_t *seq) {
  __shared__ int tokens;
  const int s = seq ? seq[blockIdx.x] : (int)blockIdx.x;
  if (!in_range(s, c.n_seqs)) return;
  if (threadIdx.x == 0) tokens = atomicExch(&c.len[s], 0);  // one of two workgroups of a sequence gets it
  __syncthreads();
  const int pages = pages_of(min(max(tokens, 0), c.max_seq_pages * kPage));
  int32_t *row = c.table + (int64_t)s * c.max_seq_pages;
  for (int i = threadIdx.x; i < pages; i += kCopyThreads) {
    const int id = row[i];
    row[i] = -1;
    if (in_range(id, c.n_pages)) atomicAdd(&c.refs[id], -1);
  }
}

// One pass over refs with f(id, used, rank among the used ones); returns their number.
template <typename F>
__device__ __forceinline__ int64_t walk_all(const PoolView &c, int64_t *sh, F f) {
  int64_t seen = 0;
  for (int64_t base = 0; base < c.n_pages; base += kPlan * 4) {
    const int64_t at = base + threadIdx.x * 4;
    bool used[4];
    int64_t mine = 0, total;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      used[k] = at + k < c.n_pages && c.refs[at + k] > 0;
      mine += used[k];
    }
    int64_t rank = seen + block_scan(mine, sh, &total);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (at + k < c.n_pages) f((int)(at + k), used[k], (int)rank);
      rank += used[k];
    }
    seen += total;
  }
  return seen;
}

// The i-th used page at or past n_live and the i-th free one below: with `live`
// used pages before id, a free id below n_live has rank id - live among the free,
// and a used one at or past it has rank live - (used ones below n_live).
__global__ __launch_bounds__(kPlan) void pages_compact_kernel(const PoolView c, const PageWork w, int32_t *n_live) {
  __shared__ int64_t sh[kPlan / 64 + 1];
  __shared__ int below;
  const int live = (int)walk_all(c, sh, [](int, bool, int) {});
  if (threadIdx.x == 0) below = 0;
  __syncthreads();
  walk_all(c, sh, [&](int id, bool used, int rank) {
    if (id < live) {
      if (!used) w.dst[id - rank] = id;
      if (id == live - 1) below = rank + used;
    }
    w.aux[id] = id;
  });
  __syncthreads();
  walk_all(c, sh, [&](int id, bool used, int rank) {
    if (used && id >= live) w.src[rank - below] = id;
  });
  __syncthreads();
  const int moves = live - below;
  for (int i = threadIdx.x; i < moves; i += kPlan) {
    const int a = w.src[i], b = w.dst[i];
    w.aux[a] = b;
    c.refs[b] = c.refs[a];
    c.refs[a] = 0;
  }
  if (threadIdx.x == 0) {
    w.count[0] = moves;
    w.count[1] = 0;
    *n_live = live;
  }
}

// Pieces of the pairs' pages in every layer, a workgroup at a time: K, then V, with
// the scales by the first piece of a page and layer.
__device__ __forceinline__ void copy_pairs(const PoolView &c, const int32_t *src, const int32_t *dst, int n, int first,
                                           int step) {
  const int64_t bytes = (int64_t)c.hkv * kPage * c.d;  // of K or V of a page in a layer
  const int64_t pieces = (bytes + kPiece - 1) / kPiece;
  const int64_t per = pieces * 2 * c.n_layers, units = per * n;
  for (int64_t u = first; u < units; u += step) {
    const int pair = (int)(u / per);
    int64_t rest = u - pair * per;
    const int layer = (int)(rest / (2 * pieces));
    rest -= (int64_t)layer * 2 * pieces;
    const bool is_v = rest >= pieces;
    const int64_t at = (is_v ? rest - pieces : rest) * kPiece;
    const int a = src[pair], b = dst[pair];
    if (!in_range(a, c.n_pages) || !in_range(b, c.n_pages) || a == b) continue;
    const int64_t l0 = (int64_t)layer * c.n_pages;
    unsigned char *pool = is_v ? c.v : c.k;
    const unsigned char *from = pool + (l0 + a) * bytes + at;
    unsigned char *to = pool + (l0 + b) * bytes + at;
    const int64_t left = bytes - at;
    u32x4 x[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int o = (k * kCopyThreads + threadIdx.x) * 16;
      if (o < left) x[k] = *reinterpret_cast<const u32x4 *>(from + o);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int o = (k * kCopyThreads + threadIdx.x) * 16;
      if (o < left) *reinterpret_cast<u32x4 *>(to + o) = x[k];
    }
    if (rest == 0)
      for (int h = threadIdx.x; h < c.hkv; h += kCopyThreads) {
        c.k_scale[(l0 + b) * c.hkv + h] = c.k_scale[(l0 + a) * c.hkv + h];
        c.v_scale[(l0 + b) * c.hkv + h] = c.v_scale[(l0 + a) * c.hkv + h];
      }
  }
}

__global__ __launch_bounds__(kCopyThreads) void pages_copy_kernel(const PoolView c, const int32_t *src,
                                                                  const int32_t *dst, int n) {
  copy_pairs(c, src, dst, n, blockIdx.x, gridDim.x);
}

// After a plan: the first `rows` workgroups work on tables, the others copy.
enum class After { kUnshare, kFork, kCompact };
template <After WHAT>
__global__ __launch_bounds__(kCopyThreads) void pages_apply_kernel(const PoolView c, const PageWork w, int rows,
                                                                   const int32_t *src, const int32_t *dst) {
  if ((int)blockIdx.x >= rows) {
    copy_pairs(c, w.src, w.dst, w.count[0], blockIdx.x - rows, gridDim.x - rows);
    return;
  }
  if constexpr (WHAT == After::kFork) {  // the full pages
    if (!w.count[1]) return;
    const int a = src[blockIdx.x], b = dst[blockIdx.x];
    const int full = seq_len(c.len, c.n_seqs, c.max_seq_pages, a) / kPage;
    for (int i = threadIdx.x; i < full; i += kCopyThreads) {
      const int id = c.table[(int64_t)a * c.max_seq_pages + i];
      c.table[(int64_t)b * c.max_seq_pages + i] = id;
      if (in_range(id, c.n_pages)) atomicAdd(&c.refs[id], 1);
    }
  }
  if constexpr (WHAT == After::kCompact) {
    for (int s = blockIdx.x; s < c.n_seqs; s += rows) {
      const int pages = pages_of(seq_len(c.len, c.n_seqs, c.max_seq_pages, s));
      int32_t *row = c.table + (int64_t)s * c.max_seq_pages;
      for (int i = threadIdx.x; i < pages; i += kCopyThreads)
        if (in_range(row[i], c.n_pages)) row[i] = w.aux[row[i]];
    }
  }
}

// Workgroups that copy up to `pairs` pages: as many as there can be pieces, at most
// 8 per CU (a workgroup has 16 KiB in flight).
int copy_grid(const PoolView &c, int64_t pairs) {
  const int64_t bytes = (int64_t)c.hkv * kPage * c.d;
  const int64_t units = pairs * 2 * c.n_layers * ((bytes + kPiece - 1) / kPiece);
  return (int)(units < 1 ? 1 : units < 2048 ? units : 2048);
}

}  // namespace

hipError_t launch_pages_extend(const PoolView &c, int n, const int32_t *seq, const int32_t *n_new, int32_t *status,
                               hipStream_t st) {
  pages_extend_kernel<<<1, kPlan, 0, st>>>(c, n, seq, n_new, status);
  return hipGetLastError();
}

hipError_t launch_pages_fork(const PoolView &c, const PageWork &w, int n, const int32_t *src, const int32_t *dst,
                             int32_t *status, hipStream_t st) {
  pages_fork_kernel<<<1, kPlan, 0, st>>>(c, w, n, src, dst, status);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  pages_apply_kernel<After::kFork><<<n + copy_grid(c, n), kCopyThreads, 0, st>>>(c, w, n, src, dst);
  return hipGetLastError();
}

hipError_t launch_pages_unshare(const UnshareLaunch &p, hipStream_t st) {
  pages_unshare_kernel<<<1, kPlan, 0, st>>>(p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int64_t rows = p.cu[p.n_req];
  const int64_t pairs = rows < p.c.n_pages ? rows : p.c.n_pages;
  pages_apply_kernel<After::kUnshare><<<copy_grid(p.c, pairs), kCopyThreads, 0, st>>>(p.c, p.w, 0, nullptr, nullptr);
  return hipGetLastError();
}

hipError_t launch_pages_free(const PoolView &c, int n, const int32_t *seq, hipStream_t st) {
  pages_free_kernel<<<n, kCopyThreads, 0, st>>>(c, n, seq);
  return hipGetLastError();
}

hipError_t launch_pages_copy(const PoolView &c, int n, const int32_t *src, const int32_t *dst, hipStream_t st) {
  pages_copy_kernel<<<copy_grid(c, n), kCopyThreads, 0, st>>>(c, src, dst, n);
  return hipGetLastError();
}

hipError_t launch_pages_compact(const PoolView &c, const PageWork &w, int32_t *n_live, hipStream_t st) {
  pages_compact_kernel<<<1, kPlan, 0, st>>>(c, w, n_live);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int rows = c.n_seqs < 1024 ? c.n_seqs : 1024;
  pages_apply_kernel<After::kCompact><<<rows + copy_grid(c, c.n_pages / 2), kCopyThreads, 0, st>>>(c, w, rows, nullptr,
                                                                                                  nullptr);
  return hipGetLastError();
}

}  // namespace daf
