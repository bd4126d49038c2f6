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

// Exclusive prefix sums over the workgroup's threads; *total gets the sum. sh: one
// word per wave. (64 bits where a sum may pass 32 on its way to being refused.)
template <typename T>
__device__ __forceinline__ T block_scan(T x, T *sh, T *total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  T s = x;
#pragma unroll
  for (int k = 1; k < 64; k <<= 1) {
    const T y = __shfl_up(s, k);
    if (lane >= k) s += y;
  }
  __syncthreads();  // sh may still be read from the scan before
  if (lane == 63) sh[wave] = s;
  __syncthreads();
  // every wave adds up the waves' sums
  T w = lane < kPlan / 64 ? sh[lane] : 0;
#pragma unroll
  for (int k = 1; k < kPlan / 64; k <<= 1) {
    const T y = __shfl_up(w, k);
    if (lane >= k) w += y;
  }
  *total = __shfl(w, kPlan / 64 - 1);
  const T before = __shfl(w, max(wave - 1, 0));
  return (wave ? before : 0) + s - x;
}

// A set of sequence numbers: open addressing over slots of which at most half are taken.
__device__ __forceinline__ unsigned hash_of(int key) { return (unsigned)key * 2654435761u >> 19; }
static_assert(kHash == 1 << 13, "hash_of gives 13 bits");
// false if the key was there already; slots: a power of two of at most kHash
__device__ __forceinline__ bool set_add(int *set, int key, int slots = kHash) {
  for (unsigned i = hash_of(key) & (slots - 1);; i = (i + 1) & (slots - 1)) {
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

// refs of the 16 pages from `at` on (a multiple of 4) as bits: used ones
__device__ __forceinline__ unsigned used_bits(const int32_t *refs, int n_pages, int64_t at) {
  unsigned bits = 0;
  i32x4 v[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const int64_t i = at + 4 * q;
    v[q] = i32x4{};
    if (i + 4 <= n_pages) {
      v[q] = *reinterpret_cast<const i32x4 *>(refs + i);
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k) v[q][k] = i + k < n_pages ? refs[i + k] : 0;
    }
  }
#pragma unroll
  for (int i = 0; i < 16; ++i) bits |= (unsigned)(v[i >> 2][i & 3] > 0) << i;
  return bits;
}

// Walks the free pages in order of their ids, 16 per thread and step, until `want` of
// them were seen: f(rank, id) for each. Returns how many there were (<= want).
template <typename F>
__device__ __forceinline__ int64_t walk_free(const int32_t *refs, int n_pages, int64_t want, int *sh, F f) {
  int64_t seen = 0;
  for (int64_t base = 0; base < n_pages && seen < want; base += kPlan * 16) {
    const int64_t at = base + threadIdx.x * 16;
    const int here = (int)min(max((int64_t)n_pages - at, (int64_t)0), (int64_t)16);
    unsigned free_ = ~used_bits(refs, n_pages, at) & ((1u << here) - 1);
    int total;
    int64_t rank = seen + block_scan(__builtin_popcount(free_), sh, &total);
    for (; free_ && rank < want; free_ &= free_ - 1, ++rank) f((int)rank, (int)at + __builtin_ctz(free_));
    seen += total;
  }
  return seen < want ? seen : want;
}

// The same into a list of kShort in LDS, which is complete if `want` is not more.
constexpr int kShort = kMaxPageSeqs;
__device__ __forceinline__ int64_t list_free(const PoolView &c, int64_t want, int *sh, int *list) {
  const int64_t found = walk_free(c.refs, c.n_pages, want, sh, [&](int rank, int id) {
    if (rank < kShort) list[rank] = id;
  });
  __syncthreads();
  return found;
}

__device__ __forceinline__ int pages_of(int tokens) { return (tokens + kPage - 1) / kPage; }
__device__ __forceinline__ bool in_range(int x, int n) { return (unsigned)x < (unsigned)n; }

__global__ __launch_bounds__(kPlan) void pages_extend_kernel(const PoolView c, int n, const int32_t *seq,
                                                             const int32_t *n_new, int32_t *status) {
  __shared__ int set[kHash];
  __shared__ int off[kMaxPageSeqs], list[kShort];
  __shared__ int64_t sh64[kPlan / 64];
  __shared__ int sh[kPlan / 64];
  __shared__ int bad;
  const int t = threadIdx.x;
  if (n > 1)  // one sequence has no double
    for (int i = t; i < kHash; i += kPlan) set[i] = -1;
  if (t == 0) bad = 0;
  int s[kPer], have[kPer], add[kPer], need[kPer];
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const int i = t * kPer + k;
    s[k] = i >= n ? -1 : seq ? seq[i] : i;
    add[k] = i >= n ? 0 : n_new ? n_new[i] : 1;
  }
#pragma unroll
  for (int k = 0; k < kPer; ++k) have[k] = seq_len(c.len, c.n_seqs, c.max_seq_pages, s[k]);
  __syncthreads();
  int64_t mine = 0;
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    need[k] = 0;
    if (t * kPer + k >= n) continue;
    if (!in_range(s[k], c.n_seqs) || add[k] < 0 || (n > 1 && !set_add(set, s[k])) ||
        (int64_t)have[k] + add[k] > (int64_t)c.max_seq_pages * kPage) {
      bad = 1;
      continue;
    }
    need[k] = pages_of(have[k] + add[k]) - pages_of(have[k]);
    mine += need[k];
  }
  int64_t want;
  int64_t at = block_scan(mine, sh64, &want);  // its barriers make `bad` final
  if (bad) {
    if (t == 0) *status = -1;
    return;
  }
  const int64_t found = list_free(c, want, sh, list);
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
  auto give = [&](int rank, int id) {
    int i = 0;  // the last request whose pages start at or below the rank
    for (int step = kMaxPageSeqs / 2; step; step >>= 1)
      if (off[i + step] <= rank) i += step;
    const int to = seq ? seq[i] : i;
    const int first = pages_of(seq_len(c.len, c.n_seqs, c.max_seq_pages, to));
    c.table[(int64_t)to * c.max_seq_pages + first + rank - off[i]] = id;
    c.refs[id] = 1;
  };
  if (want <= kShort) {
    for (int r = t; r < want; r += kPlan) give(r, list[r]);
  } else {
    walk_free(c.refs, c.n_pages, want, sh, give);
  }
  __syncthreads();  // lengths are read above
#pragma unroll
  for (int k = 0; k < kPer; ++k)
    if (t * kPer + k < n) c.len[s[k]] = have[k] + add[k];
  if (t == 0) *status = 0;
}

__global__ __launch_bounds__(kPlan) void pages_fork_kernel(const PoolView c, const PageWork w, int n,
                                                           const int32_t *src, const int32_t *dst, int32_t *status) {
  __shared__ int set[kHash];
  __shared__ int list[kShort];
  __shared__ int sh[kPlan / 64];
  __shared__ int bad;
  const int t = threadIdx.x;
  for (int i = t; i < kHash; i += kPlan) set[i] = -1;
  if (t == 0) bad = 0, w.count[0] = 0, w.count[1] = 0;
  int s[kPer], d[kPer], L[kPer], held[kPer], last[kPer], mine = 0;
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const int i = t * kPer + k;
    s[k] = i < n ? src[i] : -1;
    d[k] = i < n ? dst[i] : -1;
  }
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    held[k] = in_range(d[k], c.n_seqs) ? c.len[d[k]] : 0;
    L[k] = seq_len(c.len, c.n_seqs, c.max_seq_pages, s[k]);
  }
#pragma unroll
  for (int k = 0; k < kPer; ++k)  // the last page, where it is not full
    last[k] = L[k] % kPage ? c.table[(int64_t)s[k] * c.max_seq_pages + L[k] / kPage] : -1;
  auto own = [&](int k) { return in_range(last[k], c.n_pages); };  // one that is not there stays so
  __syncthreads();
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    if (t * kPer + k >= n) continue;
    if (!in_range(s[k], c.n_seqs) || !in_range(d[k], c.n_seqs) || held[k] > 0 || !set_add(set, d[k])) bad = 1;
    mine += own(k);
  }
  int want;
  int rank = block_scan(mine, sh, &want);
#pragma unroll
  for (int k = 0; k < kPer; ++k)
    if (in_range(s[k], c.n_seqs) && !bad && set_has(set, s[k])) bad = 1;
  __syncthreads();
  if (bad) {
    if (t == 0) *status = -1;
    return;
  }
  const int found = (int)list_free(c, want, sh, list);
  if (found < want) {
    if (t == 0) *status = want - found;
    return;
  }
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    if (t * kPer + k >= n) continue;
    if (L[k] % kPage) {
      const int id = own(k) ? list[rank] : last[k];
      c.table[(int64_t)d[k] * c.max_seq_pages + L[k] / kPage] = id;
      if (own(k)) {
        w.src[rank] = last[k];
        w.dst[rank] = id;
        c.refs[id] = 1;
        ++rank;
      }
    }
    c.len[d[k]] = L[k];
  }
  if (t == 0) {
    w.count[0] = want;
    w.count[1] = 1;  // shared pages may follow
    *status = 0;
  }
}

constexpr int kRowsPer = 8;
// Rows of the launch, kRowsPer per thread and step; a row that is its page's first in its
// request stands for the page. The pages that are shared are listed in order.
__global__ __launch_bounds__(kPlan) void pages_unshare_kernel(const UnshareLaunch p) {
  __shared__ int set[2 * kMaxCacheReqs];
  __shared__ int seqs[kMaxCacheReqs], lens[kMaxCacheReqs], cu[kMaxCacheReqs + 1];
  __shared__ int sh[kPlan / 64];
  __shared__ int bad;
  const PoolView &c = p.c;
  const int t = threadIdx.x;
  if (t < 2 * kMaxCacheReqs) set[t] = -1;
  if (t == 0) bad = 0, p.w.count[0] = 0, p.w.count[1] = 0;
  if (t <= p.n_req) cu[t] = p.cu[t];
  __syncthreads();
  if (t < p.n_req) {
    const int s = p.seq ? p.seq[t] : t;
    seqs[t] = s;
    lens[t] = seq_len(c.len, c.n_seqs, c.max_seq_pages, s);
    if (!in_range(s, c.n_seqs) || !set_add(set, s, 2 * kMaxCacheReqs)) bad = 1;
  }
  __syncthreads();
  if (bad) {
    if (t == 0) *p.status = -1;
    return;
  }
  const int rows = cu[p.n_req];
  int64_t want = 0;
  for (int64_t base = 0; base < rows; base += kPlan * kRowsPer) {
    int64_t slot[kRowsPer];
    int page[kRowsPer], seq_[kRowsPer], col[kRowsPer], mine = 0;
    bool first[kRowsPer];
#pragma unroll
    for (int k = 0; k < kRowsPer; ++k) {
      const int64_t i = base + t * kRowsPer + k;
      first[k] = false;
      if (i >= rows) continue;
      int b = 0;
      for (int step = kMaxCacheReqs / 2; step; step >>= 1)
        if (b + step < p.n_req && cu[b + step] <= i) b += step;
      const int j = (int)i - cu[b], L = lens[b];
      const int at = p.pos ? p.pos[i] : L - (cu[b + 1] - cu[b]) + j;
      const int before = j == 0 ? -1 : p.pos ? p.pos[i - 1] : at - 1;
      if (p.pos && j > 0 && before >= at) bad = 1;  // a page would be listed twice
      first[k] = at >= 0 && at < L && (before < 0 || before / kPage != at / kPage);
      seq_[k] = seqs[b];
      col[k] = at / kPage;
      slot[k] = (int64_t)seq_[k] * c.max_seq_pages + col[k];
    }
#pragma unroll
    for (int k = 0; k < kRowsPer; ++k) page[k] = first[k] ? c.table[slot[k]] : -1;
#pragma unroll
    for (int k = 0; k < kRowsPer; ++k) {
      first[k] = in_range(page[k], c.n_pages) && c.refs[page[k]] > 1;
      mine += first[k];
    }
    int total;
    int64_t rank = want + block_scan(mine, sh, &total);
#pragma unroll
    for (int k = 0; k < kRowsPer; ++k)
      if (first[k]) {
        if (rank < c.n_pages) p.w.src[rank] = page[k], p.w.seq[rank] = seq_[k], p.w.aux[rank] = col[k];
        ++rank;
      }
    want += total;
  }
  if (bad) {  // final since the last scan's barriers
    if (t == 0) *p.status = -1;
    return;
  }
  // free ids are found before any count changes: none of the old pages is among them
  const int64_t found = walk_free(c.refs, c.n_pages, want, sh, [&](int r, int id) { p.w.dst[r] = id; });
  if (found < want) {
    if (t == 0) *p.status = (int)min(want - found, (int64_t)INT32_MAX);
    return;
  }
  __syncthreads();
  for (int64_t r = t; r < want; r += kPlan) {
    const int id = p.w.dst[r];
    c.table[(int64_t)p.w.seq[r] * c.max_seq_pages + p.w.aux[r]] = id;
    c.refs[id] = 1;
    atomicAdd(&c.refs[p.w.src[r]], -1);
  }
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

// The i-th used page at or past n_live goes to the i-th free one below. A thread has a
// run of pages: with u used ones before page id, it is the (id - u)-th free one or the
// (u - below)-th used one at or past n_live, `below` of which lie below that.
__global__ __launch_bounds__(kPlan) void pages_compact_kernel(const PoolView c, const PageWork w, int32_t *n_live) {
  __shared__ int sh[kPlan / 64];
  __shared__ int below;
  const int t = threadIdx.x;
  const int run = ((c.n_pages + kPlan - 1) / kPlan + 15) / 16 * 16;
  const int64_t from = (int64_t)t * run, to = min(from + run, (int64_t)c.n_pages);
  int mine = 0;
  for (int64_t at = from; at < to; at += 16) mine += __builtin_popcount(used_bits(c.refs, c.n_pages, at));
  int live;
  const int before = block_scan(mine, sh, &live);
  if (t == 0) below = live;  // all pages are used
  __syncthreads();
  if (live >= from && live < to) {
    int u = before;
    for (int64_t at = from; at < live; at += 16)
      u += __builtin_popcount(used_bits(c.refs, c.n_pages, at) & (live - at >= 16 ? 0xffffu : (1u << (live - at)) - 1));
    below = u;
  }
  __syncthreads();
  int u = before;
  for (int64_t at = from; at < to; at += 16) {
    const unsigned bits = used_bits(c.refs, c.n_pages, at);
    const int end = (int)min(to - at, (int64_t)16);
    for (int i = 0; i < end; ++i) {
      const int id = (int)at + i;
      const bool used = (bits >> i) & 1;
      if (id >= live && used) w.src[u - below] = id;
      if (id < live && !used) w.dst[id - u] = id;
      w.aux[id] = id;
      u += used;
    }
  }
  __syncthreads();
  const int moves = live - below;
  for (int i = t; i < moves; i += kPlan) {
    const int a = w.src[i], b = w.dst[i];
    w.aux[a] = b;
    c.refs[b] = c.refs[a];
    c.refs[a] = 0;
  }
  if (t == 0) {
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
