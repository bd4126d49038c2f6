// Pages of the paged K/V cache: extend, fork, unshare, free, copy, compact.
//
// refs is the only record of what is free (0), so a free page is found by a scan,
// and which one a call takes depends on the cache's state alone: the lowest ids.
// One workgroup plans a call: it checks the arguments, counts the pages wanted and
// looks through refs for that many before anything is changed, so that a call does
// all or nothing without the host. A second launch moves the bytes with the whole
// device. Counts change by integer additions, so no result depends on an order.
// Planning is bound by latency (4 to 8 us, unshare of 4915 rows 10.4), copies by HBM (512
// pages of 128 KiB 31 us, 4.3 TB/s). A plan's code runs once per call, so its fetch is
// part of the latency: loops over sequences and pages take one per thread and
// step and are not unrolled, and loads that depend on nothing come first.
#include "cache.h"

namespace daf {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

constexpr int kPlan = 1024;               // threads of a planning workgroup
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
  i32x4 v[4] = {};
  const int whole = n_pages & ~3;
#pragma unroll
  for (int q = 0; q < 4; ++q)
    if (at + 4 * q < whole) v[q] = *reinterpret_cast<const i32x4 *>(refs + at + 4 * q);
  if (at + 16 > whole && at < n_pages)  // the last pages, one by one
    for (int i = whole; i < n_pages; ++i) bits |= (unsigned)(refs[i] > 0) << (i - at);
#pragma unroll
  for (int i = 0; i < 16; ++i) bits |= (unsigned)(v[i >> 2][i & 3] > 0) << i;
  return bits;
}

// Walks the free pages in order of their ids, 16 per thread and step, until `want` of
// them were seen: f(rank, id) for each. Returns how many there were (<= want). used0:
// used_bits of the thread's first 16 pages.
template <typename F>
__device__ __forceinline__ int64_t walk_free(const int32_t *refs, int n_pages, int64_t want, unsigned used0, int *sh,
                                             F f) {
  int64_t seen = 0;
  for (int64_t base = 0; base < n_pages && seen < want; base += kPlan * 16) {
    const int64_t at = base + threadIdx.x * 16;
    const int here = (int)min(max((int64_t)n_pages - at, (int64_t)0), (int64_t)16);
    unsigned free_ = ~(base ? used_bits(refs, n_pages, at) : used0) & ((1u << here) - 1);
    int total;
    int64_t rank = seen + block_scan(__builtin_popcount(free_), sh, &total);
    for (; free_ && rank < want; free_ &= free_ - 1, ++rank) f((int)rank, (int)at + __builtin_ctz(free_));
    seen += total;
  }
  return seen < want ? seen : want;
}

constexpr int kShort = kMaxPageSeqs;  // lists of pages in LDS

__device__ __forceinline__ int pages_of(int tokens) { return (tokens + kPage - 1) / kPage; }
__device__ __forceinline__ bool in_range(int x, int n) { return (unsigned)x < (unsigned)n; }

__global__ __launch_bounds__(kPlan) void pages_extend_kernel(const PoolView c, int n, const int32_t *seq,
                                                             const int32_t *n_new, int32_t *status) {
  __shared__ int set[kHash];
  __shared__ int seqs[kMaxPageSeqs], held[kMaxPageSeqs], off[kMaxPageSeqs];  // off: first of its new pages
  __shared__ int to[kMaxPageSeqs], list[kShort];
  __shared__ int64_t sh64[kPlan / 64];
  __shared__ int sh[kPlan / 64];
  __shared__ int bad;
  const int t = threadIdx.x;
  const unsigned used0 = used_bits(c.refs, c.n_pages, t * 16);
  if (n > 1)  // one sequence has no double
    for (int i = t; i < kHash; i += kPlan) set[i] = -1;
  if (t == 0) bad = 0;
  int64_t want = 0;
  for (int i0 = 0; i0 < n; i0 += kPlan) {
    const int i = i0 + t;
    const int s = i >= n ? -1 : seq ? seq[i] : i, add = i >= n ? 0 : n_new ? n_new[i] : 1;
    const int have = seq_len(c.len, c.n_seqs, c.max_seq_pages, s);
    __syncthreads();  // the set is empty
    int64_t need = 0;
    if (i < n) {
      if (!in_range(s, c.n_seqs) || add < 0 || (n > 1 && !set_add(set, s)) ||
          (int64_t)have + add > (int64_t)c.max_seq_pages * kPage)
        bad = 1;
      else
        need = pages_of(have + add) - pages_of(have);
    }
    int64_t total;
    const int64_t at = want + block_scan(need, sh64, &total);
    if (i < n) seqs[i] = s, held[i] = have, off[i] = (int)at, to[i] = have + add;  // at is used if it fits
    want += total;
  }
  __syncthreads();
  if (bad) {
    if (t == 0) *status = -1;
    return;
  }
  auto entry = [&](int rank) {  // the table entry that the rank-th page is for
    int i = 0;  // the last request whose pages start at or below the rank
    for (int step = kMaxPageSeqs / 2; step; step >>= 1)
      if (i + step < n && off[i + step] <= rank) i += step;
    return c.table + (int64_t)seqs[i] * c.max_seq_pages + pages_of(held[i]) + rank - off[i];
  };
  auto give = [&](int rank, int id) {
    *entry(rank) = id;
    c.refs[id] = 1;
  };
  // a walk that looks for the pages and lists them; where the list is too short, another
  // that gives them
  const bool in_list = want <= kShort;
#pragma unroll 1
  for (int pass = 0; pass < (in_list ? 1 : 2); ++pass) {
    const int64_t found = walk_free(c.refs, c.n_pages, want, used0, sh, [&](int rank, int id) {
      if (in_list) list[rank] = id;
      else if (pass) give(rank, id);
    });
    if (found < want) {
      if (t == 0) *status = (int)min(want - found, (int64_t)INT32_MAX);
      return;
    }
    __syncthreads();
  }
  if (in_list)
    for (int r = t; r < want; r += kPlan) give(r, list[r]);
  for (int i = t; i < n; i += kPlan) c.len[seqs[i]] = to[i];
  if (t == 0) *status = 0;
  if (want == 0) return;
  // Scale 0, in every layer: what a page's last owner or a new pool left there would
  // count for the tokens that a write leaves out. (The pages' heads have 4 KiB of K
  // each, so their number fits 32 bits.) Few beside the bytes that are written there
  // next: a plan of 512 pages of 4 heads in 2 layers takes 7.9 us, without them 7.1.
  __syncthreads();  // ids past the list are read from the table
  const unsigned hkv = c.hkv, all = (unsigned)want * hkv;
  for (unsigned j = t; j < all; j += kPlan) {
    const unsigned r = j / hkv;
    const int64_t id = in_list ? list[r] : *entry(r);
    float *ks = c.k_scale + id * hkv + j % hkv, *vs = c.v_scale + id * hkv + j % hkv;
#pragma unroll 1
    for (int layer = 0; layer < c.n_layers; ++layer) {
      const int64_t at = (int64_t)layer * c.n_pages * hkv;
      ks[at] = 0.f;
      vs[at] = 0.f;
    }
  }
}

__global__ __launch_bounds__(kPlan) void pages_fork_kernel(const PoolView c, const PageWork w, int n,
                                                           const int32_t *src, const int32_t *dst, int32_t *status) {
  __shared__ int set[kHash];
  __shared__ int from[kMaxPageSeqs], to[kMaxPageSeqs], lens[kMaxPageSeqs];
  __shared__ int last[kMaxPageSeqs], rank[kMaxPageSeqs];  // last page, where it is not full, and its copy's rank
  __shared__ int list[kShort];
  __shared__ int sh[kPlan / 64];
  __shared__ int bad;
  const int t = threadIdx.x;
  const unsigned used0 = used_bits(c.refs, c.n_pages, t * 16);
  for (int i = t; i < kHash; i += kPlan) set[i] = -1;
  if (t == 0) bad = 0, w.count[0] = 0, w.count[1] = 0;
  int want = 0;
  for (int i0 = 0; i0 < n; i0 += kPlan) {
    const int i = i0 + t;
    const int s = i < n ? src[i] : -1, d = i < n ? dst[i] : -1;
    const int held = in_range(d, c.n_seqs) ? c.len[d] : 0;
    const int L = seq_len(c.len, c.n_seqs, c.max_seq_pages, s);
    const int page = L % kPage ? c.table[(int64_t)s * c.max_seq_pages + L / kPage] : -1;
    __syncthreads();  // the set is empty
    if (i < n && (!in_range(s, c.n_seqs) || !in_range(d, c.n_seqs) || held > 0 || !set_add(set, d))) bad = 1;
    int total;
    const int at = want + block_scan((int)in_range(page, c.n_pages), sh, &total);  // one that is not there stays so
    if (i < n) from[i] = s, to[i] = d, lens[i] = L, last[i] = page, rank[i] = at;
    want += total;
  }
  __syncthreads();
  if (!bad)
    for (int i = t; i < n; i += kPlan)
      if (set_has(set, from[i])) bad = 1;
  const int found = (int)walk_free(c.refs, c.n_pages, want, used0, sh, [&](int r, int id) { list[r] = id; });
  __syncthreads();
  if (bad || found < want) {
    if (t == 0) *status = bad ? -1 : want - found;
    return;
  }
  for (int i = t; i < n; i += kPlan) {
    const int L = lens[i];
    if (L % kPage) {
      int id = last[i];
      if (in_range(id, c.n_pages)) {
        const int r = rank[i];
        w.src[r] = id;
        id = list[r];
        w.dst[r] = id;
        c.refs[id] = 1;
      }
      c.table[(int64_t)to[i] * c.max_seq_pages + L / kPage] = id;
    }
    c.len[to[i]] = L;
  }
  if (t == 0) {
    w.count[0] = want;
    w.count[1] = 1;  // shared pages may follow
    *status = 0;
  }
}

// Rows of the launch, kRowsPer per thread and step. A row that is its page's first in its
// request stands for the page: these are listed, and the list's shared pages again.
constexpr int kRowsPer = 8, kStepRows = kRowsPer * kPlan;
__global__ __launch_bounds__(kPlan) void pages_unshare_kernel(const UnshareLaunch p) {
  __shared__ int set[2 * kMaxCacheReqs];
  __shared__ int seqs[kMaxCacheReqs], lens[kMaxCacheReqs], cu[kMaxCacheReqs + 1];
  __shared__ int touched_req[kStepRows], touched_col[kStepRows];
  __shared__ int old[kShort], of_seq[kShort], of_col[kShort], list[kShort];  // the shared ones and their new pages
  __shared__ int sh[kPlan / 64];
  __shared__ int bad;
  const PoolView &c = p.c;
  const int t = threadIdx.x;
  const unsigned used0 = used_bits(c.refs, c.n_pages, t * 16);
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
  for (int64_t base = 0; base < rows; base += kStepRows) {
    const int64_t i0 = base + t * kRowsPer;
    const int here = (int)min(max(rows - i0, (int64_t)0), (int64_t)kRowsPer);
    int pos[kRowsPer + 1] = {}, of[kRowsPer], col[kRowsPer];  // pos: from the row before the thread's first on
    if (p.pos && here > 0) {
      const int32_t *at = p.pos + i0;
      pos[0] = at[i0 > 0 ? -1 : 0];
      if (here == kRowsPer) {
#pragma unroll
        for (int q = 0; q < kRowsPer; q += 4) {
          const i32x4 v = *reinterpret_cast<const i32x4 *>(at + q);
#pragma unroll
          for (int k = 0; k < 4; ++k) pos[1 + q + k] = v[k];
        }
      } else {
#pragma unroll
        for (int k = 0; k < kRowsPer; ++k)
          if (k < here) pos[1 + k] = at[k];
      }
    }
    int b = 0;  // request of the row
    for (int step = kMaxCacheReqs / 2; step; step >>= 1)
      if (b + step < p.n_req && cu[b + step] <= i0) b += step;
    int row0 = cu[b], next = cu[b + 1], L = lens[b];
    unsigned first = 0;
#pragma unroll
    for (int k = 0; k < kRowsPer; ++k) {
      if (k >= here) continue;
      const int i = (int)i0 + k;
      while (next <= i) row0 = next, ++b, next = cu[b + 1], L = lens[b];
      const int at = p.pos ? pos[k + 1] : L - next + i, before = p.pos ? pos[k] : at - 1;
      if (i > row0 && before >= at) bad = 1;  // a page would be listed twice
      if (at >= 0 && at < L && (i == row0 || before < 0 || before / kPage != at / kPage)) first |= 1u << k;
      of[k] = b;
      col[k] = at / kPage;
    }
    int touched;
    int to = block_scan(__builtin_popcount(first), sh, &touched);
#pragma unroll
    for (int k = 0; k < kRowsPer; ++k)
      if ((first >> k) & 1) touched_req[to] = of[k], touched_col[to++] = col[k];
    __syncthreads();
    for (int e0 = 0; e0 < touched; e0 += kPlan) {
      const int e = e0 + t, seq = e < touched ? seqs[touched_req[e]] : 0, col = e < touched ? touched_col[e] : 0;
      const int page = e < touched ? c.table[(int64_t)seq * c.max_seq_pages + col] : -1;
      const bool shared = in_range(page, c.n_pages) && c.refs[page] > 1;
      int total;
      const int64_t r = want + block_scan((int)shared, sh, &total);
      if (shared && r < c.n_pages) {
        p.w.src[r] = page, p.w.seq[r] = seq, p.w.aux[r] = col;
        if (r < kShort) old[r] = page, of_seq[r] = seq, of_col[r] = col;
      }
      want += total;
    }
    __syncthreads();  // the lists of this step are read
  }
  __syncthreads();
  if (bad) {
    if (t == 0) *p.status = -1;
    return;
  }
  // free ids are found before any count changes: none of the old pages is among them
  const int64_t found = walk_free(c.refs, c.n_pages, want, used0, sh, [&](int r, int id) {
    p.w.dst[r] = id;
    if (r < kShort) list[r] = id;
  });
  if (found < want) {
    if (t == 0) *p.status = (int)min(want - found, (int64_t)INT32_MAX);
    return;
  }
  __syncthreads();
  for (int64_t r = t; r < want; r += kPlan) {
    const bool in_lds = r < kShort;
    const int id = in_lds ? list[r] : p.w.dst[r], from = in_lds ? old[r] : p.w.src[r];
    const int seq = in_lds ? of_seq[r] : p.w.seq[r], col = in_lds ? of_col[r] : p.w.aux[r];
    c.table[(int64_t)seq * c.max_seq_pages + col] = id;
    c.refs[id] = 1;
    atomicAdd(&c.refs[from], -1);
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
