// Internal declarations of the paged 8-bit K/V cache (daf_cache_*, daf_pages_*).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "daf.h"

namespace daf {

constexpr int kPage = DAF_PAGE_TOKENS;  // tokens of a page
constexpr int kMaxCacheReqs = 256;      // requests per launch (their prefix sums are a kernel argument)
constexpr int kMaxPageSeqs = 4096;      // sequences per page call (one workgroup plans it)
constexpr int kMaxFree = 1 << 23;       // sequences per call that frees them (a workgroup each)
constexpr int kMinScaleExp = -100;      // exponent of the smallest scale
constexpr int kStoreThreads = 256, kCacheAttnThreads = 256;  // of the workgroups

// Error text of the calling thread (api.hip).
daf_status_t set_error(daf_status_t st, const char *text);

// What the kernels need of a cache; k/v and the scales start at the launch's layer.
struct CacheView {
  unsigned char *k, *v;
  float *k_scale, *v_scale;
  const int32_t *table, *len;
  int32_t n_pages, hkv, d, n_seqs, max_seq_pages;
};

// Tokens of sequence `seq`, as far as its table row reaches; 0 out of range.
__device__ __forceinline__ int seq_len(const int32_t *len, int n_seqs, int max_seq_pages, int seq) {
  if ((unsigned)seq >= (unsigned)n_seqs) return 0;
  return min(max(len[seq], 0), max_seq_pages * kPage);
}

// Row movement between rows [total][hkv][d] and the cache.
struct StoreLaunch {
  CacheView c;
  const int32_t *seq, *pos;  // nullable, at the launch's first request / row
  const void *k, *v;         // rows, at the launch's first row (nullable when reading)
  int32_t n_req;
  int32_t units;             // units of all requests: see unit0
  int32_t per_req;           // units of every request where they are equal, else 0
  int32_t cu[kMaxCacheReqs + 1];     // rows of the launch's requests, from 0
  int32_t unit0[kMaxCacheReqs + 1];  // first unit of each request
};
static_assert(sizeof(StoreLaunch) < 4096, "kernel arguments must fit 4 KiB");
constexpr int kStoreRows = 8;  // rows at positions: rows per unit
hipError_t launch_cache_store(bool write, bool bf16, const StoreLaunch &p, hipStream_t st);

// Attention over the cache.
struct CacheAttnLaunch {
  CacheView c;
  const int32_t *seq, *pos;
  const void *q;
  void *o;
  float *lse;       // nullable; [hq][lse_stride] at the launch's first row
  // n_splits > 1: normalised partial outputs and their LSE. Few rows: [hkv][n_splits]
  // [2][16 pairs] of d values; wide: [row block][hkv][tile of 16 pairs][n_splits] of
  // d / 16 x 64 lanes x 4 values in the order of the accumulators, and of 16 LSEs
  float *part_o, *part_lse;
  int32_t *line;    // few rows: the requests' first pages in the line, their pages, a piece's
  int32_t lse_stride;
  int32_t hq, group;
  int32_t max_len;
  int32_t wide;                   // the kernel for many rows
  int32_t n_splits;               // wide: splits of a row block; else workgroups per head
  int32_t split_pages;            // wide: pages per split
  float scale_log2;               // softmax scale * log2(e)
  int32_t n_req;
  int32_t blocks;                 // row blocks of all requests
  int32_t per_req;                // row blocks of every request where they are equal, else 0
  int32_t cu[kMaxCacheReqs + 1];
  int32_t blk0[kMaxCacheReqs + 1];
};
static_assert(sizeof(CacheAttnLaunch) < 4096, "kernel arguments must fit 4 KiB");
// (row, head) pairs of a row block: few rows, many rows in bf16 and in fp32
constexpr int kCacheAttnRows = 16, kCacheWideRows = 128, kCacheWideRowsF32 = 64;
// Many rows: pages of a split, at least 6 (us a call: fp32 questions over up to 7000 keys
// 15.4, 16.5 with 3, 19.7 with 12; 18 rows of 7 heads over 8000 keys 20.0, 20.9, 25.9).
constexpr int kMinSplitPages = 6;
constexpr size_t kLineBytes = (2 * kMaxCacheReqs + 64) * sizeof(int32_t);
// Few rows: least pages per workgroup, one for each wave (us a call: one sequence of 8000
// keys 11.1 with 4, 13.4 with 8, 17.2 with 16; of 16000 keys 12.0, 13.7, 17.9; with four
// K/V heads pieces grow longer by themselves past 16384 keys).
constexpr int kMinPiece = 4;
hipError_t launch_cache_attn(bool bf16, const CacheAttnLaunch &p, hipStream_t st);

// Page calls.
struct PoolView {
  unsigned char *k, *v;
  float *k_scale, *v_scale;
  int32_t *table, *len, *refs;
  int32_t n_layers, n_pages, hkv, d, n_seqs, max_seq_pages;
};
// Workspace of the page calls: counts, then four lists of n_pages.
struct PageWork {
  int32_t *count;           // [0]: pairs to copy, [1]: whether shared pages follow (fork)
  int32_t *src, *dst;       // the pairs
  int32_t *aux, *seq;       // compact: each page's new id; unshare: the table entries
};
constexpr size_t kPageWorkHead = 256;
struct UnshareLaunch {
  PoolView c;
  PageWork w;
  const int32_t *seq, *pos;
  int32_t *status;
  int32_t n_req;
  int32_t cu[kMaxCacheReqs + 1];
};
hipError_t launch_pages_extend(const PoolView &c, int n, const int32_t *seq, const int32_t *n_new, int32_t *status,
                               hipStream_t st);
hipError_t launch_pages_fork(const PoolView &c, const PageWork &w, int n, const int32_t *src, const int32_t *dst,
                             int32_t *status, hipStream_t st);
hipError_t launch_pages_unshare(const UnshareLaunch &p, hipStream_t st);
hipError_t launch_pages_free(const PoolView &c, int n, const int32_t *seq, hipStream_t st);
hipError_t launch_pages_copy(const PoolView &c, int n, const int32_t *src, const int32_t *dst, hipStream_t st);
hipError_t launch_pages_compact(const PoolView &c, const PageWork &w, int32_t *n_live, hipStream_t st);

}  // namespace daf
