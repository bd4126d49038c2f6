// Entry points of the paged 8-bit K/V cache: argument checks and launch planning.
// Every check that the host can make runs before anything is enqueued.
#include <math.h>
#include <stdarg.h>
#include <stdio.h>

#include <algorithm>

#include "cache.h"

namespace {

using namespace daf;

daf_status_t fail(daf_status_t st, const char *fmt, ...) {
  char text[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(text, sizeof(text), fmt, ap);
  va_end(ap);
  return set_error(st, text);
}

daf_status_t ok() { return set_error(DAF_OK, ""); }

daf_status_t launched(hipError_t e, const char *what) {
  return e == hipSuccess ? ok() : fail(DAF_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

daf_status_t aligned(const void *p, const char *name) {
  if (reinterpret_cast<uintptr_t>(p) % 16 != 0) return fail(DAF_ERR_ALIGNMENT, "%s is not 16-byte aligned", name);
  return DAF_OK;
}

daf_status_t need_ptr(const void *p, const char *name) {
  if (!p) return fail(DAF_ERR_INVALID_ARG, "%s is NULL", name);
  return aligned(p, name);
}

// a launch has less than 2^32 threads
bool fits(int64_t workgroups, int threads) { return workgroups <= (int64_t)UINT32_MAX / threads; }

#define CHECK(expr)                \
  do {                             \
    daf_status_t st_ = (expr);     \
    if (st_ != DAF_OK) return st_; \
  } while (0)

daf_status_t check_cache(const daf_cache_t *c) {
  if (!c) return fail(DAF_ERR_INVALID_ARG, "cache is NULL");
  if (c->n_layers < 1 || c->n_pages < 1 || c->n_kv_heads < 1 || c->n_seqs < 1 || c->max_seq_pages < 1)
    return fail(DAF_ERR_INVALID_ARG, "cache sizes must be >= 1 (layers %d, pages %d, K/V heads %d, sequences %d, pages "
                "per sequence %d)", c->n_layers, c->n_pages, c->n_kv_heads, c->n_seqs, c->max_seq_pages);
  if (c->head_dim != 64 && c->head_dim != 128)
    return fail(DAF_ERR_UNSUPPORTED, "head_dim=%d (supported: 64, 128)", c->head_dim);
  if (c->n_kv_heads > 1024) return fail(DAF_ERR_UNSUPPORTED, "Hkv=%d exceeds 1024", c->n_kv_heads);
  if (c->max_seq_pages >= 1 << 25)
    return fail(DAF_ERR_UNSUPPORTED, "max_seq_pages=%d: a sequence holds less than 2^31 tokens", c->max_seq_pages);
  CHECK(need_ptr(c->k, "cache.k"));
  CHECK(need_ptr(c->v, "cache.v"));
  CHECK(need_ptr(c->k_scale, "cache.k_scale"));
  CHECK(need_ptr(c->v_scale, "cache.v_scale"));
  CHECK(need_ptr(c->table, "cache.table"));
  CHECK(need_ptr(c->len, "cache.len"));
  return need_ptr(c->refs, "cache.refs");
}

daf_status_t check_rows(const daf_cache_rows_t *r) {
  if (!r) return fail(DAF_ERR_INVALID_ARG, "rows is NULL");
  if (r->n < 0) return fail(DAF_ERR_INVALID_ARG, "rows.n=%d must be >= 0", r->n);
  if (!r->cu) return fail(DAF_ERR_INVALID_ARG, "rows.cu must be a non-NULL host array");
  if (r->cu[0] != 0) return fail(DAF_ERR_INVALID_ARG, "rows.cu must start at 0");
  for (int b = 0; b < r->n; ++b)
    if (r->cu[b + 1] < r->cu[b])
      return fail(DAF_ERR_INVALID_ARG, "request %d: rows.cu must be non-decreasing", b);
  CHECK(aligned(r->seq, "rows.seq"));
  return aligned(r->pos, "rows.pos");
}

daf_status_t check_cfg(const daf_attn_cfg_t *cfg, const daf_cache_t *c) {
  if (!cfg) return fail(DAF_ERR_INVALID_ARG, "cfg is NULL");
  if (cfg->n_q_heads < 1 || cfg->n_kv_heads < 1 || cfg->n_q_heads % cfg->n_kv_heads != 0)
    return fail(DAF_ERR_INVALID_ARG, "Hq=%d must be a positive multiple of Hkv=%d", cfg->n_q_heads, cfg->n_kv_heads);
  if (cfg->n_q_heads > 1024) return fail(DAF_ERR_UNSUPPORTED, "Hq=%d exceeds 1024", cfg->n_q_heads);
  if (cfg->n_kv_heads != c->n_kv_heads || cfg->head_dim != c->head_dim)
    return fail(DAF_ERR_INVALID_ARG, "cfg (Hkv=%d, D=%d) does not fit the cache (Hkv=%d, D=%d)", cfg->n_kv_heads,
                cfg->head_dim, c->n_kv_heads, c->head_dim);
  if (cfg->dtype != DAF_BF16 && cfg->dtype != DAF_F32)
    return fail(DAF_ERR_UNSUPPORTED, "dtype=%d (supported: DAF_BF16, DAF_F32)", cfg->dtype);
  if (!(cfg->softmax_scale >= 0.f) || !isfinite(cfg->softmax_scale))
    return fail(DAF_ERR_INVALID_ARG, "softmax_scale must be finite and >= 0");
  return DAF_OK;
}

daf_status_t check_layer(const daf_cache_t *c, int32_t layer) {
  if (layer < 0 || layer >= c->n_layers)
    return fail(DAF_ERR_INVALID_ARG, "layer=%d is not in [0, %d)", layer, c->n_layers);
  return DAF_OK;
}

CacheView view(const daf_cache_t *c, int32_t layer) {
  const size_t page = (size_t)c->n_kv_heads * kPage * c->head_dim, pages = (size_t)layer * c->n_pages;
  CacheView v{};
  v.k = static_cast<unsigned char *>(c->k) + pages * page;
  v.v = static_cast<unsigned char *>(c->v) + pages * page;
  v.k_scale = c->k_scale + pages * c->n_kv_heads;
  v.v_scale = c->v_scale + pages * c->n_kv_heads;
  v.table = c->table;
  v.len = c->len;
  v.n_pages = c->n_pages;
  v.hkv = c->n_kv_heads;
  v.d = c->head_dim;
  v.n_seqs = c->n_seqs;
  v.max_seq_pages = c->max_seq_pages;
  return v;
}

PoolView pool(const daf_cache_t *c) {
  PoolView v{};
  v.k = static_cast<unsigned char *>(c->k);
  v.v = static_cast<unsigned char *>(c->v);
  v.k_scale = c->k_scale;
  v.v_scale = c->v_scale;
  v.table = c->table;
  v.len = c->len;
  v.refs = c->refs;
  v.n_layers = c->n_layers;
  v.n_pages = c->n_pages;
  v.hkv = c->n_kv_heads;
  v.d = c->head_dim;
  v.n_seqs = c->n_seqs;
  v.max_seq_pages = c->max_seq_pages;
  return v;
}

const char *rows_at(const void *p, int64_t row, size_t row_bytes) {
  return p ? static_cast<const char *>(p) + row * row_bytes : nullptr;
}

// Prefix sums of a launch of the requests b0 .. b0 + n: first[i] in units of f(rows),
// and the units of every request where they are equal (else 0). -1: too many.
template <typename F>
int fill(const daf_cache_rows_t *r, int b0, int n, int32_t *cu, int32_t *first, int32_t *per, F f) {
  int64_t at = 0;
  *per = 0;
  bool equal = true;
  for (int i = 0; i < n; ++i) {
    cu[i] = r->cu[b0 + i] - r->cu[b0];
    first[i] = (int32_t)at;
    const int64_t units = f(r->cu[b0 + i + 1] - r->cu[b0 + i]);
    if (i == 0) *per = (int32_t)units;
    equal = equal && units == *per;
    at += units;
    if (at > INT32_MAX) return -1;
  }
  cu[n] = r->cu[b0 + n] - r->cu[b0];
  first[n] = (int32_t)at;
  if (!equal) *per = 0;
  return (int)at;
}

daf_status_t store(bool write, const daf_attn_cfg_t *cfg, const daf_cache_t *c, int32_t layer,
                   const daf_cache_rows_t *rows, const void *k, const void *v, hipStream_t stream) {
  CHECK(check_cache(c));
  CHECK(check_cfg(cfg, c));
  CHECK(check_layer(c, layer));
  CHECK(check_rows(rows));
  const int total = rows->cu[rows->n];
  if (total == 0 || (!write && !k && !v)) return ok();
  if (write || k) CHECK(need_ptr(k, "k"));
  if (write || v) CHECK(need_ptr(v, "v"));
  const bool bf16 = cfg->dtype == DAF_BF16;
  const size_t row_bytes = (size_t)c->n_kv_heads * c->head_dim * (bf16 ? 2 : 4);
  auto units_of = [&](int64_t n) { return n == 0 ? 0 : rows->pos ? (n + kStoreRows - 1) / kStoreRows : (n + 62) / 64 + 1; };
  // every launch's grid is checked before the first launch
  for (int pass = 0; pass < 2; ++pass)
    for (int b0 = 0; b0 < rows->n; b0 += kMaxCacheReqs) {
      StoreLaunch p;
      p.c = view(c, layer);
      p.n_req = std::min(kMaxCacheReqs, rows->n - b0);
      p.units = fill(rows, b0, p.n_req, p.cu, p.unit0, &p.per_req, units_of);
      if (p.units < 0 || !fits((int64_t)p.units * c->n_kv_heads * 2, kStoreThreads))
        return fail(DAF_ERR_UNSUPPORTED, "%d rows of %d heads are too many for one call", total, c->n_kv_heads);
      if (pass == 0 || p.units == 0) continue;
      const int64_t row0 = rows->cu[b0];
      // without a list, request b0 + i is sequence b0 + i: the view starts at b0
      p.seq = rows->seq ? rows->seq + b0 : nullptr;
      if (!rows->seq) {
        if (b0 >= c->n_seqs) p.c.n_seqs = 0;
        else p.c.n_seqs -= b0, p.c.table += (int64_t)b0 * c->max_seq_pages, p.c.len += b0;
      }
      p.pos = rows->pos ? rows->pos + row0 : nullptr;
      p.k = rows_at(k, row0, row_bytes);
      p.v = rows_at(v, row0, row_bytes);
      const hipError_t e = launch_cache_store(write, bf16, p, stream);
      if (e != hipSuccess) return launched(e, write ? "cache write launch" : "cache read launch");
    }
  return ok();
}

// ---- attention ------------------------------------------------------------------
struct AttnPlan {
  int wide, block_rows;  // which kernel; (row, head) pairs of its row blocks
  int n_splits, split_pages;
  size_t lse_bytes, total;  // workspace: LSEs (and few rows' line), then partial outputs
};

int64_t row_blocks(const daf_attn_cfg_t *cfg, int64_t n, int block_rows) {
  return (n * (cfg->n_q_heads / cfg->n_kv_heads) + block_rows - 1) / block_rows;
}
// (row, head) pairs with a place of their own among the wide kernel's partial results
size_t wide_pairs(const daf_attn_cfg_t *cfg, int64_t blocks, int block_rows) {
  return (size_t)blocks * cfg->n_kv_heads * block_rows;
}

// Kernel and its splits, from the sizes that the host knows.
AttnPlan plan_attn(const daf_attn_cfg_t *cfg, const daf_cache_t *c, const daf_cache_rows_t *rows, int32_t max_len) {
  AttnPlan a{};
  int64_t most = 0, blocks = 0, least = INT32_MAX;
  for (int b = 0; b < rows->n; ++b) most = std::max<int64_t>(most, rows->cu[b + 1] - rows->cu[b]);
  // Up to four of few rows' blocks read a page from the caches as often before the wide
  // kernel's larger tiles pay (7 heads on one, us a call, few rows and wide: 8000 keys, 9
  // rows 17.4 and 19.7, 18 rows 21.3 and 20.0; 131072 keys 58.0 and 56.9, 103 and 57.4).
  a.wide = most * (cfg->n_q_heads / cfg->n_kv_heads) > 4 * kCacheAttnRows;
  a.block_rows = !a.wide ? kCacheAttnRows : cfg->dtype == DAF_BF16 ? kCacheWideRows : kCacheWideRowsF32;
  for (int b = 0; b < rows->n; ++b) {
    const int64_t n = row_blocks(cfg, rows->cu[b + 1] - rows->cu[b], a.block_rows);
    blocks += n;
    if (n > 0) least = std::min(least, n);  // row blocks of a request
  }
  const int64_t pages = std::max<int64_t>(1, ((int64_t)max_len + kPage - 1) / kPage);
  const int64_t jobs = std::max<int64_t>(1, blocks * c->n_kv_heads);
  if (a.wide) {
    // Two workgroups per CU, at once (128 rows of 7 heads on each of 4 over 32896 keys, us of
    // kernel and join by workgroups in all: 256 86.7 + 5.3, 512 71.8 + 7.5, 768 75.1 + 9.5,
    // 1024 76.4 + 12.0).
    // More row blocks than that still gain from splits of 64 pages, which end more evenly,
    // up to 4096 workgroups, whose partial results are at most 271 MB (4915 rows of 28 heads
    // on 4 over 32768 keys, ms and MiB by the bound: 4096 2.18 and 203, 16384 2.25 and 542;
    // 4096 rows over 131072 keys 7.3 and 226, 7.6 and 1016; 32768 rows over 32768 keys 10.8
    // and 0, 10.6 and 903). A request of few row blocks may be the only long one, and has to
    // fill the device by itself: up to 8192 (10 rows on each of 128 sequences, of which one
    // has 131072 keys and the others 1000, us and MiB: 4096 531 and 258, 8192 384 and 516,
    // 16384 320 and 1032).
    const int64_t alone = std::min(8192 / jobs, 512 / (least * c->n_kv_heads));
    int64_t splits = std::max(512 / jobs, std::min((pages + 63) / 64, std::max(4096 / jobs, alone)));
    splits = std::max<int64_t>(splits, 1);
    splits = std::min(splits, (pages + kMinSplitPages - 1) / kMinSplitPages);
    a.split_pages = (int)((pages + splits - 1) / splits);
    a.n_splits = (int)((pages + a.split_pages - 1) / a.split_pages);
  } else {
    // One workgroup per row block and head, or workgroups per head on the line of all row
    // blocks' pages. One takes up to 16 pages as soon as the line and its join do (us, one
    // and the line: a row of 1024 keys 11.0 and 7.8 + 3.6, of 1500 keys 13.9 and 7.9 + 3.5).
    // With more of them the device fills without the line's ends inside of workgroups
    // (ragged rows by 4 heads over up to 2000 keys: 24 rows 16.6 and 15.1 + 4.0, 64 rows
    // 18.8 and 22.9 + 5.3, 64 in fp32 22.0 and 31.0 + 4.9; 64 rows over up to 4000 keys
    // 33.9 and 35.1 + 5.4): up to a third as many pages as workgroups, and 64, of which a
    // long sequence among 191 short ones takes 31.6 us (22.9 on the line).
    a.n_splits = 1;
    if (pages > std::clamp<int64_t>(jobs / 3, 16, 64)) {
      const int64_t line = std::min<int64_t>(blocks, INT32_MAX) * pages;
      // Two workgroups per CU hide the ends of requests behind each other's loads; within
      // one request one is enough, with half as much to join (bf16 of 128 features, us a call
      // with 512 and 256: 32 ragged sequences 30.7 and 33.0, two of 30000 keys 20.4 and 21.3;
      // one of 131072 keys 32.6 and 31.9, four rows of it 44.0 and 36.2). fp32 of 128
      // features has one (32 ragged sequences 40.3 and 36.2).
      const bool two = rows->n > 1 && (cfg->dtype == DAF_BF16 || cfg->head_dim == 64);
      const int64_t wgs = (two ? 512 : 256) / c->n_kv_heads;
      a.n_splits = (int)std::max<int64_t>(2, std::min<int64_t>(wgs, (line + kMinPiece - 1) / kMinPiece));
    }
  }
  if (a.n_splits > 1) {
    const size_t pairs = a.wide ? wide_pairs(cfg, blocks, a.block_rows) * a.n_splits
                                : (size_t)a.n_splits * c->n_kv_heads * 2 * kCacheAttnRows;
    a.lse_bytes = (pairs * sizeof(float) + 255) / 256 * 256 + (a.wide ? 0 : kLineBytes);
    a.total = a.lse_bytes + pairs * cfg->head_dim * sizeof(float);
  }
  return a;
}

daf_status_t check_attn(const daf_attn_cfg_t *cfg, const daf_cache_t *c, const daf_cache_rows_t *rows, int32_t max_len) {
  CHECK(check_cache(c));
  CHECK(check_cfg(cfg, c));
  CHECK(check_rows(rows));
  if (max_len < 0 || (int64_t)max_len > (int64_t)c->max_seq_pages * kPage)
    return fail(DAF_ERR_INVALID_ARG, "max_len=%d is not in [0, %lld]", max_len,
                (long long)c->max_seq_pages * kPage);
  if ((int64_t)rows->cu[rows->n] * cfg->n_q_heads > INT32_MAX)
    return fail(DAF_ERR_UNSUPPORTED, "%d rows of %d heads are too many for one call", rows->cu[rows->n],
                cfg->n_q_heads);
  return DAF_OK;
}

daf_status_t attn(const daf_attn_cfg_t *cfg, const daf_cache_t *c, int32_t layer, const daf_cache_rows_t *rows,
                  int32_t max_len, const void *q, void *o, float *lse, void *workspace, size_t ws_bytes,
                  hipStream_t stream) {
  CHECK(check_attn(cfg, c, rows, max_len));
  CHECK(check_layer(c, layer));
  const int total = rows->cu[rows->n];
  if (total == 0) return ok();
  CHECK(need_ptr(q, "q"));
  CHECK(need_ptr(o, "o"));
  CHECK(aligned(lse, "lse"));
  const AttnPlan a = plan_attn(cfg, c, rows, max_len);
  if (a.total > 0) {
    if (!workspace || ws_bytes < a.total)
      return fail(DAF_ERR_WORKSPACE, "workspace of %zu bytes needed, %zu given", a.total, workspace ? ws_bytes : 0);
    CHECK(aligned(workspace, "workspace"));
  }
  const bool bf16 = cfg->dtype == DAF_BF16;
  const size_t row_bytes = (size_t)cfg->n_q_heads * cfg->head_dim * (bf16 ? 2 : 4);
  const float scale = cfg->softmax_scale > 0.f ? cfg->softmax_scale : 1.f / sqrtf((float)cfg->head_dim);
  for (int pass = 0; pass < 2; ++pass) {
    int64_t block0 = 0;
    for (int b0 = 0; b0 < rows->n; b0 += kMaxCacheReqs) {
      CacheAttnLaunch p;
      p.c = view(c, layer);
      p.n_req = std::min(kMaxCacheReqs, rows->n - b0);
      p.blocks = fill(rows, b0, p.n_req, p.cu, p.blk0, &p.per_req, 
                      [&](int64_t n) { return row_blocks(cfg, n, a.block_rows); });
      const int64_t pages = ((int64_t)max_len + kPage - 1) / kPage;
      const int64_t jobs = (int64_t)p.blocks * c->n_kv_heads, pairs = (int64_t)p.cu[p.n_req] * cfg->n_q_heads;
      // the grids of the kernel and of the join, and few rows' line of pages with a piece more
      const bool grids = a.wide ? fits(jobs * a.n_splits + 8, kCacheAttnThreads) &&
                                      (a.n_splits == 1 || fits(jobs * (a.block_rows / 16), cfg->head_dim * 4))
                                : fits(jobs, kCacheAttnThreads) && fits(pairs, kCacheAttnThreads);
      if (p.blocks < 0 || !grids || (!a.wide && (int64_t)p.blocks * std::max<int64_t>(pages, 1) > INT32_MAX / 2))
        return fail(DAF_ERR_UNSUPPORTED, "%d rows over %d keys are too many for one call", total, max_len);
      if (pass == 0 || p.blocks == 0) continue;
      const int64_t row0 = rows->cu[b0];
      p.seq = rows->seq ? rows->seq + b0 : nullptr;
      if (!rows->seq) {
        if (b0 >= c->n_seqs) p.c.n_seqs = 0;
        else p.c.n_seqs -= b0, p.c.table += (int64_t)b0 * c->max_seq_pages, p.c.len += b0;
      }
      p.pos = rows->pos ? rows->pos + row0 : nullptr;
      p.q = rows_at(q, row0, row_bytes);
      p.o = const_cast<char *>(rows_at(o, row0, row_bytes));
      p.lse = lse ? lse + row0 : nullptr;
      p.lse_stride = total;
      // few rows: each launch's join is done with the places before the next one's kernel
      const size_t pair0 = a.wide ? wide_pairs(cfg, block0, a.block_rows) * a.n_splits : 0;
      p.part_lse = a.total ? static_cast<float *>(workspace) + pair0 : nullptr;
      p.part_o = a.total ? reinterpret_cast<float *>(static_cast<char *>(workspace) + a.lse_bytes) +
                               pair0 * cfg->head_dim : nullptr;
      p.line = a.total && !a.wide ? reinterpret_cast<int32_t *>(static_cast<char *>(workspace) + a.lse_bytes - kLineBytes)
                                  : nullptr;
      p.hq = cfg->n_q_heads;
      p.group = cfg->n_q_heads / cfg->n_kv_heads;
      p.max_len = max_len;
      p.wide = a.wide;
      p.n_splits = a.n_splits;
      p.split_pages = a.split_pages;
      p.scale_log2 = scale * 1.4426950408889634f;
      const hipError_t e = launch_cache_attn(bf16, p, stream);
      if (e != hipSuccess) return launched(e, "cache attention launch");
      block0 += p.blocks;
    }
  }
  return ok();
}

// ---- page calls -------------------------------------------------------------------
size_t page_list_bytes(const daf_cache_t *c) { return ((size_t)c->n_pages * sizeof(int32_t) + 255) / 256 * 256; }
size_t page_ws_bytes(const daf_cache_t *c) { return kPageWorkHead + 4 * page_list_bytes(c); }

daf_status_t page_work(const daf_cache_t *c, void *ws, size_t ws_bytes, PageWork &w) {
  if (!ws || ws_bytes < page_ws_bytes(c))
    return fail(DAF_ERR_WORKSPACE, "workspace of %zu bytes needed, %zu given", page_ws_bytes(c), ws ? ws_bytes : 0);
  CHECK(aligned(ws, "workspace"));
  char *p = static_cast<char *>(ws);
  const size_t list = page_list_bytes(c);
  w.count = reinterpret_cast<int32_t *>(p);
  w.src = reinterpret_cast<int32_t *>(p + kPageWorkHead);
  w.dst = reinterpret_cast<int32_t *>(p + kPageWorkHead + list);
  w.aux = reinterpret_cast<int32_t *>(p + kPageWorkHead + 2 * list);
  w.seq = reinterpret_cast<int32_t *>(p + kPageWorkHead + 3 * list);
  return DAF_OK;
}

daf_status_t check_count(int32_t n, int32_t most) {
  if (n < 0) return fail(DAF_ERR_INVALID_ARG, "n=%d must be >= 0", n);
  if (n > most) return fail(DAF_ERR_UNSUPPORTED, "n=%d exceeds %d", n, most);
  return DAF_OK;
}

}  // namespace

extern "C" {

daf_status_t daf_cache_write(const daf_attn_cfg_t *cfg, const daf_cache_t *cache, int32_t layer,
                             const daf_cache_rows_t *rows, const void *k, const void *v, hipStream_t stream) {
  return store(true, cfg, cache, layer, rows, k, v, stream);
}

daf_status_t daf_cache_read(const daf_attn_cfg_t *cfg, const daf_cache_t *cache, int32_t layer,
                            const daf_cache_rows_t *rows, void *k, void *v, hipStream_t stream) {
  return store(false, cfg, cache, layer, rows, k, v, stream);
}

size_t daf_cache_attn_workspace_size(const daf_attn_cfg_t *cfg, const daf_cache_t *cache, const daf_cache_rows_t *rows,
                                     int32_t max_len) {
  if (check_attn(cfg, cache, rows, max_len) != DAF_OK || rows->cu[rows->n] == 0) return 0;
  return plan_attn(cfg, cache, rows, max_len).total;
}

daf_status_t daf_cache_attn(const daf_attn_cfg_t *cfg, const daf_cache_t *cache, int32_t layer,
                            const daf_cache_rows_t *rows, int32_t max_len, const void *q, void *o, float *lse,
                            void *workspace, size_t ws_bytes, hipStream_t stream) {
  return attn(cfg, cache, layer, rows, max_len, q, o, lse, workspace, ws_bytes, stream);
}

size_t daf_pages_workspace_size(const daf_cache_t *cache) {
  return check_cache(cache) == DAF_OK ? page_ws_bytes(cache) : 0;
}

daf_status_t daf_pages_extend(const daf_cache_t *cache, int32_t n, const int32_t *seq, const int32_t *n_new,
                              int32_t *status, hipStream_t stream) {
  CHECK(check_cache(cache));
  CHECK(check_count(n, kMaxPageSeqs));
  CHECK(aligned(seq, "seq"));
  CHECK(aligned(n_new, "n_new"));
  CHECK(need_ptr(status, "status"));
  return launched(launch_pages_extend(pool(cache), n, seq, n_new, status, stream), "page extend launch");
}

daf_status_t daf_pages_fork(const daf_cache_t *cache, int32_t n, const int32_t *src, const int32_t *dst,
                            int32_t *status, void *workspace, size_t ws_bytes, hipStream_t stream) {
  CHECK(check_cache(cache));
  CHECK(check_count(n, kMaxPageSeqs));
  if (n > 0) {
    CHECK(need_ptr(src, "src"));
    CHECK(need_ptr(dst, "dst"));
  }
  CHECK(need_ptr(status, "status"));
  PageWork w;
  CHECK(page_work(cache, workspace, ws_bytes, w));
  return launched(launch_pages_fork(pool(cache), w, n, src, dst, status, stream), "page fork launch");
}

daf_status_t daf_pages_unshare(const daf_cache_t *cache, const daf_cache_rows_t *rows, int32_t *status,
                               void *workspace, size_t ws_bytes, hipStream_t stream) {
  CHECK(check_cache(cache));
  CHECK(check_rows(rows));
  CHECK(check_count(rows->n, kMaxCacheReqs));
  CHECK(need_ptr(status, "status"));
  UnshareLaunch p;
  CHECK(page_work(cache, workspace, ws_bytes, p.w));
  p.c = pool(cache);
  p.seq = rows->seq;
  p.pos = rows->pos;
  p.status = status;
  p.n_req = rows->n;
  for (int b = 0; b <= rows->n; ++b) p.cu[b] = rows->cu[b];
  return launched(launch_pages_unshare(p, stream), "page unshare launch");
}

daf_status_t daf_pages_free(const daf_cache_t *cache, int32_t n, const int32_t *seq, hipStream_t stream) {
  CHECK(check_cache(cache));
  CHECK(check_count(n, kMaxFree));
  CHECK(aligned(seq, "seq"));
  if (n == 0) return ok();
  return launched(launch_pages_free(pool(cache), n, seq, stream), "page free launch");
}

daf_status_t daf_pages_copy(const daf_cache_t *cache, int32_t n, const int32_t *src, const int32_t *dst,
                            hipStream_t stream) {
  CHECK(check_cache(cache));
  if (n < 0) return fail(DAF_ERR_INVALID_ARG, "n=%d must be >= 0", n);
  if (n == 0) return ok();
  CHECK(need_ptr(src, "src"));
  CHECK(need_ptr(dst, "dst"));
  return launched(launch_pages_copy(pool(cache), n, src, dst, stream), "page copy launch");
}

daf_status_t daf_pages_compact(const daf_cache_t *cache, int32_t *n_live, void *workspace, size_t ws_bytes,
                               hipStream_t stream) {
  CHECK(check_cache(cache));
  CHECK(need_ptr(n_live, "n_live"));
  PageWork w;
  CHECK(page_work(cache, workspace, ws_bytes, w));
  return launched(launch_pages_compact(pool(cache), w, n_live, stream), "page compact launch");
}

}  // extern "C"
