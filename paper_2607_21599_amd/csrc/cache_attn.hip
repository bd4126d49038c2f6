// Attention over the paged 8-bit K/V cache (daf_cache_attn).
//
// Per head h of a row with q, over the keys 0 .. limit of its sequence:
//   s_t = q . k_t * scale,  o = sum_t exp(s_t - m) v_t / sum_t exp(s_t - m)
// with one pass over the pages: a running maximum m and sum per row, the output
// rescaled where m grows (fp32). The G query heads of a K/V head share its pages,
// so a row block is 16 (row, head) pairs of one K/V head.
//
// Matrix instructions (both kernels):
//  * e4m3 codes become bf16 exactly, and times their scale (a power of two) by the
//    same conversion instruction, so no multiplication carries the scales.
//  * S^T = K Q^T and O^T += V^T P^T on v_mfma_f32_16x16x32_bf16. With the rows of K
//    taken in the order key(t, m) = 16 (m / 4) + 4 t + m % 4 for block t and row m
//    of the operand, a lane of group g (lane / 16) ends up with the probabilities
//    of keys 16 g .. 16 g + 15 of row lane % 16, which is how the second product
//    wants them, and V^T, stored transposed, is read as 16 consecutive keys.
//  * Weights enter the product in more bits than a bf16 output shows (one bf16 value of 8
//    bits each makes the output's error 1.4 times that of its own rounding). Few rows: two
//    bf16 terms, 16 bits, whose second products the loads of pages hide for the most part
//    (131072 keys 32.0 us for 30.8 with one term, 32 ragged sequences 27.1 for 25.0). Many
//    rows: one fp16 value, 11 bits, with the codes in fp16 too; see HalfWeights. (That in
//    the few rows' kernel, with the terms beside it, needs more registers than it has.)
//    (8-bit scores are not exact enough: the 8-bit product keeps about 13 bits of a small
//    term beside a large one.)
//  * fp32: q and the probabilities enter as three bf16 terms each.
//
// Few rows: a wave takes a page (64 keys) of one head at a time from memory to
// registers, in the layout that the matrix instructions take, 16 bytes per lane and
// load, with the next page's loads in flight and without LDS; the waves of a workgroup
// take its pages in turn and join their (m, sum, O) through LDS. Bound by the pages'
// bytes: 131072 keys of 4 heads of 128 (134 MB) in 32 us, 4.2 TB/s; a short sequence
// by what one CU keeps in flight (777 keys 10.5 us, 64 keys 4.7; 8 waves or 4).
// Many rows: below. What workgroups share of a row block is joined by a second kernel
// (4 to 5 us, most of it its launch).
#include "cache_attn.h"

namespace daf {
namespace {

__device__ __forceinline__ Request find_request(const CacheAttnLaunch &p, int blk) {
  Request r;
  int b = 0;
  if (p.per_req) {
    b = blk / p.per_req;
    r.block = blk - b * p.per_req;
  } else {
    b = find_in(p.blk0, p.n_req, blk);
    r.block = blk - p.blk0[b];
  }
  r.b = b;
  r.row0 = p.cu[b];
  r.n = p.cu[b + 1] - r.row0;
  const int seq = p.seq ? p.seq[b] : b;
  r.L = min(seq_len(p.c.len, p.c.n_seqs, p.c.max_seq_pages, seq), p.max_len);
  r.pages = p.c.table + (int64_t)((unsigned)seq < (unsigned)p.c.n_seqs ? seq : 0) * p.c.max_seq_pages;
  return r;
}

// Short sequences: a workgroup per row block and head.
template <bool BF16, int D>
__global__ __launch_bounds__(kThreads, 2) void cache_attn_kernel(const CacheAttnLaunch p) {
  __shared__ FewShared<D> sh;
  const Request r = find_request(p, blockIdx.x % p.blocks);
  few_rows<BF16, D>(p, sh, r, blockIdx.x / p.blocks, 0, INT32_MAX, -1);
}

// fp32's terms of 128 features need more than 256 registers: one workgroup per CU, with
// whole pages in flight, for two whose registers spill (131072 keys, a row for 28
// heads: 30.4 us for 45.3).
template <bool BF16, int D>
constexpr int kLineWgs = BF16 || D == 64 ? 2 : 1;
template <bool BF16, int D>
__global__ __launch_bounds__(kThreads, (kLineWgs<BF16, D>)) void cache_line_kernel(const CacheAttnLaunch p) {
  __shared__ FewShared<D> sh;
  line_job<BF16, D>(p, sh, blockIdx.x % p.c.hkv, blockIdx.x / p.c.hkv);
}

// Join the pieces of one (row, head): o = sum_s e^(lse_s - lse) o_s. Groups of D / 4
// lanes take the pieces in turn, four in flight, and join their sums through LDS.
template <bool BF16, int D>
__global__ __launch_bounds__(kThreads) void cache_line_join_kernel(const CacheAttnLaunch p) {
  constexpr int LP = D / 4, GROUPS = kThreads / LP;
  __shared__ f32x4 sh_o[GROUPS][LP];
  __shared__ float sh_m[GROUPS], sh_l[GROUPS];
  const int t = threadIdx.x, g = t / LP, c = t % LP;
  const int row = blockIdx.x / p.hq, head = blockIdx.x % p.hq;
  const int piece = p.line[2 * kMaxCacheReqs];
  const int b = find_in(p.cu, p.n_req, row);
  const int h = head / p.group, pair = (row - p.cu[b]) * p.group + head % p.group;
  const int pages = p.line[kMaxCacheReqs + b], from = p.line[b] + pair / kRows * pages;
  const int k0 = from / piece, k1 = (from + pages - 1) / piece;
  if (k0 == k1) return;  // in one piece: written already
  const int n = k1 - k0 + 1;
  // piece s of the n: the first one's place is its workgroup's second
  auto at = [&](int s) { return (size_t)((h * p.n_splits + k0 + s) * 2 + (s == 0)) * kRows + pair % kRows; };
  float m = -INFINITY, l = 0.f;
  f32x4 x = {};
  for (int s0 = g; s0 < n; s0 += 4 * GROUPS) {
    float lse[4];
    f32x4 y[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int s = s0 + j * GROUPS;
      lse[j] = s < n ? p.part_lse[at(s)] : -INFINITY;
      y[j] = s < n ? *reinterpret_cast<const f32x4 *>(p.part_o + at(s) * D + c * 4) : f32x4{};
    }
    const float to = fmaxf(m, fmaxf(fmaxf(lse[0], lse[1]), fmaxf(lse[2], lse[3])));
    const float ref = to == -INFINITY ? 0.f : to;  // a row that sees no key there, or NaN
    const float a = __expf(m - ref);
    m = to;
    l *= a;
    x *= a;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float w = __expf(lse[j] - ref);
      l += w;
      x += w * y[j];
    }
  }
  sh_o[g][c] = x;
  if (c == 0) sh_m[g] = m, sh_l[g] = l;
  __syncthreads();
  if (g) return;
  for (int k = 1; k < GROUPS; ++k) m = fmaxf(m, sh_m[k]);
  const float ref = m == -INFINITY ? 0.f : m;
  l = 0.f;
  x = f32x4{};
  for (int k = 0; k < GROUPS; ++k) {
    const float w = __expf(sh_m[k] - ref);
    l += w * sh_l[k];
    x += w * sh_o[k][c];
  }
  const float inv = over(l);
  const float y[4] = {x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv};
  store_out<BF16>(p, row, head, c * 4, y, D);
  if (c == 0 && p.lse) p.lse[(size_t)head * p.lse_stride + row] = l == 0.f ? -INFINITY : m + __logf(l);
}
// The rows of a block as far as their sequence goes.
template <int MT>
struct LenRows {
  static constexpr bool kKnown = false;
  static constexpr int PAIRS = kWaves * 16 * MT;  // of a row block
  const CacheAttnLaunch &p;
  const Request &r;
  int split, pg0;
  __device__ __forceinline__ bool exact() const { return false; }
  __device__ __forceinline__ bool empty() const { return split > 0 && pg0 >= (r.L + kPage - 1) / kPage; }
  __device__ __forceinline__ int limit(int row) const { return row_limit(p, r, row); }
  __device__ __forceinline__ int seen() const {
    const int lane = threadIdx.x & 63, total = r.n * p.group;
    int last = -1;  // last key that a row of the block sees
    if (p.pos) {
#pragma unroll
      for (int i = 0; i < PAIRS; i += 64)
        last = max(last, row_limit(p, r, min(r.block * PAIRS + i + lane, total - 1) / p.group));
#pragma unroll
      for (int m = 32; m; m >>= 1) last = max(last, __shfl_xor(last, m));
    } else {
      last = row_limit(p, r, (min((r.block + 1) * PAIRS, total) - 1) / p.group);
    }
    return __builtin_amdgcn_readfirstlane((last >> 6) + 1);
  }
};

template <bool BF16, int D, int MT>
__global__ __launch_bounds__(kThreads, D == 64 ? 3 : 2) void cache_wide_kernel(const CacheAttnLaunch p) {
  using W = Wide<BF16, D, MT>;
  constexpr int DB = W::DB;
  __shared__ __align__(16) unsigned char lds[kStages * W::PAGE_BYTES];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n16 = lane & 15, quad = lane >> 4;
  // The row blocks of one (head, split) read the same pages: neighbours, on one XCD. These
  // groups go to the XCDs in turn, first splits first, so that every XCD has work where
  // sequences are far shorter than max_len (128 sequences of 8192 keys planned for 131072,
  // 10 rows each: 570 us; with a run of groups for each XCD, of which the first has all the
  // keys, 1910; planned for 8192 keys 358); the last few in equal shares.
  const int groups = p.c.hkv * p.n_splits, turns = groups / kXcdCount;
  const int xcd = blockIdx.x % kXcdCount, at_xcd = blockIdx.x / kXcdCount;
  int g = at_xcd / p.blocks * kXcdCount + xcd, blk = at_xcd % p.blocks;
  if (at_xcd >= turns * p.blocks) {
    const int rest = groups % kXcdCount * p.blocks, share = (rest + kXcdCount - 1) / kXcdCount;
    const int k = at_xcd - turns * p.blocks, i = xcd * share + k;
    if (k >= share || i >= rest) return;
    g = turns * kXcdCount + i / p.blocks;
    blk = i % p.blocks;
  }
  const int h = g % p.c.hkv, split = g / p.c.hkv;
  const Request r = find_request(p, blk);
  const int pg0 = split * p.split_pages;
  LenRows<MT> rows{p, r, split, pg0};
  W w;
  float unit;
  if (!wide_rows<BF16, D, MT>(p, lds, r, h, pg0, p.split_pages, rows, w, unit)) return;  // the join leaves this split out
  const int total = r.n * p.group;

  // results
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    const float l = row_sum(w.l[mt]), inv = over(l);
    const float lse = l == 0.f ? -INFINITY : (w.m[mt] + log2f(l)) * kLn2;
    const int tile = (r.block * kWaves + wave) * MT + mt, idx = tile * 16 + n16;
    if (p.n_splits > 1) {
      const size_t part = (((size_t)(blk * p.c.hkv + h) * kWaves + wave) * MT + mt) * p.n_splits + split;
      if (quad == 0) p.part_lse[part * 16 + n16] = lse;
#pragma unroll
      for (int db = 0; db < DB; ++db)
        *reinterpret_cast<f32x4 *>(p.part_o + (part * DB + db) * 256 + lane * 4) = w.o[mt][db] * inv * unit;
    } else if (idx < total) {
      const int row = r.row0 + idx / p.group, head = h * p.group + idx % p.group;
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        const f32x4 x = w.o[mt][db] * inv * unit;
        const float y[4] = {x[0], x[1], x[2], x[3]};
        store_out<BF16>(p, row, head, db * 16 + quad * 4, y, D);
      }
      if (quad == 0 && p.lse) p.lse[(size_t)head * p.lse_stride + row] = lse;
    }
  }
}
// Join the splits of one tile of 16 pairs: a wave per 16 features, a workgroup of its own
// (few tiles of many splits are read by the whole device), a lane with the same pair and
// features as in the kernel above, 8 splits in flight. The first ones do not
// wait for the length, which says how many splits hold keys; those beyond it were not
// written and are left out.
template <bool BF16, int D, int MT>
__global__ __launch_bounds__(64) void cache_wide_join_kernel(const CacheAttnLaunch p) {
  constexpr int DB = D / 16, FLIGHT = 8;
  const int lane = threadIdx.x, n16 = lane & 15, quad = lane >> 4;
  const int db = blockIdx.x % DB, job = blockIdx.x / DB;
  const int tile = job % (kWaves * MT), rest = job / (kWaves * MT);
  const int h = rest % p.c.hkv, blk = rest / p.c.hkv;
  const size_t part = (size_t)job * p.n_splits;
  const float *lses = p.part_lse + part * 16 + n16, *os = p.part_o + (part * DB + db) * 256 + lane * 4;
  float lse[FLIGHT];
  f32x4 y[FLIGHT];
  auto load = [&](int s0) {
#pragma unroll
    for (int j = 0; j < FLIGHT; ++j) {
      const int s = min(s0 + j, p.n_splits - 1);
      lse[j] = lses[s * 16];
      y[j] = *reinterpret_cast<const f32x4 *>(os + (size_t)s * (DB * 256));
    }
  };
  load(0);
  const Request r = find_request(p, blk);
  const int idx = (r.block * kWaves * MT + tile) * 16 + n16, total = r.n * p.group;
  const int pages = (r.L + kPage - 1) / kPage;
  const int n = max(1, (pages + p.split_pages - 1) / p.split_pages);  // splits that hold keys
  float m = -INFINITY, l = 0.f;
  f32x4 x = {};
  for (int s0 = 0;;) {
    float to = m;
#pragma unroll
    for (int j = 0; j < FLIGHT; ++j)
      if (s0 + j < n) to = fmaxf(to, lse[j]);
    const float ref = to == -INFINITY ? 0.f : to;  // a row that sees no key yet
    const float a = __expf(m - ref);
    m = to;
    l *= a;
    x *= a;
#pragma unroll
    for (int j = 0; j < FLIGHT; ++j)
      if (s0 + j < n) {
        const float w = __expf(lse[j] - ref);
        l += w;
        x += y[j] * w;
      }
    s0 += FLIGHT;
    if (s0 >= n) break;
    load(s0);
  }
  if (idx >= total) return;
  x *= over(l);
  const int row = r.row0 + idx / p.group, head = h * p.group + idx % p.group;
  const float out[4] = {x[0], x[1], x[2], x[3]};
  store_out<BF16>(p, row, head, db * 16 + quad * 4, out, D);
  if (db == 0 && quad == 0 && p.lse) p.lse[(size_t)head * p.lse_stride + row] = l == 0.f ? -INFINITY : m + __logf(l);
}

template <bool BF16, int D>
hipError_t launch(const CacheAttnLaunch &p, hipStream_t st) {
  constexpr int MT = BF16 ? kCacheWideRows / 64 : kCacheWideRowsF32 / 64;
  const int jobs = p.blocks * p.c.hkv, pairs = p.cu[p.n_req] * p.hq;
  if (p.wide) {
    const int groups = p.c.hkv * p.n_splits, rest = groups % kXcdCount * p.blocks;
    const int per_xcd = groups / kXcdCount * p.blocks + (rest + kXcdCount - 1) / kXcdCount;
    cache_wide_kernel<BF16, D, MT><<<per_xcd * kXcdCount, kThreads, 0, st>>>(p);
  } else if (p.n_splits > 1) {
    cache_line_kernel<BF16, D><<<p.n_splits * p.c.hkv, kThreads, 0, st>>>(p);
  } else {
    cache_attn_kernel<BF16, D><<<jobs, kThreads, 0, st>>>(p);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.n_splits == 1) return e;
  if (p.wide) cache_wide_join_kernel<BF16, D, MT><<<jobs * kWaves * MT * (D / 16), 64, 0, st>>>(p);
  else cache_line_join_kernel<BF16, D><<<pairs, kThreads, 0, st>>>(p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_cache_attn(bool bf16, const CacheAttnLaunch &p, hipStream_t st) {
  if (p.c.d == 128) return bf16 ? launch<true, 128>(p, st) : launch<false, 128>(p, st);
  return bf16 ? launch<true, 64>(p, st) : launch<false, 64>(p, st);
}

}  // namespace daf
