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
#include <math.h>

#include <type_traits>

#include "cache.h"

namespace daf {
namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = kCacheAttnThreads;
constexpr int kWaves = kThreads / 64;
constexpr int kRows = kCacheAttnRows;
constexpr int kXcdCount = 8;  // workgroups go to the XCDs in turn
constexpr float kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

// eight codes (8 bytes) times a power of two, as bf16
__device__ __forceinline__ bf16x8 widen(unsigned lo, unsigned hi, float scale) {
#if defined(__HIP_DEVICE_COMPILE__)
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
#else
  return bf16x8{};
#endif
}

// the same as fp16, exactly for scales from 2^-15 to 1
__device__ __forceinline__ f16x8 widen_f16(unsigned lo, unsigned hi, float scale) {
#if defined(__HIP_DEVICE_COMPILE__)
  const f16x2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, scale, false);
  const f16x2 b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, scale, true);
  const f16x2 c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, scale, false);
  const f16x2 d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, scale, true);
  return f16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
#else
  return f16x8{};
#endif
}

__device__ __forceinline__ f32x4 mfma(const bf16x8 &a, const bf16x8 &b, const f32x4 &c) {
#if defined(__HIP_DEVICE_COMPILE__)
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
#else
  return c;
#endif
}
__device__ __forceinline__ f32x4 mfma(const f16x8 &a, const f16x8 &b, const f32x4 &c) {
#if defined(__HIP_DEVICE_COMPILE__)
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
#else
  return c;
#endif
}

// x and the same register of the lanes that hold the same row (lane ^ 16, ^ 32)
__device__ __forceinline__ float row_max(float x) {
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}
__device__ __forceinline__ float row_sum(float x) {
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}

// 1 / sum of a row's weights. 0 is the row that sees no key; a NaN among the scores makes
// the sum NaN, which goes on to o and the LSE (a test for > 0 would turn it into no key).
__device__ __forceinline__ float over(float sum) { return sum == 0.f ? 0.f : 1.f / sum; }

// TERMS bf16 values whose sum is x, to 8 bits each
template <int TERMS>
__device__ __forceinline__ void split_terms(const float (&x)[8], bf16x8 (&out)[TERMS]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float r = x[i];
#pragma unroll
    for (int j = 0; j < TERMS; ++j) {
      out[j][i] = (__bf16)r;
      r -= (float)out[j][i];
    }
  }
}

// A row of q as the B operand, in T terms: put(term, step, x). Lane quad holds
// features 64 c + 16 quad + 8 e .. + 7 of step 2 c + e, e < 2.
template <bool BF16, int D, typename F>
__device__ __forceinline__ void load_q(const CacheAttnLaunch &p, size_t at, int quad, F put) {
#pragma unroll
  for (int ds = 0; ds < D / 32; ++ds) {
    const int f = (ds >> 1) * 64 + quad * 16 + (ds & 1) * 8;
    if constexpr (BF16) {
      put(0, ds, *reinterpret_cast<const bf16x8 *>((const __bf16 *)p.q + at + f));
    } else {
      const f32x4 a = *reinterpret_cast<const f32x4 *>((const float *)p.q + at + f);
      const f32x4 c = *reinterpret_cast<const f32x4 *>((const float *)p.q + at + f + 4);
      const float x[8] = {a[0], a[1], a[2], a[3], c[0], c[1], c[2], c[3]};
      bf16x8 part[3];
      split_terms<3>(x, part);
#pragma unroll
      for (int j = 0; j < 3; ++j) put(j, ds, part[j]);
    }
  }
}

// Maxima in one instruction each: fmaxf on results of matrix instructions brings a
// second one. max2 is for those results: the wait that they need before a vector
// instruction reads them is put in for instructions that the compiler knows, and not
// for max3's, which is therefore given results of vector instructions alone.
__device__ __forceinline__ float max2(float a, float b) {
  float inf = INFINITY;
  asm("" : "+s"(inf));  // a known infinity makes this fmaxf again
  return __builtin_amdgcn_fmed3f(a, b, inf);
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}
// of a lane's scores of 8 keys
__device__ __forceinline__ float max_score(const f32x4 &a, const f32x4 &b) {
  const float x = max2(a[0], a[1]), y = max2(a[2], a[3]), z = max2(b[0], b[1]), w = max2(b[2], b[3]);
  return max3(max3(x, y, z), w, w);
}

struct Request {
  int b, block;      // request of the launch and row block in it
  int row0, n;       // its rows
  int L;             // tokens of its sequence
  const int32_t *pages;
};

// The b < n with prefix[b] <= at < prefix[b + 1]: every lane looks at one of each 64
// (a binary search would wait for a load per step).
__device__ __forceinline__ int find_in(const int32_t *prefix, int n, int at) {
  const int lane = threadIdx.x & 63;
  int b = 0;
  for (int i = 0; i < n; i += 64) b += __builtin_popcountll(__ballot(i + lane < n && prefix[i + lane + 1] <= at));
  return b;
}

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

// last key that row j of the request sees, -1 if none
__device__ __forceinline__ int row_limit(const CacheAttnLaunch &p, const Request &r, int j) {
  return max(-1, p.pos ? min(p.pos[r.row0 + j], r.L - 1) : r.L - r.n + j);
}

__device__ __forceinline__ u32x2 pack4(const f32x4 &x) {
  return u32x2{__builtin_bit_cast(unsigned, bf16x2{(__bf16)x[0], (__bf16)x[1]}),
               __builtin_bit_cast(unsigned, bf16x2{(__bf16)x[2], (__bf16)x[3]})};
}

template <bool BF16>
__device__ __forceinline__ void store_out(const CacheAttnLaunch &p, int row, int head, int col, const float (&x)[4], int d) {
  const size_t at = ((size_t)row * p.hq + head) * d + col;
  if constexpr (BF16) {
    *reinterpret_cast<u32x2 *>((__bf16 *)p.o + at) = pack4(f32x4{x[0], x[1], x[2], x[3]});
  } else {
    *reinterpret_cast<f32x4 *>((float *)p.o + at) = f32x4{x[0], x[1], x[2], x[3]};
  }
}

// K and V of one page of one head, in operand layout
template <int D>
struct Frags {
  u32x4 k[4][D / 64];  // [key block][64 features]: 16 features of one key per lane
  u32x4 v[D / 16];     // [16 features]: 16 keys of one feature per lane
  float ks, vs;
};

// ---- few rows --------------------------------------------------------------------
template <int D>
struct FewShared {
  float o[kWaves][kRows][D + 4];
  float m[kWaves][kRows], l[kWaves][kRows];
};

// Row block r.block of a request over the pages pg0 .. pg_end - 1 of its sequence, by
// the whole workgroup. Results go to the output, or with `slot` >= 0 to that place
// among the partial ones.
template <bool BF16, int D>
__device__ __forceinline__ void few_rows(const CacheAttnLaunch &p, FewShared<D> &sh, const Request &r, int h, int pg0,
                                         int pg_end, int slot) {
  constexpr int T = BF16 ? 1 : 3, TW = BF16 ? 2 : 3, DS = D / 32, DB = D / 16;  // terms of q and of a weight
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n16 = lane & 15, quad = lane >> 4;
  // the ids of this wave's pages (pg0 + wave + 4 i), 64 at a time in the lanes; they do
  // not wait for the length
  auto load_ids = [&](int i) {
    const int64_t pg = (int64_t)pg0 + wave + 4 * (i + lane);
    return pg < p.c.max_seq_pages ? r.pages[pg] : -1;
  };
  int ids = load_ids(0), ids_at = 0;
  const int total = r.n * p.group;
  const int idx = r.block * kRows + n16;      // this lane's (row, head) pair
  const int idc = min(idx, total - 1);        // pairs past the end repeat the last one
  const int row = idc / p.group, head = h * p.group + idc % p.group;
  bf16x8 qf[T][DS];
  load_q<BF16, D>(p, ((size_t)(r.row0 + row) * p.hq + head) * D, quad,
                  [&](int j, int ds, const bf16x8 &x) { qf[j][ds] = x; });
  const int limit = row_limit(p, r, row);
  // range of limits over the block's rows
  int lim_hi = limit, lim_lo = limit;
#pragma unroll
  for (int m = 8; m; m >>= 1) {
    lim_hi = max(lim_hi, __shfl_xor(lim_hi, m));
    lim_lo = min(lim_lo, __shfl_xor(lim_lo, m));
  }
  lim_hi = __builtin_amdgcn_readfirstlane(lim_hi);
  lim_lo = __builtin_amdgcn_readfirstlane(lim_lo);
  const int pg1 = min(min(pg_end, (r.L + kPage - 1) / kPage), (lim_hi >> 6) + 1);

  f32x4 o[DB] = {};
  float m_run = -INFINITY, l_run = 0.f;

  auto page_id = [&](int i) {  // i-th page of this wave
    if (i >= ids_at + 64) {
      ids_at = i;
      ids = load_ids(i);
    }
    return __builtin_amdgcn_readlane(ids, i - ids_at);
  };
  // first page from the i-th on that is there; -1 if none
  int id_next = -1;
  auto next_page = [&](int i) {
    for (; pg0 + wave + 4 * i < pg1; ++i) {
      id_next = page_id(i);
      if ((unsigned)id_next < (unsigned)p.c.n_pages) return i;
    }
    return -1;
  };
  auto load = [&](Frags<D> &f, int id) {
    const size_t at = (size_t)id * p.c.hkv + h;
    const unsigned char *kp = p.c.k + at * (kPage * D), *vp = p.c.v + at * (kPage * D);
    const int krow = (n16 >> 2) * 16 + (n16 & 3);
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int c = 0; c < D / 64; ++c)
        f.k[t][c] = *reinterpret_cast<const u32x4 *>(kp + (krow + t * 4) * D + c * 64 + quad * 16);
#pragma unroll
    for (int db = 0; db < DB; ++db) f.v[db] = *reinterpret_cast<const u32x4 *>(vp + (db * 16 + n16) * kPage + quad * 16);
    f.ks = p.c.k_scale[at];
    f.vs = p.c.v_scale[at];
  };
  auto work = [&](Frags<D> &f, int pg) {
    f32x4 s[4] = {};
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int ds = 0; ds < DS; ++ds) {
        const bf16x8 a = widen(f.k[t][ds >> 1][(ds & 1) * 2], f.k[t][ds >> 1][(ds & 1) * 2 + 1], f.ks);
#pragma unroll
        for (int j = T - 1; j >= 0; --j) s[t] = mfma(a, qf[j][ds], s[t]);  // small terms first
      }
    const int key0 = pg * kPage + quad * 16;  // s[t][i]: key0 + 4 t + i
    if (pg * kPage + kPage - 1 > lim_lo) {
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (key0 + 4 * t + i > limit) s[t][i] = -INFINITY;
      // keys that no row of the block sees may hold NaN codes: their values become 0
      if (pg * kPage + kPage - 1 > lim_hi) {
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const int left = lim_hi + 1 - (key0 + 4 * t);
          const unsigned keep = left >= 4 ? ~0u : left <= 0 ? 0u : (1u << 8 * left) - 1;
#pragma unroll
          for (int db = 0; db < DB; ++db) f.v[db][t] &= keep;
        }
      }
    }
    const float upper = max_score(s[2], s[3]), mx = max3(max_score(s[0], s[1]), upper, upper);
    const float m_new = fmaxf(m_run, row_max(mx) * p.scale_log2);
    if (__ballot(m_new > m_run)) {
      const float alpha = m_new > m_run ? exp2_(m_run - m_new) : 1.f;
      l_run *= alpha;
#pragma unroll
      for (int db = 0; db < DB; ++db) o[db] *= alpha;
      m_run = m_new;
    }
    const float ref = m_run == -INFINITY ? 0.f : m_run;  // a row that has seen no key
    float e[2][8];
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        e[t >> 1][(t & 1) * 4 + i] = exp2_(__builtin_fmaf(s[t][i], p.scale_log2, -ref));
        l_run += e[t >> 1][(t & 1) * 4 + i];
      }
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      bf16x8 pf[TW];
      split_terms<TW>(e[ks], pf);
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        const bf16x8 a = widen(f.v[db][2 * ks], f.v[db][2 * ks + 1], f.vs);
#pragma unroll
        for (int j = TW - 1; j >= 0; --j) o[db] = mfma(a, pf[j], o[db]);
      }
    }
  };

  Frags<D> fa, fb;
  int i = next_page(0);
  if (i >= 0) load(fa, id_next);
  while (i >= 0) {
    int i2 = next_page(i + 1);
    if (i2 >= 0) load(fb, id_next);
    work(fa, pg0 + wave + 4 * i);
    if (i2 < 0) break;
    i = next_page(i2 + 1);
    if (i >= 0) load(fa, id_next);
    work(fb, pg0 + wave + 4 * i2);
  }

  // join the waves
  l_run = row_sum(l_run);
  if (quad == 0) sh.m[wave][n16] = m_run, sh.l[wave][n16] = l_run;
#pragma unroll
  for (int db = 0; db < DB; ++db) *reinterpret_cast<f32x4 *>(&sh.o[wave][n16][db * 16 + quad * 4]) = o[db];
  __syncthreads();
  const int rr = threadIdx.x >> 4, c0 = threadIdx.x & 15;  // 16 lanes per pair
  const int out = r.block * kRows + rr;
  if (out >= total) return;
  const int orow = r.row0 + out / p.group, ohead = h * p.group + out % p.group;
  float m = sh.m[0][rr], w[kWaves], l = 0.f;
#pragma unroll
  for (int k = 1; k < kWaves; ++k) m = fmaxf(m, sh.m[k][rr]);
#pragma unroll
  for (int k = 0; k < kWaves; ++k) {
    w[k] = sh.m[k][rr] == -INFINITY ? 0.f : exp2_(sh.m[k][rr] - m);
    l += w[k] * sh.l[k][rr];
  }
  const float inv = over(l);
  const float lse = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
#pragma unroll
  for (int c = c0 * 4; c < D; c += 64) {
    float x[4] = {};
#pragma unroll
    for (int k = 0; k < kWaves; ++k) {
      const f32x4 v = *reinterpret_cast<const f32x4 *>(&sh.o[k][rr][c]);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = __builtin_fmaf(w[k], v[e], x[e]);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] *= inv;
    if (slot < 0)
      store_out<BF16>(p, orow, ohead, c, x, D);
    else
      *reinterpret_cast<f32x4 *>(p.part_o + ((size_t)slot * kRows + rr) * D + c) = f32x4{x[0], x[1], x[2], x[3]};
  }
  if (c0 == 0) {
    if (slot >= 0) p.part_lse[slot * kRows + rr] = lse;
    else if (p.lse) p.lse[(size_t)ohead * p.lse_stride + orow] = lse;
  }
}

// Short sequences: a workgroup per row block and head.
template <bool BF16, int D>
__global__ __launch_bounds__(kThreads, 2) void cache_attn_kernel(const CacheAttnLaunch p) {
  __shared__ FewShared<D> sh;
  const Request r = find_request(p, blockIdx.x % p.blocks);
  few_rows<BF16, D>(p, sh, r, blockIdx.x / p.blocks, 0, INT32_MAX, -1);
}

// Long ones: the row blocks' pages, one block after the other, make one line per head,
// of which every workgroup takes an equal piece, whatever the lengths are on the device
// (a batch is planned for the longest that it may have, and a captured one grows). A
// workgroup's first and last row block may be shared with its neighbours: their
// partial results have two places per workgroup, 0 for a block that did not begin
// in it and 1 for one that does not end in it.
//
// The line lies in the lanes of every wave: lane i has requests 4 i .. 4 i + 3.
struct Line {
  int first;               // of the lane's requests' pages in the line
  int units[4], L[4], seq[4];
  int end, piece;          // pages of the line, and of a workgroup
};
static_assert(kMaxCacheReqs == 4 * 64, "four requests per lane");

__device__ __forceinline__ int line_pages(int L) { return max(1, (L + kPage - 1) / kPage); }

__device__ __forceinline__ Line build_line(const CacheAttnLaunch &p) {
  Line s;
  const int lane = threadIdx.x & 63;
  int sum = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int b = 4 * lane + j;
    s.seq[j] = b >= p.n_req ? -1 : p.seq ? p.seq[b] : b;
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) s.L[j] = min(seq_len(p.c.len, p.c.n_seqs, p.c.max_seq_pages, s.seq[j]), p.max_len);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int b = 4 * lane + j;
    s.units[j] = b < p.n_req ? (p.blk0[b + 1] - p.blk0[b]) * line_pages(s.L[j]) : 0;
    sum += s.units[j];
  }
  int upto = sum;
#pragma unroll
  for (int k = 1; k < 64; k <<= 1) {
    const int y = __shfl_up(upto, k);
    if (lane >= k) upto += y;
  }
  s.first = upto - sum;
  s.end = __builtin_amdgcn_readlane(upto, 63);
  s.piece = max(kMinPiece, (s.end + p.n_splits - 1) / p.n_splits);
  return s;
}

// fp32's terms of 128 features need more than 256 registers: one workgroup per CU, with
// whole pages in flight, for two whose registers spill (131072 keys, a row for 28
// heads: 30.4 us for 45.3).
template <bool BF16, int D>
constexpr int kLineWgs = BF16 || D == 64 ? 2 : 1;
template <bool BF16, int D>
__global__ __launch_bounds__(kThreads, (kLineWgs<BF16, D>)) void cache_line_kernel(const CacheAttnLaunch p) {
  __shared__ FewShared<D> sh;
  const int lane = threadIdx.x & 63;
  const int h = blockIdx.x % p.c.hkv, k = blockIdx.x / p.c.hkv;
  const Line line = build_line(p);
  if (blockIdx.x == 0 && threadIdx.x < 64) {  // for the join
    int first = line.first;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      p.line[4 * lane + j] = first;
      p.line[kMaxCacheReqs + 4 * lane + j] = line_pages(line.L[j]);
      first += line.units[j];
    }
    if (lane == 0) p.line[2 * kMaxCacheReqs] = line.piece;
  }
  int at = k * line.piece;  // the host keeps n_splits * piece within 32 bits
  const int to = min(at + line.piece, line.end);
  while (at < to) {
    // the lane, then the request of the page `at`
    const int last = __builtin_popcountll(__ballot(line.first <= at)) - 1;
    int first = __builtin_amdgcn_readlane(line.first, last), j = 0, L = __builtin_amdgcn_readlane(line.L[0], last),
        seq = __builtin_amdgcn_readlane(line.seq[0], last);
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      const int next = first + __builtin_amdgcn_readlane(line.units[i], last);
      if (j == i && at >= next) {
        first = next;
        j = i + 1;
        L = __builtin_amdgcn_readlane(line.L[i + 1], last);
        seq = __builtin_amdgcn_readlane(line.seq[i + 1], last);
      }
    }
    Request r;
    r.b = 4 * last + j;
    r.L = L;
    const int pages = line_pages(L), rest = at - first;
    r.block = rest / pages;
    r.row0 = p.cu[r.b];
    r.n = p.cu[r.b + 1] - r.row0;
    r.pages = p.c.table + (int64_t)((unsigned)seq < (unsigned)p.c.n_seqs ? seq : 0) * p.c.max_seq_pages;
    const int pg0 = rest - r.block * pages, pg_end = min(pages, pg0 + to - at);
    const int slot = pg0 == 0 && pg_end == pages ? -1 : (h * p.n_splits + k) * 2 + (pg0 == 0);
    few_rows<BF16, D>(p, sh, r, h, pg0, pg_end, slot);
    at += pg_end - pg0;
    __syncthreads();  // sh is free
  }
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

// ---- many rows -------------------------------------------------------------------
// A row block is 4 waves of 16 MT (row, head) pairs, which share every page through
// LDS: copies go from memory to LDS in the layout that the waves read (16 bytes per
// lane of the operand, in lane order: no bank conflicts for K), two pages ahead.
//
// Half pages (32 keys) go through three stages, each of another half: the scores of
// half h + 1, the weights of half h and the value product of half h - 1 make one
// block of straight code, in which every matrix instruction has 3 to 4 vector
// instructions of the other stages beside it: a SIMD with two waves overlaps them (4
// matrix and 9 vector instructions in turn take 35.5 ns, alone 27.5 and 19.9).
//
// Bound by that issue: 128 rows of 28 heads on 4 of 128 over 32896 keys, 60 GFLOP, take
// 70 us (860 TFLOP/s; the first calls after a pause 77). Of the 145,000 cycles that a CU is
// busy its SIMDs' matrix instructions are 40% and their vector instructions 48% (per 32
// keys and 32 rows 32 and 155, 64 of them conversions of codes).
// The prologue is 4 us, and of the two workgroups of a CU the older is served first and
// leaves the younger alone for the last quarter. 8 waves per workgroup, weights through
// LDS, K converted once for all waves and pages further ahead did not take less.
//
// The reference m of a row is an integer (base-2 units), so that raising it scales O and
// the sum by a power of two, exactly. It is raised before a half whose scores pass it by
// more than kLift + kSlack, to kLift below the ceiling of the row's maximum: a weight is
// at most 2^(kLift + kSlack), a row's largest one at least 2^(kLift - 1).
constexpr int kStages = 3;
constexpr float kNoReference = -3e38f;  // before the first visible key

// How weights enter the value product: as bf16 terms, with the values in bf16, at any
// scales; a weight is off by 2^-8N of itself.
template <int N>
struct BfWeights {
  static constexpr int TERMS = N;
  static constexpr float kLift = 0.f, kSlack = 8.f;
  using V = bf16x8;
  static __device__ __forceinline__ V values(unsigned lo, unsigned hi, float scale) { return widen(lo, hi, scale); }
  static __device__ __forceinline__ void weights(const float (&x)[8], V (&out)[N]) { split_terms<N>(x, out); }
};
// Or in fp16, with the codes in fp16 in units of the workgroup's largest scale of V: one
// product where two bf16 terms are two (128 question rows over 32896 keys, us a call: 76
// for 96).
// A weight is off by 2^-11 of itself, or 2^-35 of the row's largest one: small ones are
// held in steps of 2^-24. So that this does not show beside the values of any page, the
// scales may be 2^4 apart; where they are further, the workgroup takes two bf16 terms.
// (Slack of 4: raises cost nothing yet; 76.4 us, with 8 76.4, with 2 78.7, with 1 82.2.)
struct HalfWeights {
  static constexpr int TERMS = 1;
  static constexpr float kLift = 11.f, kSlack = 4.f;
  using V = f16x8;
  static __device__ __forceinline__ V values(unsigned lo, unsigned hi, float scale) { return widen_f16(lo, hi, scale); }
  static __device__ __forceinline__ void weights(const float (&x)[8], V (&out)[1]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) out[0][i] = (_Float16)x[i];
  }
};
constexpr float kHalfSpread = 16.f;

template <int N>
__device__ __forceinline__ void wait_vm() {
  __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | 0x0F70);  // vmcnt(N); the other counters at their maxima
}
__device__ __forceinline__ void lds_barrier() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_barrier" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

// One 1 KiB copy: lane i's 16 bytes at byte voff + soff of the buffer go to LDS byte
// lds + 16 i. In asm, so that the compiler does not wait for the copies in flight at
// each LDS read: wait_vm counts them, the barriers order them. The s_nop makes up the
// five wait states between a vector instruction that writes one of the scalar operands
// and this read of it, which the compiler does not see here.
__device__ __forceinline__ void copy_to_lds(const u32x4 &rsrc, uint32_t voff, uint32_t soff, uint32_t lds) {
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile(
      "s_mov_b32 m0, %0\n\t"
      "s_nop 3\n\t"
      "buffer_load_dwordx4 %1, %2, %3 offen lds"
      :
      : "s"(lds), "v"(voff), "s"(rsrc), "s"(soff)
      : "memory", "m0");
#endif
}

template <bool BF16, int D, int MT>
struct Wide {
  static constexpr int T = BF16 ? 1 : 3, DS = D / 32, DB = D / 16;
  static constexpr int C = D / 64;                         // 16-byte pieces of a key that a lane reads
  static constexpr int UNITS = 4 * C;                      // steps of the scores of a half
  static constexpr int PAGE_BYTES = 2 * kPage * D;
  using Scores = f32x4[MT][2];   // a lane's 8 keys of a half, per row
  template <typename P>
  using Weights = typename P::V[MT][P::TERMS];
  bf16x8 q[T][MT][DS];
  f32x4 o[MT][DB];
  float m[MT], l[MT], top[MT];   // reference, sum, largest score that needs no raise
  int limit[MT];
  float scale_log2;
  int lane, lim_hi;

  // K of half HALF of a page in LDS: of 16 keys, a lane's pieces
  template <int HALF>
  __device__ __forceinline__ void read_k(const unsigned char *page, u32x4 (&k)[2][C]) const {
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int c = 0; c < C; ++c)
        k[t][c] = *reinterpret_cast<const u32x4 *>(page + ((2 * HALF + t) * C + c) * 1024 + lane * 16);
  }
  // V of a page: of 16 features, a lane's 16 keys (the first 8 are half 0)
  __device__ __forceinline__ void read_v(const unsigned char *page, u32x4 (&v)[DB]) const {
#pragma unroll
    for (int db = 0; db < DB; ++db) v[db] = *reinterpret_cast<const u32x4 *>(page + kPage * D + db * 1024 + lane * 16);
  }
  // step u of the scores, u < UNITS
  __device__ __forceinline__ void score_unit(int u, const u32x4 (&k)[2][C], float ks, Scores &s) const {
    const int t = u & 1, e = (u >> 1) & 1, c = u >> 2;
    const bf16x8 a = widen(k[t][c][2 * e], k[t][c][2 * e + 1], ks);
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int j = T - 1; j >= 0; --j)
        s[mt][t] = mfma(a, q[j][mt][2 * c + e], c + e == 0 && j == T - 1 ? f32x4{} : s[mt][t]);
  }
  template <typename P, int HALF>
  __device__ __forceinline__ void value_unit(int db, const u32x4 (&v)[DB], float vs, const Weights<P> &pf) {
    const typename P::V a = P::values(v[db][2 * HALF], v[db][2 * HALF + 1], vs);
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int j = P::TERMS - 1; j >= 0; --j) o[mt][db] = mfma(a, pf[mt][j], o[mt][db]);
  }
  // keys (key, key + 1, ...: a lane's 8) past a row's limit get no weight, and the
  // values of those that no row of the wave sees, which may be NaN codes, become 0
  __device__ __forceinline__ void mask_scores(Scores &s, int key) const {
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (key + i > limit[mt]) s[mt][i >> 2][i & 3] = -INFINITY;
  }
  __device__ __forceinline__ void mask_values(u32x4 (&v)[DB], int key) const {
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const int left = lim_hi + 1 - key - 4 * t;
      const unsigned keep = left >= 4 ? ~0u : left <= 0 ? 0u : (1u << 8 * left) - 1;
#pragma unroll
      for (int db = 0; db < DB; ++db) v[db][t] &= keep;
    }
  }
  // Raises the references that the scores s need raised; true if there are any. O follows
  // after the block, with the weights in flight: rescale.
  template <typename P>
  __device__ __forceinline__ bool raise(const Scores &s, float (&alpha)[MT]) {
    bool need = false;
    float mx[MT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      mx[mt] = max_score(s[mt][0], s[mt][1]);
      need |= mx[mt] > top[mt];
    }
    if (__builtin_expect(__ballot(need) == 0, 1)) return false;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      const float to = fmaxf(m[mt], ceilf(row_max(mx[mt]) * scale_log2) - P::kLift);
      alpha[mt] = exp2_(m[mt] - to);  // a power of two; 0 for the first keys
      m[mt] = to;
      top[mt] = (to + P::kLift + P::kSlack) / scale_log2;
      l[mt] *= alpha[mt];
    }
    return true;
  }
  __device__ __forceinline__ void rescale(const float (&alpha)[MT]) {
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int db = 0; db < DB; ++db) o[mt][db] *= alpha[mt];
  }
  // The block: weights of scores s into pf (l grows), scores of K k into s, value
  // product of the weights that pf held.
  template <typename P, int HALF>  // of v's page
  __device__ __forceinline__ void block(Scores &s, Weights<P> &pf, const u32x4 (&k)[2][C], float ks, const u32x4 (&v)[DB],
                                        float vs) {
    Scores next;
    float e[MT][8];
#pragma unroll
    for (int step = 0; step < 8; ++step) {
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        e[mt][step] = exp2_(__builtin_fmaf(s[mt][step >> 2][step & 3], scale_log2, -m[mt]));
        l[mt] += e[mt][step];
      }
      if (step * UNITS % 8 == 0) score_unit(step * UNITS / 8, k, ks, next);
      if (step * DB % 8 == 0) value_unit<P, HALF>(step * DB / 8, v, vs, pf);
    }
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      P::weights(e[mt], pf[mt]);
      s[mt][0] = next[mt][0];
      s[mt][1] = next[mt][1];
    }
    // a matrix instruction, then four others, and so on
#pragma unroll
    for (int i = 0; i < (UNITS * T + DB * P::TERMS) * MT; ++i) {  // its matrix instructions
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x402, 4, 0);
    }
  }
};

template <bool BF16, int D, int MT>
__global__ __launch_bounds__(kThreads, D == 64 ? 3 : 2) void cache_wide_kernel(const CacheAttnLaunch p) {
  using W = Wide<BF16, D, MT>;
  constexpr int DB = W::DB, C = W::C;
  constexpr int PAGE_BYTES = W::PAGE_BYTES, IPW = PAGE_BYTES / 1024 / kWaves;  // copies per wave and page
  __shared__ __align__(16) unsigned char lds[kStages * PAGE_BYTES];
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
  // page ids, 64 at a time in the lanes; the first ones do not wait for the length
  auto load_ids = [&](int i) {
    return i + lane < p.split_pages && pg0 + i + lane < p.c.max_seq_pages ? r.pages[pg0 + i + lane] : -1;
  };
  int id = load_ids(0);
  const int pages = (r.L + kPage - 1) / kPage;
  if (split > 0 && pg0 >= pages) return;  // no keys here: the join leaves this split out
  const int total = r.n * p.group;
  constexpr int PAIRS = kWaves * 16 * MT;  // of a row block
  int last = -1;                           // last key that a row of the block sees
  if (p.pos) {
#pragma unroll
    for (int i = 0; i < PAIRS; i += 64)
      last = max(last, row_limit(p, r, min(r.block * PAIRS + i + lane, total - 1) / p.group));
#pragma unroll
    for (int m = 32; m; m >>= 1) last = max(last, __shfl_xor(last, m));
  } else {
    last = row_limit(p, r, (min((r.block + 1) * PAIRS, total) - 1) / p.group);
  }
  const int seen = __builtin_amdgcn_readfirstlane((last >> 6) + 1);  // pages

  W w;
  w.scale_log2 = p.scale_log2;
  w.lane = lane;
  int lim_hi = INT32_MIN, lim_lo = INT32_MAX;
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    const int idx = min((r.block * kWaves + wave) * 16 * MT + mt * 16 + n16, total - 1);  // past the end: the last pair
    const int row = idx / p.group, head = h * p.group + idx % p.group;
    w.limit[mt] = row_limit(p, r, row);
    lim_hi = max(lim_hi, w.limit[mt]);
    lim_lo = min(lim_lo, w.limit[mt]);
    const size_t q_at = ((size_t)(r.row0 + row) * p.hq + head) * D;
    load_q<BF16, D>(p, q_at, quad, [&](int j, int ds, const bf16x8 &x) { w.q[j][mt][ds] = x; });
    w.m[mt] = kNoReference;
    w.top[mt] = kNoReference / p.scale_log2;
    w.l[mt] = 0.f;
#pragma unroll
    for (int db = 0; db < DB; ++db) w.o[mt][db] = f32x4{};
  }
#pragma unroll
  for (int m = 8; m; m >>= 1) {
    lim_hi = max(lim_hi, __shfl_xor(lim_hi, m));
    lim_lo = min(lim_lo, __shfl_xor(lim_lo, m));
  }
  w.lim_hi = __builtin_amdgcn_readfirstlane(lim_hi);
  lim_lo = __builtin_amdgcn_readfirstlane(lim_lo);

  // Of 64 of this split's pages, from the i-th on, those that are there and that a row of
  // the block sees, one per lane, in order: id becomes theirs.
  const int span = min(p.split_pages, seen - pg0);  // pages of the split that a row sees
  int n = 0, firsts = 0;                            // how many; first keys
  float kss = 0.f, vss = 0.f;                       // scales
  auto settle = [&](int i) {
    const unsigned long long mask = __ballot(i + lane < span && (unsigned)id < (unsigned)p.c.n_pages);
    n = __builtin_popcountll(mask);
    firsts = (pg0 + i + lane) * kPage;
    if (mask & (mask + 1)) {  // pages are missing in between: close the gaps
      const int to = (mask >> lane) & 1 ? __builtin_popcountll(mask & ((1ull << lane) - 1)) * 4 : 252;
      const int a = __builtin_amdgcn_ds_permute(to, id), f = __builtin_amdgcn_ds_permute(to, firsts);
      id = a;
      firsts = f;
    }
    const size_t at = (size_t)(lane < n ? id : 0) * p.c.hkv + h;
    kss = p.c.k_scale[at];
    vss = lane < n ? p.c.v_scale[at] : 0.f;
  };
  auto of_page = [](float x, int i) {
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), i));
  };
  // copies of this wave: half of the K (waves 0 and 1) or V (2 and 3) of a page
  const uint32_t voff = wave < 2 ? ((n16 >> 2) * 16 + (n16 & 3)) * D + quad * 16 : n16 * kPage + quad * 16;
  auto soff = [&](int i) {
    const int j = (wave & 1) * IPW + i;
    return wave < 2 ? j / (D / 64) * 4 * D + j % (D / 64) * 64 : j * 16 * kPage;
  };
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char *)lds + wave * IPW * 1024;
  const unsigned char *pool = wave < 2 ? p.c.k : p.c.v;
  auto fetch = [&](int i) {
    const int pid = __builtin_amdgcn_readlane(id, i);
    const uint64_t base = (uint64_t)(pool + ((size_t)pid * p.c.hkv + h) * (kPage * D));
    const u32x4 rsrc = {(uint32_t)base, (uint32_t)(base >> 32) & 0xffffu, (uint32_t)(kPage * D), 0x00020000u};
    const uint32_t to = lds0 + i % kStages * PAGE_BYTES;
#pragma unroll
    for (int c = 0; c < IPW; ++c) copy_to_lds(rsrc, voff, soff(c), to + c * 1024);
  };
  auto stage = [&](int i) { return lds + i % kStages * PAGE_BYTES; };

  auto begin = [&] {
    if (n > 0) fetch(0);
    if (n > 1) fetch(1);
  };
  // The products of the n pages, with weights as P has them.
  auto pages_of_64 = [&](auto weights) {
    using P = decltype(weights);
    typename W::Scores s;
    typename W::template Weights<P> pf = {};
    u32x4 v[DB] = {};
    // Page i: its scores of half 0 are in s, the weights of the page before's half 1 in pf.
    auto step = [&](int i, auto masked) {
      constexpr bool MASK = decltype(masked)::value;
      const int key = __builtin_amdgcn_readlane(firsts, i) + quad * 16;
      const float ks = of_page(kss, i), vs = of_page(vss, i);
      const float ks_next = of_page(kss, min(i + 1, n - 1)), vs_before = of_page(vss, max(i - 1, 0));
      // page i + 1 is here for every wave, and all are done with page i - 1, whose place
      // the copies of page i + 2 take
      wait_vm<0>();
      lds_barrier();
      if (i + 2 < n) fetch(i + 2);
      u32x4 k[2][C];
      w.template read_k<1>(stage(i), k);
      if constexpr (MASK) w.mask_scores(s, key);
      float alpha[MT];
      bool raised = w.template raise<P>(s, alpha);
      w.template block<P, 1>(s, pf, k, ks, v, vs_before);  // v: of page i - 1 (zeros for the first)
      w.template read_k<0>(stage(i + 1), k);
      w.read_v(stage(i), v);
      if (__builtin_expect(raised, 0)) w.rescale(alpha);
      if constexpr (MASK) {
        w.mask_scores(s, key + 8);
        w.mask_values(v, key);
      }
      raised = w.template raise<P>(s, alpha);
      w.template block<P, 0>(s, pf, k, ks_next, v, vs);  // past the last page: scores that nobody uses
      if (__builtin_expect(raised, 0)) w.rescale(alpha);
    };
    wait_vm<0>();
    __syncthreads();
    u32x4 k[2][C];
    w.template read_k<0>(stage(0), k);
#pragma unroll
    for (int u = 0; u < W::UNITS; ++u) w.score_unit(u, k, of_page(kss, 0), s);
    // pages that every row of the wave sees whole, then the others
    const int whole = __builtin_popcountll(__ballot(lane < n && firsts + kPage - 1 <= lim_lo));
    int i = 0;
    for (; i < whole; ++i) step(i, std::false_type{});
    for (; i < n; ++i) step(i, std::true_type{});
#pragma unroll
    for (int db = 0; db < DB; ++db) w.template value_unit<P, 1>(db, v, of_page(vss, n - 1), pf);
  };
  float unit = 1.f, per_unit = 1.f;  // of O and V's scales
  auto run = [&](auto weights) {
    for (int i = 0;;) {
      vss *= per_unit;
      if (n > 0) pages_of_64(weights);
      i += 64;
      if (i >= span) break;
      id = load_ids(i);
      settle(i);
      lds_barrier();  // every wave is done with the pages before
      begin();
    }
  };
  settle(0);
  begin();
  if constexpr (BF16) {
    // the largest scale of V of all pages, and whether one is further from it than fp16 takes
    float most = vss, least = vss > 0.f ? vss : INFINITY;
    bool odd = !(vss >= 0.f);
    for (int i = 64; i < span; i += 64) {
      const int next = load_ids(i);
      if (i + lane < span && (unsigned)next < (unsigned)p.c.n_pages) {
        const float vs = p.c.v_scale[(size_t)next * p.c.hkv + h];
        most = fmaxf(most, vs);
        least = vs > 0.f ? fminf(least, vs) : least;
        odd |= !(vs >= 0.f);
      }
    }
#pragma unroll
    for (int m = 32; m; m >>= 1) most = fmaxf(most, __shfl_xor(most, m));
    if (__ballot(odd || least * kHalfSpread < most) == 0) {
      unit = most;
      per_unit = most > 0.f ? 1.f / most : 0.f;
      run(HalfWeights{});
    } else {
      run(BfWeights<2>{});
    }
  } else {
    run(BfWeights<3>{});
  }

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
