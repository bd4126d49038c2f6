// Rows into and out of the paged 8-bit K/V cache (daf_cache_write, daf_cache_read).
//
// A value x is held as code * s, code in e4m3, s a power of two per page and head:
// s = 2^e with the smallest e >= -100 for which max |x| <= 448 * 2^e. Dividing by s
// is exact, so a code's only rounding is that of e4m3 (half a step: 2^-4 of the
// value for normal codes), and where a later row raises s the codes that stay
// change only if they leave the normal range.
//
// A workgroup owns K or V of one page of one head, so that the page's maximum, its
// scale and the 64-byte lines of the transposed V (64 tokens of one feature) have
// one writer. K goes 8 elements per lane; for V a lane takes two features of 16
// (D = 64: 8) consecutive slots, so that its transposed codes are whole pieces
// without a pass through LDS. All rows are loaded before the maximum is taken.
// Bound by HBM for long runs of rows: 32768 rows of 4 heads of 128 (67 MB in bf16, 34 MB
// of codes) are written in 28 us and read back in 17; by latency for scattered ones
// (4915 rows over 512 pages, 57 MB, 23 us: chains of dependent loads, a page's at a
// time, of which more rows per unit or fewer took as long) and for a few (32 rows 4.9 and
// 3.5 us).
#include "cache.h"

namespace daf {
namespace {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = kStoreThreads;

// Rows of one dtype, held as they are in memory until they are converted: N elements
// in words() 32-bit words.
template <bool BF16>
struct Elem {
  static constexpr int kBytes = BF16 ? 2 : 4;
  static constexpr float kMax = BF16 ? 3.38953139e38f : 3.402823466e38f;  // largest finite value
  static constexpr int words(int n) { return n * kBytes / 4; }
  // N * kBytes bytes at p, which is aligned to them or to 16
  template <int N>
  static __device__ __forceinline__ void load(const unsigned char *p, unsigned (&w)[words(N)]) {
    constexpr int W = words(N);
    if constexpr (W >= 4) {
#pragma unroll
      for (int i = 0; i < W / 4; ++i) {
        const u32x4 v = reinterpret_cast<const u32x4 *>(p)[i];
#pragma unroll
        for (int j = 0; j < 4; ++j) w[4 * i + j] = v[j];
      }
    } else if constexpr (W == 2) {
      const u32x2 v = *reinterpret_cast<const u32x2 *>(p);
      w[0] = v[0], w[1] = v[1];
    } else {
      w[0] = *reinterpret_cast<const unsigned *>(p);
    }
  }
  // element i; LIMITED: infinities as the largest finite value, NaN as it is
  template <bool LIMITED, int W>
  static __device__ __forceinline__ float get(const unsigned (&w)[W], int i) {
    const unsigned u = !BF16 ? w[i] : i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16;
    const float x = __builtin_bit_cast(float, u);
    return !LIMITED ? x : x > kMax ? kMax : x < -kMax ? -kMax : x;
  }
  // the larger of m and the magnitudes in w, as bits, per half in bf16
  static __device__ __forceinline__ unsigned max_bits(unsigned m, unsigned w) {
    if constexpr (!BF16) return max(m, w & 0x7fffffffu);
    return __builtin_bit_cast(unsigned, __builtin_elementwise_max(__builtin_bit_cast(u16x2, m),
                                                                  __builtin_bit_cast(u16x2, w & 0x7fff7fffu)));
  }
  // the same as the bits of one fp32 value
  static __device__ __forceinline__ unsigned whole(unsigned m) {
    return !BF16 ? m : max(m & 0xffff0000u, m << 16);
  }
  // values that the dtype holds exactly (a NaN keeps a set mantissa bit)
  template <int N>
  static __device__ __forceinline__ void store(unsigned char *p, const float (&x)[N]) {
    constexpr int W = words(N);
    unsigned w[W];
#pragma unroll
    for (int i = 0; i < W; ++i)
      w[i] = !BF16 ? __builtin_bit_cast(unsigned, x[i])
                   : __builtin_bit_cast(unsigned, x[2 * i]) >> 16 | (__builtin_bit_cast(unsigned, x[2 * i + 1]) & 0xffff0000u);
    if constexpr (W >= 4) {
#pragma unroll
      for (int i = 0; i < W / 4; ++i)
        reinterpret_cast<u32x4 *>(p)[i] = u32x4{w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]};
    } else if constexpr (W == 2) {
      *reinterpret_cast<u32x2 *>(p) = u32x2{w[0], w[1]};
    } else {
      *reinterpret_cast<unsigned *>(p) = w[0];
    }
  }
};

// four values to codes / four codes to values (nearest even; NaN stays NaN)
__device__ __forceinline__ unsigned to_codes(float a, float b, float c, float d) {
#if defined(__HIP_DEVICE_COMPILE__)
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return __builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
#else
  return 0;
#endif
}
__device__ __forceinline__ void from_codes(unsigned w, float *x) {
#if defined(__HIP_DEVICE_COMPILE__)
  const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
  x[0] = a[0], x[1] = a[1], x[2] = b[0], x[3] = b[1];
#endif
}
__device__ __forceinline__ unsigned rescale(unsigned w, float ratio) {
  float x[4];
  from_codes(w, x);
  return to_codes(x[0] * ratio, x[1] * ratio, x[2] * ratio, x[3] * ratio);
}

// The smallest power of two >= 2^kMinScaleExp under which top is at most 448 =
// 1.75 * 2^8; 0 for 0. From the bits of top, so exact.
__device__ __forceinline__ float scale_for(float top) {
  if (top == 0.f) return 0.f;
  const unsigned u = __builtin_bit_cast(unsigned, top);
  const int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
  return __builtin_bit_cast(float, (unsigned)(max(e, kMinScaleExp) + 127) << 23);
}
// 1 / s of a power of two in [2^-100, 2^120], 0 for 0
__device__ __forceinline__ float inverse(float s) {
  return s == 0.f ? 0.f : __builtin_bit_cast(float, (254u << 23) - __builtin_bit_cast(unsigned, s));
}

__device__ __forceinline__ unsigned wave_max(unsigned x) {
#pragma unroll
  for (int m = 32; m; m >>= 1) x = max(x, (unsigned)__shfl_xor((int)x, m));
  return x;
}

struct Shared {
  int row[kPage];  // per slot: the request's row that lies there, or -1
  unsigned top[2][4];  // per wave: largest magnitude, its bits; the same of finite ones
  float scale;     // present scale
};

// A lane's share of K or V of a page. A lane has PASSES pieces of N elements of a
// row. K: 8 features of every SPP-th slot. V: 2 features of PASSES consecutive
// slots, so that its codes are whole 16-byte (D = 64: 8-byte) pieces of the
// transposed page, Q words of four.
template <int D, bool IS_V>
struct Share {
  static constexpr int N = IS_V ? 2 : 8, CH = D / 8, SPP = kThreads / CH;
  static constexpr int PASSES = IS_V ? 16 * D / 128 : kPage / SPP, LPS = kPage / PASSES;
  static constexpr int Q = IS_V ? PASSES / 4 : 1;
};

// Codes of the rows in x (those in `mine`; zeros elsewhere) into the page; kept codes
// stay, times `ratio` where the scale grew.
template <bool BF16, int D, bool IS_V, bool LIMITED, typename X, typename Old>
__device__ __forceinline__ void put(const X &x, Old &old, unsigned char *codes, unsigned mine, bool kept, bool grow,
                                    float inv, float ratio, int slot0, int d0) {
  using E = Elem<BF16>;
  using S = Share<D, IS_V>;
  if constexpr (!IS_V) {
#pragma unroll
    for (int i = 0; i < S::PASSES; ++i) {
      u32x2 *dst = reinterpret_cast<u32x2 *>(codes + (slot0 + i * S::SPP) * D + d0);
      if (!kept || ((mine >> i) & 1)) {  // zeros where no row goes
        float y[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = E::template get<LIMITED>(x[i], j) * inv;
        *dst = u32x2{to_codes(y[0], y[1], y[2], y[3]), to_codes(y[4], y[5], y[6], y[7])};
      } else if (grow) {
        const u32x2 w = *dst;
        *dst = u32x2{rescale(w[0], ratio), rescale(w[1], ratio)};
      }
    }
  } else {
    if (kept && !mine && !grow) return;
    if (grow && !mine)
#pragma unroll
      for (int f = 0; f < 2; ++f) Elem<false>::template load<S::Q>(codes + (d0 + f) * kPage + slot0, old[f]);
#pragma unroll
    for (int f = 0; f < 2; ++f) {
      unsigned w[S::Q];
#pragma unroll
      for (int j = 0; j < S::Q; ++j) {
        float y[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = E::template get<LIMITED>(x[4 * j + e], f) * inv;
        w[j] = to_codes(y[0], y[1], y[2], y[3]);
        if (kept) {
          unsigned m = (mine >> 4 * j) & 15u;  // new rows among the four slots, as bytes
          m = ((m & 1) | (m & 2) << 7 | (m & 4) << 14 | (m & 8) << 21) * 255u;
          const unsigned stay = grow ? rescale(old[f][j], ratio) : old[f][j];
          w[j] = (w[j] & m) | (stay & ~m);
        }
      }
      unsigned *dst = reinterpret_cast<unsigned *>(codes + (d0 + f) * kPage + slot0);
      if constexpr (S::PASSES == 16)
        *reinterpret_cast<u32x4 *>(dst) = u32x4{w[0], w[1], w[2], w[3]};
      else
        *reinterpret_cast<u32x2 *>(dst) = u32x2{w[0], w[1]};
    }
  }
}

// K (IS_V false) or V of one page of one head: the rows in sh.row (set, and a
// barrier passed). tokens: of the page, at the call's end; held: before it (write).
template <bool BF16, int D, bool WRITE, bool IS_V>
__device__ __forceinline__ void do_page(const StoreLaunch &p, Shared &sh, int64_t row0, int h, int page, int tokens,
                                        int held) {
  using E = Elem<BF16>;
  using S = Share<D, IS_V>;
  constexpr int N = S::N, CH = S::CH, SPP = S::SPP, PASSES = S::PASSES, LPS = S::LPS, Q = S::Q;
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const size_t rowb = (size_t)p.c.hkv * D * E::kBytes;
  const bool there = (unsigned)page < (unsigned)p.c.n_pages;
  const size_t blk = there ? (size_t)page * p.c.hkv + h : 0;
  unsigned char *codes = (IS_V ? p.c.v : p.c.k) + blk * (kPage * D);
  float *scale = (IS_V ? p.c.v_scale : p.c.k_scale) + blk;
  // V: when writing, LPS neighbouring lanes hold the 64 tokens of two features (whole
  // 64-byte lines of codes), when reading, the lanes of D / 2 hold a row
  const int slot0 = !IS_V ? t / CH : WRITE ? lane % LPS * PASSES : (t / (D / 2)) * PASSES;
  const int d0 = !IS_V ? t % CH * 8 : WRITE ? (wave * (64 / LPS) + lane / LPS) * 2 : t % (D / 2) * 2;
  auto slot = [&](int i) { return IS_V ? slot0 + i : slot0 + i * SPP; };
  const unsigned char *rows = static_cast<const unsigned char *>(IS_V ? p.v : p.k);
  auto at = [&](int i) { return rows + (row0 + sh.row[slot(i)]) * rowb + ((size_t)h * D + d0) * E::kBytes; };

  const unsigned long long asked = __ballot(sh.row[lane] >= 0);
  // rows that can be moved: below the sequence's tokens, in a page that is there
  const unsigned long long can = asked & (tokens >= 64 ? ~0ull : (1ull << max(tokens, 0)) - 1);
  const unsigned long long go = there ? can : 0ull;
  auto bits = [&](unsigned long long m) {  // of this lane's slots
    if constexpr (IS_V) return (unsigned)(m >> slot0) & ((1u << PASSES) - 1);
    unsigned r = 0;
#pragma unroll
    for (int i = 0; i < PASSES; ++i) r |= ((unsigned)(m >> slot(i)) & 1) << i;
    return r;
  };
  const unsigned mine = bits(go);

  if constexpr (WRITE) {
    unsigned x[PASSES][E::words(N)] = {};
    const unsigned rows_mine = bits(can);  // not `go`: these loads need not wait for the page's id
#pragma unroll
    for (int i = 0; i < PASSES; ++i)
      if ((rows_mine >> i) & 1) E::template load<N>(at(i), x[i]);
    if (!go) return;  // uniform in the workgroup
    float present = 0.f;
    if (t == 0) present = *scale;
    const bool kept = ((held >= 64 ? ~0ull : (1ull << held) - 1) & ~go) != 0;
    // V: the codes that stay beside a new one in a piece
    unsigned old[2][Q] = {};
    auto load_old = [&] {
#pragma unroll
      for (int f = 0; f < 2; ++f) Elem<false>::template load<Q>(codes + (d0 + f) * kPage + slot0, old[f]);
    };
    if constexpr (IS_V)
      if (kept && mine) load_old();
    unsigned top = 0;
#pragma unroll
    for (int i = 0; i < PASSES; ++i)
#pragma unroll
      for (int j = 0; j < E::words(N); ++j) top = E::max_bits(top, x[i][j]);
    top = wave_max(E::whole(top));
    if (lane == 0) sh.top[0][wave] = top;
    if (t == 0) sh.scale = present;
    __syncthreads();
    top = max(max(sh.top[0][0], sh.top[0][1]), max(sh.top[0][2], sh.top[0][3]));
    const bool special = top >= 0x7f800000u;  // infinities or NaN among the rows
    if (special) {
      float m = 0.f;
#pragma unroll
      for (int i = 0; i < PASSES; ++i)
#pragma unroll
        for (int j = 0; j < N; ++j) m = fmaxf(m, fabsf(E::template get<true>(x[i], j)));
      top = wave_max(__builtin_bit_cast(unsigned, m));
      if (lane == 0) sh.top[1][wave] = top;
      __syncthreads();
      top = max(max(sh.top[1][0], sh.top[1][1]), max(sh.top[1][2], sh.top[1][3]));
    }
    const float s0 = kept ? sh.scale : 0.f;
    const float s1 = fmaxf(s0, scale_for(__builtin_bit_cast(float, top)));
    const float inv = inverse(s1), ratio = s0 * inv;
    const bool grow = kept && s1 > s0;
    if (t == 0) *scale = s1;
    special ? put<BF16, D, IS_V, true>(x, old, codes, mine, kept, grow, inv, ratio, slot0, d0)
            : put<BF16, D, IS_V, false>(x, old, codes, mine, kept, grow, inv, ratio, slot0, d0);
  } else {
    const unsigned out = bits(asked);
    if (!out) return;
    const float s = there ? *scale : 0.f;
    if constexpr (!IS_V) {
      u32x2 w[PASSES] = {};
#pragma unroll
      for (int i = 0; i < PASSES; ++i)
        if ((mine >> i) & 1) w[i] = *reinterpret_cast<const u32x2 *>(codes + slot(i) * D + d0);
#pragma unroll
      for (int i = 0; i < PASSES; ++i) {
        if (!((out >> i) & 1)) continue;
        float x[8];
        from_codes(w[i][0], x);
        from_codes(w[i][1], x + 4);
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] *= s;
        E::template store<8>(const_cast<unsigned char *>(at(i)), x);
      }
    } else {
      unsigned w[2][Q] = {};
#pragma unroll
      for (int f = 0; f < 2; ++f)
        if (mine) Elem<false>::template load<Q>(codes + (d0 + f) * kPage + slot0, w[f]);
#pragma unroll
      for (int j = 0; j < Q; ++j) {
        float a[4], b[4];
        from_codes(w[0][j], a);
        from_codes(w[1][j], b);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int i = 4 * j + e;
          const bool ok = (mine >> i) & 1;
          const float x[2] = {ok ? a[e] * s : 0.f, ok ? b[e] * s : 0.f};
          if ((out >> i) & 1) E::template store<2>(const_cast<unsigned char *>(at(i)), x);
        }
      }
    }
  }
}

// Units of a request: with positions, kStoreRows rows each, of which every one that
// is its page's first takes the page; else one page each of those that its n last
// rows can touch.
template <bool BF16, int D, bool WRITE>
__global__ __launch_bounds__(kThreads) void cache_store_kernel(const StoreLaunch p) {
  __shared__ Shared sh;
  const int t = threadIdx.x;
  const int half = p.units * p.c.hkv;  // workgroups of K, then those of V
  const bool is_v = (int)blockIdx.x >= half || !p.k;
  const int job = (int)blockIdx.x >= half ? blockIdx.x - half : blockIdx.x;
  const int h = job % p.c.hkv, unit = job / p.c.hkv;
  int b = 0;
  if (p.per_req) {
    b = unit / p.per_req;
  } else {
    for (int step = kMaxCacheReqs / 2; step; step >>= 1)
      if (b + step < p.n_req && p.unit0[b + step] <= unit) b += step;
  }
  const int u = unit - (p.per_req ? b * p.per_req : p.unit0[b]);
  const int row0 = p.cu[b], n = p.cu[b + 1] - row0;
  const int seq = p.seq ? p.seq[b] : b;
  const int L = seq_len(p.c.len, p.c.n_seqs, p.c.max_seq_pages, seq);
  const int32_t *pages = p.c.table + (int64_t)((unsigned)seq < (unsigned)p.c.n_seqs ? seq : 0) * p.c.max_seq_pages;
  auto page_of = [&](int pg) {  // L is 0 for a sequence out of range
    return pg >= 0 && (int64_t)pg * kPage < L ? pages[pg] : -1;
  };
  if (!p.pos) {
    const int64_t first = (int64_t)L - n;
    const int64_t pg64 = (first >> 6) + u;  // may lie before the sequence
    if (pg64 * kPage >= L) return;
    if (t < kPage) {
      const int64_t j = pg64 * kPage + t - first;
      sh.row[t] = j >= 0 && j < n ? (int)j : -1;
    }
    __syncthreads();
    const int pg = (int)(pg64 < 0 ? -1 : pg64);
    const int held = (int)min(max(first - pg64 * kPage, (int64_t)0), (int64_t)kPage);
    const int tokens = pg < 0 ? 0 : min(L - pg * kPage, kPage);
    is_v ? do_page<BF16, D, WRITE, true>(p, sh, row0, h, page_of(pg), tokens, held)
         : do_page<BF16, D, WRITE, false>(p, sh, row0, h, page_of(pg), tokens, held);
    return;
  }
  // which of the unit's rows are their page's first, from one load per lane
  const int32_t *pos = p.pos + row0;
  const int r0 = u * kStoreRows, lane = t & 63;
  const int mine = lane < kStoreRows && r0 + lane < n ? pos[r0 + lane] >> 6 : INT32_MIN;
  const int before = lane < kStoreRows && r0 + lane > 0 && r0 + lane < n ? pos[r0 + lane - 1] >> 6 : INT32_MAX;
  unsigned firsts = (unsigned)__ballot(lane < kStoreRows && r0 + lane < n && mine != before);
  for (; firsts; firsts &= firsts - 1) {
    const int i = __builtin_ctz(firsts), r = r0 + i;
    const int pg = __builtin_amdgcn_readlane(mine, i);
    __syncthreads();  // the page before is done with sh
    if (t < kPage) {
      sh.row[t] = -1;
      // same wave, in order
      const int at = r + t < n ? pos[r + t] : 0;
      if (r + t < n && at >> 6 == pg) sh.row[at & 63] = r + t;
    }
    __syncthreads();
    const int tokens = pg < 0 || (int64_t)pg * kPage >= L ? 0 : min(L - pg * kPage, kPage);
    is_v ? do_page<BF16, D, WRITE, true>(p, sh, row0, h, page_of(pg), tokens, tokens)
         : do_page<BF16, D, WRITE, false>(p, sh, row0, h, page_of(pg), tokens, tokens);
  }
}

}  // namespace

hipError_t launch_cache_store(bool write, bool bf16, const StoreLaunch &p, hipStream_t st) {
  const unsigned grid = (unsigned)p.units * p.c.hkv * (p.k && p.v ? 2 : 1);
  auto go = [&](auto kern) { kern<<<grid, kThreads, 0, st>>>(p); };
  if (p.c.d == 128) {
    if (bf16) write ? go(cache_store_kernel<true, 128, true>) : go(cache_store_kernel<true, 128, false>);
    else write ? go(cache_store_kernel<false, 128, true>) : go(cache_store_kernel<false, 128, false>);
  } else {
    if (bf16) write ? go(cache_store_kernel<true, 64, true>) : go(cache_store_kernel<true, 64, false>);
    else write ? go(cache_store_kernel<false, 64, true>) : go(cache_store_kernel<false, 64, false>);
  }
  return hipGetLastError();
}

}  // namespace daf
