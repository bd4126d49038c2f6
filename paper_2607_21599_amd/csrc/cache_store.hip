// Rows into and out of the paged 8-bit K/V cache (daf_cache_write, daf_cache_read).
//
// A value x is held as code * s, code in e4m3, s a power of two per page and head:
// s = 2^e with the smallest e >= -100 for which max |x| <= 448 * 2^e. Dividing by s
// is exact, so a code's only rounding is that of e4m3 (half a step: 2^-4 of the
// value for normal codes), and where a later row raises s the codes that stay
// change only if they leave the normal range.
//
// A workgroup owns one page of one head, so that the page's maxima, its scale and
// the 64-byte lines of the transposed V (64 tokens of one feature) have one
// writer. K rows go 16 bytes of input per lane; for V a lane takes two features and
// 16 (D = 64: 8) consecutive slots, so that its transposed bytes are whole 16-byte
// pieces without a pass through LDS. Both are loaded before the maxima are taken.
// Bound by HBM for long runs of rows, by latency for a few.
#include "cache.h"

namespace daf {
namespace {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;

// Elements of one dtype: E of them as 32-bit words in memory.
template <bool BF16>
struct Elem;
template <>
struct Elem<true> {
  static constexpr int kBytes = 2;
  static constexpr float kMax = 3.38953139e38f;  // 0x7f7f
  template <int N>
  static __device__ __forceinline__ void load(const unsigned char *p, float (&x)[N]) {
    unsigned w[N / 2];
    if constexpr (N == 8) {
      const u32x4 v = *reinterpret_cast<const u32x4 *>(p);
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = v[i];
    } else {
      w[0] = *reinterpret_cast<const unsigned *>(p);
    }
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
      x[2 * i] = __builtin_bit_cast(float, w[i] << 16);
      x[2 * i + 1] = __builtin_bit_cast(float, w[i] & 0xffff0000u);
    }
  }
  // values that bf16 holds exactly (NaN keeps a set mantissa bit of the upper half)
  template <int N>
  static __device__ __forceinline__ void store(unsigned char *p, const float (&x)[N]) {
    unsigned w[N / 2];
#pragma unroll
    for (int i = 0; i < N / 2; ++i)
      w[i] = (__builtin_bit_cast(unsigned, x[2 * i]) >> 16) | (__builtin_bit_cast(unsigned, x[2 * i + 1]) & 0xffff0000u);
    if constexpr (N == 8)
      *reinterpret_cast<u32x4 *>(p) = u32x4{w[0], w[1], w[2], w[3]};
    else
      *reinterpret_cast<unsigned *>(p) = w[0];
  }
};
template <>
struct Elem<false> {
  static constexpr int kBytes = 4;
  static constexpr float kMax = 3.402823466e38f;
  template <int N>
  static __device__ __forceinline__ void load(const unsigned char *p, float (&x)[N]) {
    if constexpr (N == 8) {
      const f32x4 a = *reinterpret_cast<const f32x4 *>(p), b = *reinterpret_cast<const f32x4 *>(p + 16);
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = a[i], x[4 + i] = b[i];
    } else {
      const f32x2 a = *reinterpret_cast<const f32x2 *>(p);
      x[0] = a[0], x[1] = a[1];
    }
  }
  template <int N>
  static __device__ __forceinline__ void store(unsigned char *p, const float (&x)[N]) {
    if constexpr (N == 8) {
      *reinterpret_cast<f32x4 *>(p) = f32x4{x[0], x[1], x[2], x[3]};
      *reinterpret_cast<f32x4 *>(p + 16) = f32x4{x[4], x[5], x[6], x[7]};
    } else {
      *reinterpret_cast<f32x2 *>(p) = f32x2{x[0], x[1]};
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

__device__ __forceinline__ float limited(float x, float most) {
  return x > most ? most : x < -most ? -most : x;  // NaN passes
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

__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
  for (int m = 32; m; m >>= 1) x = fmaxf(x, __shfl_xor(x, m));
  return x;
}

struct Shared {
  int row[kPage];      // per slot: the request's row that lies there, or -1
  float top[2][4];     // per wave: largest magnitude of K and V
  float scale[2];      // present scales
};

// One page of one head: the rows in sh.row (set, and a barrier passed). `held`:
// tokens of the page that the sequence had before (write).
template <bool BF16, int D, bool WRITE>
__device__ __forceinline__ void do_page(const StoreLaunch &p, Shared &sh, int64_t row0, int h, int page, int tokens,
                                        int held) {
  using E = Elem<BF16>;
  constexpr int CH = D / 8, SPP = kThreads / CH, PASSES = kPage / SPP;  // K: 8 elements per lane
  constexpr int LPR = D / 2, SPT = 16 * D / 128;                        // V: 2 features, SPT slots per lane
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const size_t rowb = (size_t)p.c.hkv * D * E::kBytes;
  const bool there = (unsigned)page < (unsigned)p.c.n_pages;
  const size_t blk = there ? (size_t)page * p.c.hkv + h : 0;
  unsigned char *kp = p.c.k + blk * (kPage * D), *vp = p.c.v + blk * (kPage * D);
  const int slot0 = wave * 16 + lane / LPR * SPT, d0 = lane % LPR * 2;

  const int mine = sh.row[lane];
  const unsigned long long asked = __ballot(mine >= 0);
  // rows that can be moved: below the sequence's tokens, in a page that is there
  const unsigned long long have = !there ? 0ull : tokens >= 64 ? ~0ull : (1ull << max(tokens, 0)) - 1;
  const unsigned long long go = asked & have;
  const unsigned wave_go = (unsigned)(go >> (16 * wave)) & 0xffffu, wave_asked = (unsigned)(asked >> (16 * wave)) & 0xffffu;

  if constexpr (WRITE) {
    if (!go) return;  // uniform in the workgroup
    const bool kept = ((held >= 64 ? ~0ull : (1ull << held) - 1) & ~go) != 0;
    float kx[PASSES][8], vx[SPT][2];
    float top_k = 0.f, top_v = 0.f;
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
      const int slot = i * SPP + t / CH;
      if ((go >> slot) & 1)
        E::template load<8>((const unsigned char *)p.k + (row0 + sh.row[slot]) * rowb + (size_t)h * D * E::kBytes +
                                t % CH * 8 * E::kBytes, kx[i]);
    }
#pragma unroll
    for (int s = 0; s < SPT; ++s)
      if ((go >> (slot0 + s)) & 1)
        E::template load<2>((const unsigned char *)p.v + (row0 + sh.row[slot0 + s]) * rowb +
                                ((size_t)h * D + d0) * E::kBytes, vx[s]);
    // the V bytes that stay, where this wave's slots take a new row
    unsigned old_v[2][SPT / 4];
    const bool merge = kept && wave_go;
    auto load_old = [&] {
#pragma unroll
      for (int f = 0; f < 2; ++f)
#pragma unroll
        for (int j = 0; j < SPT / 4; ++j)
          old_v[f][j] = reinterpret_cast<const unsigned *>(vp + (d0 + f) * kPage + slot0)[j];
    };
    if (merge) load_old();
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
      const int slot = i * SPP + t / CH;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        kx[i][j] = (go >> slot) & 1 ? limited(kx[i][j], E::kMax) : 0.f;
        top_k = fmaxf(top_k, fabsf(kx[i][j]));
      }
    }
#pragma unroll
    for (int s = 0; s < SPT; ++s)
#pragma unroll
      for (int f = 0; f < 2; ++f) {
        vx[s][f] = (go >> (slot0 + s)) & 1 ? limited(vx[s][f], E::kMax) : 0.f;
        top_v = fmaxf(top_v, fabsf(vx[s][f]));
      }
    top_k = wave_max(top_k);
    top_v = wave_max(top_v);
    if (lane == 0) sh.top[0][wave] = top_k, sh.top[1][wave] = top_v;
    if (t == 0) sh.scale[0] = p.c.k_scale[blk], sh.scale[1] = p.c.v_scale[blk];
    __syncthreads();
    float s0[2], s1[2], inv[2], ratio[2];
#pragma unroll
    for (int f = 0; f < 2; ++f) {
      const float top = fmaxf(fmaxf(sh.top[f][0], sh.top[f][1]), fmaxf(sh.top[f][2], sh.top[f][3]));
      s0[f] = kept ? sh.scale[f] : 0.f;
      s1[f] = fmaxf(s0[f], scale_for(top));
      inv[f] = inverse(s1[f]);
      ratio[f] = s0[f] * inv[f];
    }
    if (t == 0) p.c.k_scale[blk] = s1[0], p.c.v_scale[blk] = s1[1];
    const bool grow_k = kept && s1[0] > s0[0], grow_v = kept && s1[1] > s0[1];
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
      const int slot = i * SPP + t / CH;
      u32x2 *dst = reinterpret_cast<u32x2 *>(kp + slot * D + t % CH * 8);
      if (!kept || ((go >> slot) & 1)) {  // zeros where no row goes
        const float *x = kx[i];
        *dst = u32x2{to_codes(x[0] * inv[0], x[1] * inv[0], x[2] * inv[0], x[3] * inv[0]),
                     to_codes(x[4] * inv[0], x[5] * inv[0], x[6] * inv[0], x[7] * inv[0])};
      } else if (grow_k) {
        const u32x2 w = *dst;
        *dst = u32x2{rescale(w[0], ratio[0]), rescale(w[1], ratio[0])};
      }
    }
    if (kept && !wave_go && !grow_v) return;
    if (grow_v && !merge) load_old();
#pragma unroll
    for (int f = 0; f < 2; ++f) {
      unsigned w[SPT / 4];
#pragma unroll
      for (int j = 0; j < SPT / 4; ++j) {
        w[j] = to_codes(vx[4 * j][f] * inv[1], vx[4 * j + 1][f] * inv[1], vx[4 * j + 2][f] * inv[1],
                        vx[4 * j + 3][f] * inv[1]);
        if (kept) {
          unsigned m = (unsigned)(go >> (slot0 + 4 * j)) & 15u;  // new rows among the four slots, as bytes
          m = ((m & 1) | (m & 2) << 7 | (m & 4) << 14 | (m & 8) << 21) * 255u;
          const unsigned stay = grow_v ? rescale(old_v[f][j], ratio[1]) : old_v[f][j];
          w[j] = (w[j] & m) | (stay & ~m);
        }
      }
      unsigned *dst = reinterpret_cast<unsigned *>(vp + (d0 + f) * kPage + slot0);
      if constexpr (SPT == 16)
        *reinterpret_cast<u32x4 *>(dst) = u32x4{w[0], w[1], w[2], w[3]};
      else
        *reinterpret_cast<u32x2 *>(dst) = u32x2{w[0], w[1]};
    }
  } else {
    if (!asked) return;
    if (p.k) {
      const float s = there ? p.c.k_scale[blk] : 0.f;
#pragma unroll
      for (int i = 0; i < PASSES; ++i) {
        const int slot = i * SPP + t / CH;
        if (!((asked >> slot) & 1)) continue;
        float x[8] = {};
        if ((go >> slot) & 1) {
          const u32x2 w = *reinterpret_cast<const u32x2 *>(kp + slot * D + t % CH * 8);
          from_codes(w[0], x);
          from_codes(w[1], x + 4);
#pragma unroll
          for (int j = 0; j < 8; ++j) x[j] *= s;
        }
        E::template store<8>((unsigned char *)p.k + (row0 + sh.row[slot]) * rowb + (size_t)h * D * E::kBytes +
                                 t % CH * 8 * E::kBytes, x);
      }
    }
    if (p.v && wave_asked) {
      const float s = there ? p.c.v_scale[blk] : 0.f;
      float x[SPT][2] = {};
      if (wave_go) {
#pragma unroll
        for (int f = 0; f < 2; ++f)
#pragma unroll
          for (int j = 0; j < SPT / 4; ++j) {
            float y[4];
            from_codes(reinterpret_cast<const unsigned *>(vp + (d0 + f) * kPage + slot0)[j], y);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[4 * j + e][f] = (go >> (slot0 + 4 * j + e)) & 1 ? y[e] * s : 0.f;
          }
      }
#pragma unroll
      for (int i = 0; i < SPT; ++i)
        if ((asked >> (slot0 + i)) & 1)
          E::template store<2>((unsigned char *)p.v + (row0 + sh.row[slot0 + i]) * rowb +
                                   ((size_t)h * D + d0) * E::kBytes, x[i]);
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
  const int h = blockIdx.x % p.c.hkv, unit = blockIdx.x / p.c.hkv;
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
    do_page<BF16, D, WRITE>(p, sh, row0, h, page_of(pg), pg < 0 ? 0 : min(L - pg * kPage, kPage), held);
    return;
  }
  const int32_t *pos = p.pos + row0;
  for (int r = u * kStoreRows, end = min(n, r + kStoreRows); r < end; ++r) {
    const int pg = pos[r] >> 6;
    if (r > 0 && pos[r - 1] >> 6 == pg) continue;
    __syncthreads();  // the page before is done with sh
    if (t < kPage) sh.row[t] = -1;
    __syncthreads();
    if (t < kPage && r + t < n && pos[r + t] >> 6 == pg) sh.row[pos[r + t] & 63] = r + t;
    __syncthreads();
    const int tokens = pg < 0 || (int64_t)pg * kPage >= L ? 0 : min(L - pg * kPage, kPage);
    do_page<BF16, D, WRITE>(p, sh, row0, h, page_of(pg), tokens, tokens);
  }
}

}  // namespace

hipError_t launch_cache_store(bool write, bool bf16, const StoreLaunch &p, hipStream_t st) {
  const int grid = p.units * p.c.hkv;
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
