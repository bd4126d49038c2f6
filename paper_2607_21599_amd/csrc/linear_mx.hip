// Projections of few rows with weights in 4 bits (daf_linear_mx): C = A W^T (+ bias)
// (+ residual), W as e2m1 codes with a power-of-two scale per 32 of a row, A in bf16 or
// as e4m3 codes with such scales (daf_add_rmsnorm).
//
// Codes times their scale become bf16 by one conversion instruction per two values, exactly,
// so the products of v_mfma_f32_16x16x32_bf16 are exact and sums are fp32. (The
// instruction that takes the codes and scales themselves keeps about 13 bits of a small
// term beside a large one.)
//
// A wave has 16 NT rows of W (output features) and 16 MT rows of A, and takes K in
// turns of 256, the waves of a workgroup one after the other, from memory to registers
// in operand layout: lane (n, g) reads 16 bytes of row n, the 32 values with one scale at
// k = 32 g of 128, which are four operands of 8 values; A is read in the same order
// of k. The waves' sums are joined through LDS in a fixed order.
#include "step.h"

namespace daf {
namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ f32x4 mfma(const bf16x8 &a, const bf16x8 &b, const f32x4 &c) {
#if defined(__HIP_DEVICE_COMPILE__)
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
#else
  return c;
#endif
}

// 2^(b - 127) of a scale's byte, which counts as one of 27 .. 247 (2^-100 .. 2^120) so that
// no value of a code is lost or infinite; 255 is NaN
__device__ __forceinline__ float scale_of(unsigned b) {
  const unsigned e = b == 255 ? 0x7fc00000u : min(max(b, 27u), 247u) << 23;
  return __builtin_bit_cast(float, e);
}

// eight e2m1 codes (the low half of a byte first) times a scale
__device__ __forceinline__ bf16x8 widen4(unsigned w, float scale) {
#if defined(__HIP_DEVICE_COMPILE__)
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
#else
  return bf16x8{};
#endif
}
// eight e4m3 codes times a scale
__device__ __forceinline__ bf16x8 widen8(unsigned lo, unsigned hi, float scale) {
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

// A lane's 32 values of a row of A at one k
template <bool MX>
struct RowsA {
  u32x4 x[MX ? 2 : 4];
  float scale;
  __device__ __forceinline__ void load(const MxLaunch &p, size_t row, int k) {
    const unsigned char *at = p.a + (row * p.k + k) * (MX ? 1 : 2);
#pragma unroll
    for (int i = 0; i < (MX ? 2 : 4); ++i) x[i] = reinterpret_cast<const u32x4 *>(at)[i];
    if constexpr (MX) scale = scale_of(p.a_scales[row * (p.k / kBlockValues) + k / kBlockValues]);
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < (MX ? 2 : 4); ++i) x[i] = u32x4{};
    scale = 1.f;
  }
  __device__ __forceinline__ bf16x8 operand(int j) const {
    if constexpr (MX) return widen8(x[j / 2][j % 2 * 2], x[j / 2][j % 2 * 2 + 1], scale);
    else return __builtin_bit_cast(bf16x8, x[j]);
  }
};

struct RowsW {
  u32x4 x;
  unsigned scale;
};

template <bool MX, int MT, int NT>
__global__ __launch_bounds__(64 * kMxWaves) void linear_mx_kernel(const MxLaunch p, int row_blocks) {
  __shared__ f32x4 sums[kMxWaves][NT][MT][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n16 = lane & 15, g = lane >> 4;
  const int n0 = blockIdx.x / row_blocks * (16 * NT);
  const int64_t m0 = (int64_t)(blockIdx.x % row_blocks) * (16 * MT);
  const int split = blockIdx.y;
  // rows past the end repeat the last one; nothing of theirs is stored
  size_t wrow[NT], arow[MT];
#pragma unroll
  for (int i = 0; i < NT; ++i) wrow[i] = min(n0 + 16 * i + n16, p.n - 1);
#pragma unroll
  for (int i = 0; i < MT; ++i) arow[i] = min(m0 + 16 * i + n16, p.m - 1);
  const int units = (p.k + kMxUnit - 1) / kMxUnit;
  const int u0 = (int)((int64_t)units * split / p.splits), u1 = (int)((int64_t)units * (split + 1) / p.splits);

  f32x4 acc[NT][MT] = {};
  RowsW w[2][2][NT];
  RowsA<MX> a[2][2][MT];
  auto load = [&](int buf, int u) {
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const int k = u * kMxUnit + s * 128 + g * 32;
      const bool in = k < p.k;  // past the end: zeros of A beside weights of the row
      const int kc = in ? k : 0;
#pragma unroll
      for (int i = 0; i < NT; ++i) {
        w[buf][s][i].x = *reinterpret_cast<const u32x4 *>(p.w + (wrow[i] * p.k + kc) / 2);
        w[buf][s][i].scale = p.w_scales[wrow[i] * (p.k / kBlockValues) + kc / kBlockValues];
      }
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        a[buf][s][i].load(p, arow[i], kc);
        if (!in) a[buf][s][i].clear();
      }
    }
  };
  auto work = [&](int buf) {
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      float scale[NT];
#pragma unroll
      for (int i = 0; i < NT; ++i) scale[i] = scale_of(w[buf][s][i].scale);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        bf16x8 b[MT];
#pragma unroll
        for (int i = 0; i < MT; ++i) b[i] = a[buf][s][i].operand(j);
#pragma unroll
        for (int i = 0; i < NT; ++i) {
          const bf16x8 x = widen4(w[buf][s][i].x[j], scale[i]);
#pragma unroll
          for (int e = 0; e < MT; ++e) acc[i][e] = mfma(x, b[e], acc[i][e]);
        }
      }
    }
  };
  int u = u0 + wave;
  if (u < u1) load(0, u);
  for (; u < u1; u += 2 * kMxWaves) {
    if (u + kMxWaves < u1) load(1, u + kMxWaves);
    work(0);
    if (u + kMxWaves >= u1) break;
    if (u + 2 * kMxWaves < u1) load(0, u + 2 * kMxWaves);
    work(1);
  }
#pragma unroll
  for (int i = 0; i < NT; ++i)
#pragma unroll
    for (int e = 0; e < MT; ++e) sums[wave][i][e][lane] = acc[i][e];
  __syncthreads();
  // a thread has 4 features of a row
  for (int c = threadIdx.x; c < NT * MT * 64; c += 64 * kMxWaves) {
    const int i = c / 4 % NT, quad = c % 4, row = c / (4 * NT);
    const int64_t m = m0 + row;
    const int n = n0 + 16 * i + quad * 4;
    if (m >= p.m || n >= p.n) continue;
    f32x4 x = sums[0][i][row / 16][quad * 16 + row % 16];
#pragma unroll
    for (int k = 1; k < kMxWaves; ++k) x += sums[k][i][row / 16][quad * 16 + row % 16];
    if (p.splits > 1) {
      float *to = p.part + ((size_t)split * p.m + m) * p.n + n;
      if (p.n % 4 == 0) *reinterpret_cast<f32x4 *>(to) = x;
      else
        for (int k = 0; k < 4 && n + k < p.n; ++k) to[k] = x[k];
      continue;
    }
    const size_t at = (size_t)m * p.n + n;
    const __bf16 *bias = static_cast<const __bf16 *>(p.bias), *res = static_cast<const __bf16 *>(p.residual);
    __bf16 *to = static_cast<__bf16 *>(p.c) + at;
    if (p.n % 4 == 0) {
      if (bias) {
        const bf16x4 v = *reinterpret_cast<const bf16x4 *>(bias + n);
#pragma unroll
        for (int k = 0; k < 4; ++k) x[k] += (float)v[k];
      }
      if (res) {
        const bf16x4 v = *reinterpret_cast<const bf16x4 *>(res + at);
#pragma unroll
        for (int k = 0; k < 4; ++k) x[k] += (float)v[k];
      }
      *reinterpret_cast<bf16x4 *>(to) = bf16x4{(__bf16)x[0], (__bf16)x[1], (__bf16)x[2], (__bf16)x[3]};
    } else {
      for (int k = 0; k < 4 && n + k < p.n; ++k) {
        float y = x[k];
        if (bias) y += (float)bias[n + k];
        if (res) y += (float)res[at + k];
        to[k] = (__bf16)y;
      }
    }
  }
}

// The sum of the splits, in their order.
__global__ __launch_bounds__(256) void linear_mx_join_kernel(const MxLaunch p) {
  const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x, total = p.m * p.n;
  if (at >= total) return;
  float x = p.part[at];
  for (int s = 1; s < p.splits; ++s) x += p.part[s * total + at];
  if (p.bias) x += (float)static_cast<const __bf16 *>(p.bias)[at % p.n];
  if (p.residual) x += (float)static_cast<const __bf16 *>(p.residual)[at];
  static_cast<__bf16 *>(p.c)[at] = (__bf16)x;
}

template <bool MX, int MT, int NT>
hipError_t launch(const MxLaunch &p, hipStream_t st) {
  const int row_blocks = (int)((p.m + 16 * MT - 1) / (16 * MT)), tiles = (p.n + 16 * NT - 1) / (16 * NT);
  linear_mx_kernel<MX, MT, NT><<<dim3((unsigned)((int64_t)tiles * row_blocks), p.splits), 64 * kMxWaves, 0, st>>>(p, row_blocks);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.splits == 1) return e;
  linear_mx_join_kernel<<<(unsigned)((p.m * p.n + 255) / 256), 256, 0, st>>>(p);
  return hipGetLastError();
}

template <bool MX>
hipError_t launch(const MxPlan &plan, const MxLaunch &p, hipStream_t st) {
  if (plan.mt == 1) return plan.nt == 1 ? launch<MX, 1, 1>(p, st) : plan.nt == 2 ? launch<MX, 1, 2>(p, st) : launch<MX, 1, 4>(p, st);
  if (plan.mt == 2) return plan.nt == 1 ? launch<MX, 2, 1>(p, st) : plan.nt == 2 ? launch<MX, 2, 2>(p, st) : launch<MX, 2, 4>(p, st);
  return plan.nt == 1 ? launch<MX, 4, 1>(p, st) : launch<MX, 4, 2>(p, st);
}

}  // namespace

MxPlan plan_linear_mx(int64_t m, int32_t n, int32_t k) {
  MxPlan a;
  a.mt = m <= 16 ? 1 : m <= 32 ? 2 : 4;
  a.nt = n >= 16384 ? a.mt == 4 ? 2 : 4 : a.mt == 1 ? 1 : 2;
  const int64_t blocks = (m + 16 * a.mt - 1) / (16 * a.mt), tiles = ((int64_t)n + 16 * a.nt - 1) / (16 * a.nt);
  const int units = (k + kMxUnit - 1) / kMxUnit;
  a.splits = 1;
  while (tiles * blocks * a.splits < 200 && units / (a.splits * 2) >= 2 * kMxWaves) a.splits *= 2;
  return a;
}

hipError_t launch_linear_mx(const MxPlan &plan, const MxLaunch &p, hipStream_t st) {
  return p.a_scales ? launch<true>(plan, p, st) : launch<false>(plan, p, st);
}

}  // namespace daf
