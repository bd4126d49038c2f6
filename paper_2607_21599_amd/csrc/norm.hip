// The residual's addition and the RMS norm between two projections (daf_add_rmsnorm):
//   s = x + delta, rounded to the rows' type;  y = s / sqrt(mean(s^2) + eps) * w
// with y in the rows' type, or for a projection of few bits as e4m3 codes, one
// power-of-two scale per 32 values (the smallest under which the largest magnitude is
// at most 448), or both. fp32 arithmetic; the codes are rounded once, from the fp32
// value.
//
// A row of up to 16384 values stays in registers between the sum of squares and its use, so
// that every input is read once; 8 values per thread and piece, 4 neighbouring lanes have
// the 32 values of a scale. Sums go in a fixed order: a call's result depends on its inputs
// alone. Bound by HBM: 5043 rows of 3584 with all outputs (163 MB) in 32 us, the rate of a
// large copy (fp32: 308 MB in 59); one row in 2.0 us, of which most is the launch.
#include "e4m3.h"
#include "step.h"

namespace daf {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));

// 8 values of a row
template <bool BF16>
struct Piece {
  static __device__ __forceinline__ void load(const void *p, int64_t at, float (&x)[8]) {
    if constexpr (BF16) {
      const bf16x8 v = *reinterpret_cast<const bf16x8 *>(static_cast<const __bf16 *>(p) + at);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = (float)v[e];
    } else {
      const f32x4 a = *reinterpret_cast<const f32x4 *>(static_cast<const float *>(p) + at);
      const f32x4 b = *reinterpret_cast<const f32x4 *>(static_cast<const float *>(p) + at + 4);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = a[e], x[e + 4] = b[e];
    }
  }
  static __device__ __forceinline__ void store(void *p, int64_t at, const float (&x)[8]) {
    if constexpr (BF16) {
      bf16x8 v;
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = (__bf16)x[e];
      *reinterpret_cast<bf16x8 *>(static_cast<__bf16 *>(p) + at) = v;
    } else {
      *reinterpret_cast<f32x4 *>(static_cast<float *>(p) + at) = f32x4{x[0], x[1], x[2], x[3]};
      *reinterpret_cast<f32x4 *>(static_cast<float *>(p) + at + 4) = f32x4{x[4], x[5], x[6], x[7]};
    }
  }
};

// WAVES per row (of a workgroup of kNormThreads), PIECES per thread that stay in
// registers; 0: rows of any width, whose sum is read or made a second time.
template <bool BF16, int WAVES, int PIECES>
__global__ __launch_bounds__(kNormThreads) void add_rmsnorm_kernel(const NormLaunch p) {
  constexpr int ROWS = kNormThreads / 64 / WAVES, THREADS = 64 * WAVES;
  __shared__ float part[kNormThreads / 64];
  const int t = threadIdx.x % THREADS, wave = threadIdx.x >> 6;
  const int64_t row = (int64_t)blockIdx.x * ROWS + threadIdx.x / THREADS;
  const bool have = row < p.rows;
  if (WAVES == 1 && !have) return;  // one wave per row: none waits for another
  const int64_t row0 = row * p.width;
  const int pieces = have ? p.width / 8 : 0;  // waves past the last row still reach the barrier
  constexpr int HELD = PIECES > 0 ? PIECES : 1;
  float s[HELD][8], ss = 0.f;
  auto sum = [&](int j, float (&v)[8], bool again) {  // of x and delta, in the rows' type
    const int64_t at = row0 + 8 * j;
    if (again && p.sum) return Piece<BF16>::load(p.sum, at, v);
    Piece<BF16>::load(p.x, at, v);
    if (!p.delta) return;
    float d[8];
    Piece<BF16>::load(p.delta, at, d);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = BF16 ? (float)(__bf16)(v[e] + d[e]) : v[e] + d[e];
    if (!again && p.sum) Piece<BF16>::store(p.sum, at, v);
  };
  auto square = [&](const float (&v)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) ss = __builtin_fmaf(v[e], v[e], ss);
  };
  if constexpr (PIECES > 0) {
#pragma unroll
    for (int k = 0; k < PIECES; ++k)
      if (t + k * THREADS < pieces) {
        sum(t + k * THREADS, s[k], false);
        square(s[k]);
      }
  } else {
    for (int j = t; j < pieces; j += THREADS) {
      sum(j, s[0], false);
      square(s[0]);
    }
  }
#pragma unroll
  for (int m = 32; m; m >>= 1) ss += __shfl_xor(ss, m);
  if constexpr (WAVES > 1) {
    if ((threadIdx.x & 63) == 0) part[wave] = ss;
    __syncthreads();
    ss = 0.f;
#pragma unroll
    for (int i = 0; i < WAVES; ++i) ss += part[threadIdx.x / THREADS * WAVES + i];
  }
  const float inv = 1.f / sqrtf(ss / (float)p.width + p.eps);
  auto finish = [&](int j, const float (&v)[8]) {
    const int64_t at = row0 + 8 * j;
    float y[8];
    Piece<BF16>::load(p.w, 8 * j, y);
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] *= v[e] * inv;
    if (p.y) Piece<BF16>::store(p.y, at, y);
    if (!p.codes) return;
    float top = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      y[e] = y[e] > kMostF32 ? kMostF32 : y[e] < -kMostF32 ? -kMostF32 : y[e];  // NaN stays, and does not count
      top = fmaxf(top, fabsf(y[e]));
    }
    top = fmaxf(top, __shfl_xor(top, 1));
    top = fmaxf(top, __shfl_xor(top, 2));
    const float scale = top == 0.f ? kMinScale : scale_for(top), over = inverse(scale);
    *reinterpret_cast<u32x2 *>(p.codes + at) = u32x2{to_codes(y[0] * over, y[1] * over, y[2] * over, y[3] * over),
                                                     to_codes(y[4] * over, y[5] * over, y[6] * over, y[7] * over)};
    if (j % 4 == 0) p.scales[at / 32] = (unsigned char)(__builtin_bit_cast(unsigned, scale) >> 23);
  };
  if constexpr (PIECES > 0) {
#pragma unroll
    for (int k = 0; k < PIECES; ++k)
      if (t + k * THREADS < pieces) finish(t + k * THREADS, s[k]);
  } else {
    for (int j = t; j < pieces; j += THREADS) {
      sum(j, s[0], true);
      finish(j, s[0]);
    }
  }
}

template <bool BF16>
hipError_t launch(const NormLaunch &p, hipStream_t st) {
  auto go = [&](auto kern, int waves) {
    const int rows = kNormThreads / 64 / waves;
    kern<<<(unsigned)((p.rows + rows - 1) / rows), kNormThreads, 0, st>>>(p);
  };
  // As many waves per row as give every thread one piece: rows of all sums and outputs, us by
  // 1, 2, 4 and 8 waves: 40000 of 256 21.6, 26.5, 36.0, 52.2; 16000 of 1024 32.3, 29.6, 29.6,
  // 34.8; 5043 of 3584 45.8, 39.6, 35.2, 32.4; 2000 of 8192 47.6, 40.4, 34.8, 32.9.
  const int pieces = (p.width / 8 + 63) / 64;  // of a lane of one wave
  if (pieces <= 1) go(add_rmsnorm_kernel<BF16, 1, 1>, 1);
  else if (pieces <= 2) go(add_rmsnorm_kernel<BF16, 2, 1>, 2);
  else if (pieces <= 4) go(add_rmsnorm_kernel<BF16, 4, 1>, 4);
  else if (pieces <= 8) go(add_rmsnorm_kernel<BF16, 8, 1>, 8);
  else if (pieces <= 16) go(add_rmsnorm_kernel<BF16, 8, 2>, 8);
  else if (pieces <= 32) go(add_rmsnorm_kernel<BF16, 8, 4>, 8);
  else go(add_rmsnorm_kernel<BF16, 8, 0>, 8);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_add_rmsnorm(bool bf16, const NormLaunch &p, hipStream_t st) {
  return bf16 ? launch<true>(p, st) : launch<false>(p, st);
}

}  // namespace daf
