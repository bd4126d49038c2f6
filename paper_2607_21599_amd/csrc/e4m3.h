// e4m3 codes (OCP: 3 mantissa bits, largest 448, no infinities) and their power-of-two scales.
#pragma once

#include <hip/hip_runtime.h>

namespace daf {

constexpr int kMinScaleExp = -100;  // exponent of the smallest scale

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
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
  x[0] = a[0], x[1] = a[1], x[2] = b[0], x[3] = b[1];
#endif
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

}  // namespace daf
