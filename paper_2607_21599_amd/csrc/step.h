// Internal declarations of the row-wise and few-row steps between two attention calls
// of a decode step (daf_add_rmsnorm, daf_linear_mx).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace daf {

constexpr float kMostF32 = 3.402823466e38f;        // largest finite value
constexpr float kMinScale = 7.8886090522101181e-31f;  // 2^kMinScaleExp, the scale of zeros
constexpr int kBlockValues = 32;                   // values per scale

struct NormLaunch {
  const void *x, *delta, *w;  // delta nullable
  void *sum, *y;              // nullable
  unsigned char *codes, *scales;  // both or neither
  int64_t rows;
  int32_t width;
  float eps;
};
constexpr int kNormThreads = 512;
hipError_t launch_add_rmsnorm(bool bf16, const NormLaunch &p, hipStream_t st);

// C = A W^T (+ bias) (+ residual) with weights in 4 bits.
struct MxLaunch {
  const unsigned char *a;         // bf16, or e4m3 codes with a_scales
  const unsigned char *a_scales;  // nullable
  const unsigned char *w, *w_scales;
  const void *bias, *residual;    // nullable
  void *c;
  float *part;                    // splits > 1: [splits][M][N]
  int64_t m;
  int32_t n, k;
  int32_t splits;
};
// Which kernel, and how K is split over workgroups.
struct MxPlan {
  int mt, nt;  // 16-row tiles of A and of W per wave
  int splits;
};
constexpr int kMxUnit = 256;  // k per turn of a wave: 128 bytes of a row of W
constexpr int kMxWaves = 8;
MxPlan plan_linear_mx(int64_t m, int32_t n, int32_t k);
hipError_t launch_linear_mx(const MxPlan &plan, const MxLaunch &p, hipStream_t st);

}  // namespace daf
