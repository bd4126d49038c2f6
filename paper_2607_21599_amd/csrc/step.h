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
  // A workgroup has one of `row_blocks` blocks of 16 mt rows of A, one of `splits` ranges of K
  // and one of `groups` ranges of 16-row tiles of W; of its kMxWaves waves 2^kwaves_log2
  // have a part of the range of K each, at most `steps` times kMxStep.
  int32_t row_blocks, groups, splits, kwaves_log2;
  int32_t mt, steps;
  int32_t part_steps, longer_parts;    // steps of a wave's part: one more in the first longer_parts
  int32_t group_tiles, longer_groups;  // the same of tiles
};
constexpr int kMxStep = 128;  // k of a step: a lane has 32 of them, 16 bytes of W
constexpr int kMxWavesLog2 = 3, kMxWaves = 1 << kMxWavesLog2;
void plan_linear_mx(MxLaunch &p);  // from m, n and k
hipError_t launch_linear_mx(const MxLaunch &p, hipStream_t st);

}  // namespace daf
