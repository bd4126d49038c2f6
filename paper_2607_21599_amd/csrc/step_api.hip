// Entry points of the steps between two attention calls of a decode step: argument
// checks and launches. Every check that the host can make runs before anything is
// enqueued.
#include <math.h>

#include "api_checks.h"
#include "step.h"

using namespace daf;

namespace {

daf_status_t check_linear(int64_t M, int32_t N, int32_t K) {
  if (M < 0) return fail(DAF_ERR_INVALID_ARG, "M=%lld is negative", (long long)M);
  if (N <= 0) return fail(DAF_ERR_INVALID_ARG, "N=%d must be positive", N);
  if (K <= 0 || K % kBlockValues != 0)
    return fail(DAF_ERR_UNSUPPORTED, "K=%d is not a positive multiple of %d", K, kBlockValues);
  // the grids of the kernel and of the join, and offsets in a tile
  if (M > 32 * 65535 || N > 256 * 65535 || K > 1 << 24 || !fits(M * ((N + 255) / 256), 256))
    return fail(DAF_ERR_UNSUPPORTED, "M=%lld rows by N=%d, K=%d are too many for one call", (long long)M, N, K);
  return DAF_OK;
}

MxLaunch planned(int64_t M, int32_t N, int32_t K) {
  MxLaunch p{};
  p.m = M;
  p.n = N;
  p.k = K;
  plan_linear_mx(p);
  return p;
}

size_t linear_bytes(const MxLaunch &p) { return p.splits > 1 ? (size_t)p.splits * p.m * p.n * sizeof(float) : 0; }

}  // namespace

extern "C" {

daf_status_t daf_add_rmsnorm(int32_t dtype, int64_t rows, int32_t width, const void *x, const void *delta,
                             const void *w, float eps, void *sum, void *y, void *codes, uint8_t *scales,
                             hipStream_t stream) {
  if (dtype != DAF_BF16 && dtype != DAF_F32)
    return fail(DAF_ERR_UNSUPPORTED, "dtype=%d (supported: DAF_BF16, DAF_F32)", dtype);
  if (rows < 0) return fail(DAF_ERR_INVALID_ARG, "rows=%lld is negative", (long long)rows);
  if (width <= 0 || width % 8 != 0) return fail(DAF_ERR_UNSUPPORTED, "width=%d is not a positive multiple of 8", width);
  if (!(eps >= 0.f) || !isfinite(eps)) return fail(DAF_ERR_INVALID_ARG, "eps must be finite and >= 0");
  if (!codes != !scales) return fail(DAF_ERR_INVALID_ARG, "codes and scales go together");
  if (!y && !codes) return fail(DAF_ERR_INVALID_ARG, "neither y nor codes is given");
  if (codes && width % kBlockValues != 0)
    return fail(DAF_ERR_UNSUPPORTED, "width=%d is not a multiple of %d, which codes need", width, kBlockValues);
  if (sum && !delta) return fail(DAF_ERR_INVALID_ARG, "sum without delta");
  if (sum && sum == y) return fail(DAF_ERR_INVALID_ARG, "sum and y are the same rows");
  if (rows == 0) return ok();
  CHECK(need_ptr(x, "x"));
  CHECK(need_ptr(w, "w"));
  CHECK(aligned(delta, "delta"));
  CHECK(aligned(sum, "sum"));
  CHECK(aligned(y, "y"));
  CHECK(aligned(codes, "codes"));
  if (!fits(rows, kNormThreads)) return fail(DAF_ERR_UNSUPPORTED, "rows=%lld are too many for one call", (long long)rows);
  const NormLaunch p{x, delta, w, sum, y, static_cast<unsigned char *>(codes), scales, rows, width, eps};
  return launched(launch_add_rmsnorm(dtype == DAF_BF16, p, stream), "add_rmsnorm launch");
}

size_t daf_linear_mx_workspace_size(int64_t M, int32_t N, int32_t K) {
  if (check_linear(M, N, K) != DAF_OK || M == 0) return 0;
  return linear_bytes(planned(M, N, K));
}

daf_status_t daf_linear_mx(int64_t M, int32_t N, int32_t K, const void *A, const uint8_t *a_scales, const void *W,
                           const uint8_t *w_scales, const void *bias, const void *residual, void *C, void *workspace,
                           size_t ws_bytes, hipStream_t stream) {
  CHECK(check_linear(M, N, K));
  if (M == 0) return ok();
  CHECK(need_ptr(A, "A"));
  CHECK(need_ptr(W, "W"));
  if (!w_scales) return fail(DAF_ERR_INVALID_ARG, "w_scales is NULL");
  CHECK(aligned(bias, "bias"));
  CHECK(aligned(residual, "residual"));
  CHECK(need_ptr(C, "C"));
  MxLaunch p = planned(M, N, K);
  const size_t need = linear_bytes(p);
  if (need > 0) {
    if (!workspace || ws_bytes < need)
      return fail(DAF_ERR_WORKSPACE, "workspace of %zu bytes needed, %zu given", need, workspace ? ws_bytes : 0);
    CHECK(aligned(workspace, "workspace"));
  }
  p.a = static_cast<const unsigned char *>(A);
  p.a_scales = a_scales;
  p.w = static_cast<const unsigned char *>(W);
  p.w_scales = w_scales;
  p.bias = bias;
  p.residual = residual;
  p.c = C;
  p.part = static_cast<float *>(workspace);
  return launched(launch_linear_mx(p, stream), "linear_mx launch");
}

}  // extern "C"
