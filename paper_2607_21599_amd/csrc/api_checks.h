// Checks that entry points make on the host, and how they report what they find.
#pragma once

#include <hip/hip_runtime.h>
#include <stdarg.h>
#include <stdint.h>
#include <stdio.h>

#include "daf.h"

namespace daf {

// Error text of the calling thread (api.hip).
daf_status_t set_error(daf_status_t st, const char *text);

inline daf_status_t fail(daf_status_t st, const char *fmt, ...) {
  char text[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(text, sizeof(text), fmt, ap);
  va_end(ap);
  return set_error(st, text);
}

inline daf_status_t ok() { return set_error(DAF_OK, ""); }

inline daf_status_t launched(hipError_t e, const char *what) {
  return e == hipSuccess ? ok() : fail(DAF_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

inline daf_status_t aligned(const void *p, const char *name) {
  if (reinterpret_cast<uintptr_t>(p) % 16 != 0) return fail(DAF_ERR_ALIGNMENT, "%s is not 16-byte aligned", name);
  return DAF_OK;
}

inline daf_status_t need_ptr(const void *p, const char *name) {
  if (!p) return fail(DAF_ERR_INVALID_ARG, "%s is NULL", name);
  return aligned(p, name);
}

// a launch has less than 2^32 threads
inline bool fits(int64_t workgroups, int threads) { return workgroups <= (int64_t)UINT32_MAX / threads; }

}  // namespace daf

#define CHECK(expr)                \
  do {                             \
    daf_status_t st_ = (expr);     \
    if (st_ != DAF_OK) return st_; \
  } while (0)
