// Host-side helpers of the C entry points: the error message, status macros, pointer checks.
#pragma once

#include "mt_internal.h"

namespace mt {

extern thread_local char g_err[512];  // message of the last failed call on this thread

// sets the message and returns s
mt_status fail(mt_status s, const char *fmt, ...) __attribute__((format(printf, 2, 3)));

// the text of a call's error, which is reported with it: the check after the next launch would find it again
inline const char *hip_error(hipError_t e) {
  (void)hipGetLastError();
  return hipGetErrorString(e);
}

inline size_t rup(size_t x, size_t a) { return (x + a - 1) / a * a; }

inline bool aligned(const void *p, size_t a) { return ((uintptr_t)p % a) == 0; }

inline mt_status check_dev_ptr(const void *p, const char *name, size_t align = 16) {
  if (!p) return fail(MT_ERR_ARG, "%s is NULL", name);
  if (!aligned(p, align)) return fail(MT_ERR_ARG, "%s is not %zu-byte aligned", name, align);
  return MT_OK;
}

}  // namespace mt

#define HIP_TRY(expr)                                                              \
  do {                                                                             \
    hipError_t e_ = (expr);                                                        \
    if (e_ != hipSuccess) return fail(MT_ERR_HIP, "%s: %s", #expr, hip_error(e_)); \
  } while (0)

#define CHECK(expr)                 \
  do {                              \
    mt_status s_ = (expr);          \
    if (s_ != MT_OK) return s_;     \
  } while (0)
