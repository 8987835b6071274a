// Host-side helpers of the C entry points: the error message, status macros, pointer checks.
#pragma once

#include <initializer_list>

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

namespace mt {

inline mt_status query_device(int *dev, int *ncu) {
  if (hipGetDevice(dev) != hipSuccess ||
      hipDeviceGetAttribute(ncu, hipDeviceAttributeMultiprocessorCount, *dev) != hipSuccess || *ncu <= 0)
    return fail(MT_ERR_HIP, "cannot query the device's compute units");
  return MT_OK;
}

inline mt_status check_device(int device) {
  int dev = -1;
  HIP_TRY(hipGetDevice(&dev));
  if (dev != device) return fail(MT_ERR_STATE, "loaded on device %d, but device %d is current", device, dev);
  return MT_OK;
}

inline mt_status alloc(void **p, size_t bytes) {
  const hipError_t e = hipMalloc(p, bytes);
  if (e != hipSuccess) {
    *p = nullptr;
    return fail(MT_ERR_OOM, "hipMalloc(%zu): %s", bytes, hip_error(e));
  }
  return MT_OK;
}

// A range of rows of a wider matrix that a call reads or writes
struct Span {
  const char *name;
  const void *p;
  long long rows, ld, width;  // bytes
};

// Whether two spans share a byte.  Spans of one stride whose columns do not meet do not; other
// strides are compared by their whole ranges.
inline bool overlap(const Span &a, const Span &b) {
  if (!a.p || !b.p || a.rows <= 0 || b.rows <= 0 || a.width <= 0 || b.width <= 0) return false;
  const uintptr_t a0 = (uintptr_t)a.p, b0 = (uintptr_t)b.p;
  const uintptr_t a1 = a0 + (uintptr_t)((a.rows - 1) * a.ld + a.width), b1 = b0 + (uintptr_t)((b.rows - 1) * b.ld + b.width);
  if (a1 <= b0 || b1 <= a0) return false;
  if (a.ld != b.ld || a.ld <= 0) return true;
  const long long off = (long long)((b0 > a0 ? b0 - a0 : a0 - b0) % (uintptr_t)a.ld);
  const long long lo = b0 > a0 ? a.width : b.width, hi = b0 > a0 ? b.width : a.width;  // of the lower, the upper one
  return off < lo || off + hi > a.ld;
}

// Outputs against every input and against each other (out[i] == in[i] allowed where `same` says so)
inline mt_status check_overlaps(std::initializer_list<Span> outs, std::initializer_list<Span> ins) {
  for (auto o = outs.begin(); o != outs.end(); ++o) {
    for (const Span &i : ins)
      if (overlap(*o, i)) return fail(MT_ERR_ARG, "%s overlaps %s", o->name, i.name);
    for (auto q = outs.begin(); q != o; ++q)
      if (overlap(*o, *q)) return fail(MT_ERR_ARG, "%s overlaps %s", o->name, q->name);
  }
  return MT_OK;
}

inline mt_status check_rows(const void *p, const char *name, int64_t ld, int64_t width, int esize) {
  CHECK(check_dev_ptr(p, name, esize));
  if (ld < width || ld > (1ll << 32))
    return fail(MT_ERR_SHAPE, "row stride %lld of %s: need at least its %lld columns", (long long)ld, name,
                (long long)width);
  return MT_OK;
}

}  // namespace mt
