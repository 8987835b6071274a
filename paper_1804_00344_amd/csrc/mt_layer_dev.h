// Device helpers shared by the recurrent layer's kernels.
#pragma once

#include "mt_layer.h"

namespace mt {

// VEC consecutive elements of a row as floats (one access where VEC > 1: the caller has checked
// that the row is aligned to it)
template <typename T, int VEC>
struct Vec {
  static_assert(VEC * sizeof(T) <= 16, "one 16-byte access");
  struct __attribute__((aligned(VEC * sizeof(T)))) Raw {
    T v[VEC];
  };
  __device__ __forceinline__ static Raw raw(const T *p) { return *(const Raw *)p; }
  // the same from and to any address of an element: global memory takes whole vectors there too
  struct __attribute__((packed, aligned(sizeof(T)))) Any {
    T v[VEC];
  };
  __device__ __forceinline__ static Raw raw_any(const T *p) {
    const Any a = *(const Any *)p;
    Raw r;
    __builtin_memcpy(&r, &a, sizeof r);
    return r;
  }
  __device__ __forceinline__ static void store_any(T *p, const Raw &r) {
    Any a;
    __builtin_memcpy(&a, &r, sizeof a);
    *(Any *)p = a;
  }
  // STREAM: past the L2
  template <bool STREAM>
  __device__ __forceinline__ static void store(T *p, const Raw &r) {
    if constexpr (STREAM) {
      static_assert(sizeof(Raw) == 16, "streamed in whole vectors");
      typedef int v4 __attribute__((ext_vector_type(4)));
      v4 q;
      __builtin_memcpy(&q, &r, 16);
      __builtin_nontemporal_store(q, (v4 *)p);
    } else {
      *(Raw *)p = r;
    }
  }
  template <bool STREAM = false>
  __device__ __forceinline__ static void put(T *p, const float (&f)[VEC]) {
    Raw r;
#pragma unroll
    for (int i = 0; i < VEC; ++i) r.v[i] = (T)f[i];
    store<STREAM>(p, r);
  }
  __device__ __forceinline__ static void put_any(T *p, const float (&f)[VEC]) {
    Raw r;
#pragma unroll
    for (int i = 0; i < VEC; ++i) r.v[i] = (T)f[i];
    store_any(p, r);
  }
};

// e^v for v <= 0 to a few roundings at any v: the product with log2(e) in two parts (one rounding of
// it alone costs a relative |v| 2^-24)
__device__ __forceinline__ float exp_acc(float v) {
  const float t = v * 1.4426950408889634f;
  const float lo = fmaf(v, 1.4426950408889634f, -t) + v * 1.9259629911e-8f;
  const float e = __builtin_amdgcn_exp2f(t);
  return e > 0.f ? fmaf(e, lo * 0.6931471805599453f, e) : e;
}

// v * sigmoid(v).  The sigmoid's exponential is at most e^88 here: beyond, it is infinite and its
// reciprocal 0, which times v is 0 as well (v finite).
__device__ __forceinline__ float silu(float v) { return v * rcp_fast(1.0f + exp_fast(-v)); }

}  // namespace mt
