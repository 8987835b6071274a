// Device helpers shared by the attention kernels: what a query sees, the ends of masks, where a call's parts go.
#pragma once

#include "mt_layer_dev.h"
#include "mt_mha.h"

namespace mt {

constexpr float kNegInf = -__builtin_inff();

// A weight of the matrix kernels is 2^(s scale - m) by one multiply-add, whose product is not rounded while m is a rounded one: the
// largest score's exponent is what m was rounded by, up to 2 for scores (in units of log2) of 2^26.  From there on the product is
// rounded first, so that the difference to the maximum is 0 again; with 2^32 the weights would pass all powers of two.
constexpr float kFarScore = 67108864.f;

__device__ __forceinline__ float rounded_product(float x, float y) {
#pragma clang fp contract(off)
  return x * y;
}

// x y, or zero where either is zero, whatever the other (v_mul_legacy_f32): of rows without any weight nothing is left of values
// that are no numbers
extern "C" __device__ float times_or_zero(float x, float y) __asm("llvm.amdgcn.fmul.legacy");

// The score from which a running maximum moves: one that is 2^8 larger, or, of scores that far, any, so that the branch that moves it
// takes their weights too (a branch of its own in every tile: 4 x 1000 positions of 16 heads of 64 in bf16 25.5 -> 27.5 us, this
// way 26.7)
__device__ __forceinline__ float max_bound(float m) { return fabsf(m) >= kFarScore ? kNegInf : m + 8.f; }

// The lengths of row b: positions and new ones (paged), or keys and queries (cross); clamped, reported where tell is set
struct RowSpan {
  int len, n;  // keys, queries
  int first;   // paged: position of query 0
};
template <bool PAGED>
__device__ __forceinline__ RowSpan row_span(const MhaArgs &a, int b, bool tell) {
  RowSpan r;
  const int n0 = a.n_new ? a.n_new[b] : a.S;
  r.n = min(max(n0, 0), a.S);
  bool bad = n0 != r.n;
  if (PAGED) {
    const int l0 = a.len[b];
    r.len = min(max(l0, 0), a.n_blocks << a.page_log2);
    bad |= l0 != r.len;
  } else {
    r.len = a.Sk;
  }
  r.first = r.len - r.n;
  if (tell && bad) atomicOr(a.err, kErrLen);
  return r;
}

// keys [lo, hi) that query i may see
template <bool PAGED>
__device__ __forceinline__ void seen_keys(const MhaArgs &a, const RowSpan &r, int i, int &lo, int &hi) {
  lo = 0;
  hi = r.len;
  if (PAGED) {
    hi = r.first + i + 1;
    if (a.window) lo = max(0, hi - a.window);
  }
}

// The first valid position of a mask and one past its last, of the positions t, t + step, ..: U loads on their way at a time
// (64 sentences of up to 1000 positions, 4 queries of 8 heads of 64 in bf16, the waves of a workgroup together: 17.4 -> 14.4 us)
template <int U>
__device__ __forceinline__ void mask_ends(const float *mask, int n, int t, int step, int &first, int &last) {
  first = n;
  last = 0;
  for (int j0 = t; j0 < n; j0 += U * step) {
    float v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = mask[min(j0 + u * step, n - 1)];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int j = j0 + u * step;
      const bool valid = j < n && v[u] != 0.f;
      first = valid ? min(first, j) : first;
      last = valid ? j + 1 : last;
    }
  }
}

// Where a call's parts of a result go that the key axis is cut for: part s of row (b*Hk + h)*S*G + i*G + g holds the
// sums of its keys, the maximum that they are relative to and their weights' sum (both halves of a pair)
struct Parts {
  float *o;   // [parts][rows][Dh]
  float2 *ml; // [parts][rows]
};
__host__ __device__ inline Parts parts_of(void *ws, long long rows, int parts) {
  Parts p;
  p.ml = (float2 *)ws;
  p.o = (float *)ws + ((rows * parts * 2 + 63) & ~63ll);
  return p;
}
inline size_t parts_bytes(long long rows, int parts, int Dh) {
  return (size_t)(((rows * parts * 2 + 63) & ~63ll) + rows * parts * Dh) * 4;
}

}  // namespace mt
