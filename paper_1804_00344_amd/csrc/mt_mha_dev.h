// Device helpers shared by the attention kernels: where a key's features are, what a query sees, and one query by one wave.
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

// page of block j of row b; a number out of range is clamped, and reported by who asks
__device__ __forceinline__ int block_page(const MhaArgs &a, int b, int j, bool &bad) {
  const int p = a.table[(long long)b * a.n_blocks + j];
  bad |= (unsigned)p >= (unsigned)a.n_pages;
  return min(max(p, 0), a.n_pages - 1);
}

// element offset of key j of row b and key head h from the cache's (or the rows') beginning
template <bool PAGED>
__device__ __forceinline__ long long key_at(const MhaArgs &a, int b, int h, int j, long long ld, bool &bad) {
  if (PAGED)
    return ((((long long)block_page(a, b, j >> a.page_log2, bad) * a.Hk + h) << a.page_log2) + (j & ((1 << a.page_log2) - 1))) * a.Dh;
  return ((long long)b * a.Sk + j) * ld + h * a.Dh;
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

// One query head of one query by one wave over its keys in [k0, k1): 64 keys at a time, a key per lane for the scores
// (running maximum and sum in 32 bits), a feature per lane for the values.  qs: 256 floats of LDS of the wave.  A key
// that is not seen is not read.  Gives the result, or where po is set the sums and their pair.
template <typename T, bool PAGED>
__device__ void attend_one(const MhaArgs &a, const RowSpan &r, int b, int i, int hq, int k0, int k1, float *qs,
                           float *po, float2 *pml) {
  constexpr int VEC = 16 / sizeof(T);
  typedef Vec<T, VEC> V;
  const int lane = threadIdx.x & 63, h = hq / a.G;
  const long long row = (long long)b * a.S + i;
  const T *q = (const T *)a.q + row * a.ldq + (long long)hq * a.Dh;
  for (int d = lane; d < a.Dh; d += 64) qs[d] = (float)q[d];
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  int lo, hi;
  seen_keys<PAGED>(a, r, i, lo, hi);
  lo = max(lo, k0);
  hi = min(hi, k1);
  float m = kNegInf, l = 0.f, acc[4] = {};
  bool bad = false;  // reported by the caller's own reads
  for (int t = lo; t < hi; t += 64) {
    const int j = t + lane;
    const bool seen = j < hi && (PAGED || !a.mask || a.mask[(long long)b * a.Sk + j] != 0.f);
    float s = kNegInf;
    if (seen) {
      const T *k = (const T *)a.k + key_at<PAGED>(a, b, h, j, a.ldk, bad);
      float x = 0.f;
      for (int d = 0; d < a.Dh; d += VEC) {
        const typename V::Raw v = V::raw_any(k + d);
#pragma unroll
        for (int e = 0; e < VEC; ++e) x = fmaf(qs[d + e], (float)v.v[e], x);
      }
      s = rounded_product(x, a.scale);
    }
    const float mn = fmaxf(m, wave_max(s)), use = mn == kNegInf ? 0.f : mn;
    const float p = seen ? __builtin_amdgcn_exp2f(s - use) : 0.f;
    const float c = m == kNegInf ? 0.f : __builtin_amdgcn_exp2f(m - use);
    m = mn;
    l = l * c + wave_sum(p);
#pragma unroll
    for (int f = 0; f < 4; ++f) acc[f] *= c;
    for (unsigned long long left = __ballot(seen); left; left &= left - 1) {
      const int kk = __builtin_ctzll(left);
      const float w = lane_f(p, kk);
      const T *v = (const T *)a.v + key_at<PAGED>(a, b, h, t + kk, a.ldv, bad);
#pragma unroll
      for (int f = 0; f < 4; ++f)
        if (lane + 64 * f < a.Dh) acc[f] = fmaf(w, (float)v[lane + 64 * f], acc[f]);
    }
  }
  T *y = (T *)a.y + row * a.ldy + (long long)hq * a.Dh;
#pragma unroll
  for (int f = 0; f < 4; ++f) {
    const int d = lane + 64 * f;
    if (d >= a.Dh) continue;
    if (po)
      po[d] = acc[f];
    else
      Store<T>::put(y + d, l == 0.f ? 0.f : acc[f] / l);
  }
  if (po && lane == 0) *pml = make_float2(m, l);
  __builtin_amdgcn_wave_barrier();
}

}  // namespace mt
