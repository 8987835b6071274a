// Attention by tiles of 128 query rows: kernel and launch, instantiated by mt_mha_tile_*.hip.
#pragma once

#include "mt_mha_dev.h"

namespace mt {

typedef float f32x16 __attribute__((ext_vector_type(16)));

// The two element types' MFMAs of 32 keys (rows) by 32 queries (columns).  An operand's lane holds row or column
// lane % 32; a result's lane holds column lane % 32 and rows 8 (r / 4) + 4 (lane / 32) + r % 4.  Which depth a lane's
// elements stand for is free as long as both operands agree: the weights P of a tile leave the first product with
// a lane's keys 4 (lane / 32) + .. of every eight, and are taken for the second one in just that order.
template <typename T>
struct Tile;

template <>
struct Tile<bf16> {
  static constexpr int KT = 64;    // keys of a tile
  static constexpr int STEP = 16;  // features of a step of q.k
  typedef bf16x8 Q;                // features 16 s + 8 (lane / 32) + ..
  // chunks of 16 bytes of a row are permuted by its number: 8 rows read at one feature (keys), or 4 rows at 16
  // neighbouring ones (values, transposed), fall into different banks
  __device__ static __forceinline__ int swap_k(int row) { return row & 7; }
  __device__ static __forceinline__ int swap_v(int row) { return (row & 3) << 1; }
  __device__ static __forceinline__ void qk(f32x16 &s, const char *k, const Q &q) {
    s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*(const bf16x8 *)k, q, s, 0, 0, 0);
  }
};

template <>
struct Tile<float> {
  static constexpr int KT = 32;
  static constexpr int STEP = 8;
  typedef f32x4 Q;  // features 8 s + 4 (lane / 32) + ..
  __device__ static __forceinline__ int swap_k(int row) { return row & 7; }
  __device__ static __forceinline__ int swap_v(int) { return 0; }
  __device__ static __forceinline__ void qk(f32x16 &s, const char *k, const Q &q) {
    const f32x4 kk = *(const f32x4 *)k;
#pragma unroll
    for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_32x32x2f32(kk[e], q[e], s, 0, 0, 0);
  }
};

__device__ __forceinline__ float both_halves_max(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_int(v), __float_as_int(v), false, false);
  return fmaxf(__int_as_float(r[0]), __int_as_float(r[1]));
}
__device__ __forceinline__ float both_halves_sum(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_int(v), __float_as_int(v), false, false);
  return __int_as_float(r[0]) + __int_as_float(r[1]);
}

template <typename T>
__device__ __forceinline__ bool any_nonfinite(const int4 &v) {
  const unsigned w[4] = {(unsigned)v.x, (unsigned)v.y, (unsigned)v.z, (unsigned)v.w};
  bool bad = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (sizeof(T) == 2) bad |= (w[i] & 0x7f80u) == 0x7f80u;
    bad |= (w[i] & 0x7f800000u) == 0x7f800000u;
  }
  return bad;
}

constexpr int kTileRows = 128;

// What a launch of the tile kernel has decided
struct TilePlan {
  int tiles;  // of kTileRows rows of a sequence's key head
  int parts;  // the key axis is cut into
  int first;  // workgroup of this launch
};

// A workgroup of four waves takes 128 rows of one key head of one sequence: row r is query r / G, head r % G of those
// that share the key head.  Keys and values pass through LDS a tile at a time, the next tile's on their way in registers
// while this one's is computed.  Scores transposed: S = K Q^T has a query per lane and its keys in registers, so the
// softmax needs one exchange between a wave's halves, and P^T is the second product's operand as it stands.
template <typename T, int DP, bool PAGED>
__global__ void __launch_bounds__(256, DP <= 128 ? 2 : 1) tile_kernel(MhaArgs a, TilePlan plan) {
  typedef Tile<T> M;
  constexpr int KT = M::KT, ES = sizeof(T), CH = DP * ES / 16, ROWB = DP * ES, TB = KT * ROWB;
  constexpr int NL = KT * CH / 256;  // chunks of each operand that a thread moves per tile
  constexpr int KB = KT / 32, DB = DP / 32, STEPS = DP / M::STEP;
  static_assert(KT * CH % 256 == 0, "every thread moves as many");
  __shared__ __attribute__((aligned(1024))) char lds[4 * TB];
  __shared__ int dirty, edge[2];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5, col = lane & 31;
  // consecutive tiles of a key head run on one XCD, whose L2 holds its keys and values; the last tiles, which see the
  // most keys, first
  const int w = plan.first + xcd_remap(blockIdx.x, gridDim.x);
  const int part = w % plan.parts, u = w / plan.parts, bh = u / plan.tiles;
  const int tile = plan.tiles - 1 - (u - bh * plan.tiles);
  const int b = bh / a.Hk, h = bh - b * a.Hk;
  const RowSpan span = row_span<PAGED>(a, b, h == 0 && tile == 0 && part == 0 && threadIdx.x == 0);
  const int R = span.n * a.G, r0 = tile * kTileRows;
  if (r0 >= R) return;
  const int i_first = r0 / a.G, i_last = min(r0 + kTileRows - 1, R - 1) / a.G;
  int lo, hi, lo2, hi2;  // keys that some row sees: [lo, hi2); that all see: [lo2, hi)
  seen_keys<PAGED>(a, span, i_first, lo, hi);
  seen_keys<PAGED>(a, span, i_last, lo2, hi2);
  if (threadIdx.x == 0) dirty = 0;
  const float *mask = !PAGED && a.mask ? a.mask + (long long)b * a.Sk : nullptr;
  if (!PAGED && mask) {  // the first and the last valid position
    if (threadIdx.x == 0) edge[0] = a.Sk, edge[1] = 0;
    __syncthreads();
    int first = a.Sk, last = 0;
    for (int j = threadIdx.x; j < a.Sk; j += 256)
      if (mask[j] != 0.f) first = min(first, j), last = j + 1;
    if (last) atomicMin(&edge[0], first), atomicMax(&edge[1], last);
    __syncthreads();
    lo = edge[0];
    hi2 = edge[1];
  }
  if (PAGED) __syncthreads();  // dirty is set from here on
  lo &= ~(KT - 1);
  int nt = hi2 > lo ? (hi2 - lo + KT - 1) / KT : 0;  // tiles of keys, this part's of them
  {
    const int per = (nt + plan.parts - 1) / plan.parts;
    const int t0 = min(nt, part * per);
    nt = min(nt, t0 + per) - t0;
    lo += t0 * KT;
  }
  // ---- this lane's query
  const int r = r0 + wave * 32 + col;
  const bool live = r < R;
  const int qi = (live ? r : R - 1) / a.G, hq = h * a.G + (live ? r : R - 1) - qi * a.G;
  int qlo, qhi;
  seen_keys<PAGED>(a, span, qi, qlo, qhi);
  typename M::Q qf[STEPS];
  {
    constexpr int VEC = 16 / ES;
    const T *q = (const T *)a.q + ((long long)b * a.S + qi) * a.ldq + (long long)hq * a.Dh;
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      const int d = s * M::STEP + half * VEC;
      typename Vec<T, VEC>::Raw v = {};
      if (live && d < a.Dh) v = Vec<T, VEC>::raw_any(q + d);
      __builtin_memcpy(&qf[s], &v, 16);
    }
  }
  f32x16 o[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d) o[d] = (f32x16)(0.f);
  float m = kNegInf, l = 0.f;
  // ---- tiles of keys: this thread's chunks
  int4 kr[NL], vr[NL];
  unsigned long long seen_next = 0;  // keys of the next tile that are there and not masked
  auto fetch = [&](int k0) {
    if (!PAGED) {
      const int j = k0 + lane;
      seen_next = __ballot(lane < KT && j < hi2 && (!mask || mask[j] != 0.f));
    }
#pragma unroll
    for (int x = 0; x < NL; ++x) {
      const int id = threadIdx.x + x * 256, row = id / CH, c = id % CH;
      const int j = min(k0 + row, hi2 - 1);  // keys behind the last one are not read
      kr[x] = make_int4(0, 0, 0, 0);
      vr[x] = make_int4(0, 0, 0, 0);
      if (c * 16 < a.Dh * ES) {
        const T *ks = (const T *)a.k + key_at<PAGED>(a, b, h, j, a.ldk);
        const T *vs = (const T *)a.v + (PAGED ? ks - (const T *)a.k : key_at<PAGED>(a, b, h, j, a.ldv));
        if (PAGED) {
          kr[x] = *(const int4 *)((const char *)ks + c * 16);
          vr[x] = *(const int4 *)((const char *)vs + c * 16);
        } else {
          const auto kv = Vec<T, 16 / ES>::raw_any(ks + c * (16 / ES)), vv = Vec<T, 16 / ES>::raw_any(vs + c * (16 / ES));
          __builtin_memcpy(&kr[x], &kv, 16);
          __builtin_memcpy(&vr[x], &vv, 16);
        }
      }
    }
  };
  // Values that no row may see are zeros (their weights are); values that some rows see and others not have to be
  // numbers, or the weights' zeros would not hide them.
  auto put = [&](int k0, char *buf) {
    const bool mixed = k0 + KT > hi || k0 < lo2;
#pragma unroll
    for (int x = 0; x < NL; ++x) {
      const int id = threadIdx.x + x * 256, row = id / CH, c = id % CH;
      const bool there = PAGED ? k0 + row < hi2 : (seen_next >> row) & 1;
      if (!there) vr[x] = make_int4(0, 0, 0, 0);
      if (PAGED && mixed && any_nonfinite<T>(vr[x])) dirty = 1;
      *(int4 *)(buf + row * ROWB + ((c ^ M::swap_k(row)) << 4)) = kr[x];
      *(int4 *)(buf + TB + row * ROWB + ((c ^ M::swap_v(row)) << 4)) = vr[x];
    }
  };
  if (nt > 0) {
    fetch(lo);
    put(lo, lds);
  }
  for (int t = 0; t < nt; ++t) {
    const int k0 = lo + t * KT;
    const char *buf = lds + (t & 1) * 2 * TB;
    const unsigned long long seen = seen_next;
    __syncthreads();
    if (t + 1 < nt) fetch(k0 + KT);
    // ---- scores
    f32x16 s[KB];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      s[kb] = (f32x16)(0.f);
      const int row = kb * 32 + col;
#pragma unroll
      for (int st = 0; st < STEPS; ++st)
        M::qk(s[kb], buf + row * ROWB + (((2 * st + half) ^ M::swap_k(row)) << 4), qf[st]);
    }
    if (PAGED ? (k0 + KT > hi || k0 < lo2) : seen != (KT == 64 ? ~0ull : (1ull << KT) - 1)) {
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int kk = kb * 32 + 8 * (e / 4) + 4 * half + e % 4;
          const bool ok = PAGED ? k0 + kk >= qlo && k0 + kk < qhi : (seen >> kk) & 1;
          s[kb][e] = ok ? s[kb][e] : kNegInf;
        }
    }
    // ---- weights relative to a maximum that only moves where a score passes it by 2^8: the sums stay far inside
    // 32 bits, and the accumulators are rescaled a few times in a row's life
    float mx = kNegInf;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int e = 0; e < 16; ++e) mx = fmaxf(mx, s[kb][e]);
    mx = both_halves_max(mx) * a.scale;
    if (__any(mx > m + 8.f)) {
      const float mn = fmaxf(m, mx), c = m == kNegInf ? 0.f : __builtin_amdgcn_exp2f(m - mn);
      m = mn;
      l *= c;
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[d][e] *= c;
    }
    const float use = m == kNegInf ? 0.f : m;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        s[kb][e] = __builtin_amdgcn_exp2f(fmaf(s[kb][e], a.scale, -use));
        l += s[kb][e];
      }
    // ---- values
    const char *vb = buf + TB;
    if constexpr (ES == 2) {
      const int l16 = lane & 15;
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
          bf16x8 p;
#pragma unroll
          for (int e = 0; e < 8; ++e) p[e] = (bf16)s[kb][hf * 8 + e];
          const int row = kb * 32 + hf * 16 + 4 * half + l16 / 4;
#pragma unroll
          for (int d = 0; d < DB; ++d) {
            const int c = 4 * d + 2 * ((lane >> 4) & 1) + ((l16 & 3) >> 1), by = (l16 & 1) * 8;
            typedef short s16x4 __attribute__((ext_vector_type(4)));
            typedef s16x4 __attribute__((address_space(3))) * Lp;
            union {
              s16x4 q[2];
              bf16x8 v;
            } f;
            f.q[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lp)(vb + row * ROWB + ((c ^ M::swap_v(row)) << 4) + by));
            f.q[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lp)(vb + (row + 8) * ROWB + ((c ^ M::swap_v(row)) << 4) + by));
            o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f.v, p, o[d], 0, 0, 0);
          }
        }
    } else {
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int row = 8 * (e / 4) + 4 * half + e % 4;
#pragma unroll
        for (int d = 0; d < DB; ++d)
          o[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(*(const float *)(vb + row * ROWB + (d * 32 + col) * 4), s[0][e], o[d], 0, 0, 0);
      }
    }
    if (t + 1 < nt) put(k0 + KT, lds + ((t + 1) & 1) * 2 * TB);
  }
  // ---- results
  l = both_halves_sum(l);
  const long long rows = (long long)a.B * a.Hq * a.S;
  const Parts parts = parts_of(a.ws, rows, plan.parts);
  const long long prow = part * rows + (long long)bh * a.S * a.G;
  if (live) {
    if (plan.parts > 1) {
      float *po = parts.o + (prow + r) * a.Dh;
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int e = 0; e < 16; e += 4) {
          const int f = d * 32 + 2 * e + 4 * half;
          if (f < a.Dh) *(float4 *)(po + f) = make_float4(o[d][e], o[d][e + 1], o[d][e + 2], o[d][e + 3]);
        }
      if (half == 0) parts.ml[prow + r] = make_float2(m, l);
    } else {
      const float inv = l == 0.f ? 0.f : 1.f / l;
      T *y = (T *)a.y + ((long long)b * a.S + qi) * a.ldy + (long long)hq * a.Dh;
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int e = 0; e < 16; e += 4) {
          const int f = d * 32 + 2 * e + 4 * half;
          const float v[4] = {o[d][e] * inv, o[d][e + 1] * inv, o[d][e + 2] * inv, o[d][e + 3] * inv};
          if (f < a.Dh) Vec<T, 4>::put_any(y + f, v);
        }
    }
  }
  if (!PAGED) return;
  // values that are no numbers where some rows see them and others not: row by row instead
  __syncthreads();
  if (!dirty) return;
  for (int x = wave; x < kTileRows && r0 + x < R; x += 4) {
    const int ii = (r0 + x) / a.G, hh = h * a.G + (r0 + x) - ii * a.G;
    const bool cut = plan.parts > 1;
    attend_one<T, PAGED>(a, span, b, ii, hh, lo, lo + nt * KT, (float *)lds + wave * 256,
                         cut ? parts.o + (prow + r0 + x) * a.Dh : nullptr, cut ? parts.ml + prow + r0 + x : nullptr);
  }
}

template <typename T, bool PAGED>
hipError_t launch_tiles_as(const MhaArgs &a, TilePlan plan, hipStream_t st) {
  const long long all = (long long)a.B * a.Hk * plan.tiles * plan.parts, most = 1 << 22;  // workgroups of a launch
  for (long long first = 0; first < all; first += most) {
    plan.first = (int)first;
    const dim3 grid((unsigned)(all - first < most ? all - first : most)), block(256);
    if (a.Dh <= 64)
      hipLaunchKernelGGL((tile_kernel<T, 64, PAGED>), grid, block, 0, st, a, plan);
    else if (a.Dh <= 128)
      hipLaunchKernelGGL((tile_kernel<T, 128, PAGED>), grid, block, 0, st, a, plan);
    else
      hipLaunchKernelGGL((tile_kernel<T, 256, PAGED>), grid, block, 0, st, a, plan);
  }
  return hipGetLastError();
}

hipError_t launch_tiles_bf16(const MhaArgs &a, const TilePlan &plan, hipStream_t st);
hipError_t launch_tiles_f32(const MhaArgs &a, const TilePlan &plan, hipStream_t st);

}  // namespace mt
