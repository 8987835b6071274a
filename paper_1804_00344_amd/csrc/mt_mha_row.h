// Attention of tiles of up to four query rows by the vector units: kernel and launch, instantiated by mt_mha_row_*.hip.
#pragma once

#include "mt_mha_step.h"

namespace mt {

constexpr int kRowRows = 4;  // of a tile

// Where the vector units are faster than the matrix units, which have no step kernel for more than 128 features (16 sentences
// of up to 1000 positions, 8 heads of 256 in fp32: 8 rows a head 57 us, 16 rows 97, 32 rows 165, by tiles of 128 rows 172 to 182;
// heads of 128: 8 rows 34, 12 rows 51, by the step kernel 41 and 37; 264 tokens over 336, 8 heads of 88 that share one: 42, 50)
constexpr bool few_rows(long long rows, int Dh, bool f32) {
  return f32 ? rows <= (Dh > 128 ? 16 : Dh > 64 ? 8 : kRowRows) : rows <= (Dh > 128 ? kRowRows : 1);
}

// v of all lanes that differ in bits O .. 32 of their number, combined
template <int O, typename F>
__device__ __forceinline__ float across(float v, F f) {
  if constexpr (O == 1) return across<2>(f(v, dpp_mov<kDppQuadSwap1>(v)), f);
  if constexpr (O == 2) return across<4>(f(v, dpp_mov<kDppQuadSwap2>(v)), f);
  if constexpr (O == 4) return across<8>(f(v, dpp_mov<0x1B>(dpp_mov<0x141>(v))), f);  // eight lanes reversed, then each four
  if constexpr (O == 8) return across<16>(f(v, dpp_mov<kDppRowRor8>(v)), f);
  if constexpr (O == 16) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_int(v), __float_as_int(v), false, false);
    return across<32>(f(__int_as_float(r[0]), __int_as_float(r[1])), f);
  }
  if constexpr (O == 32) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_int(v), __float_as_int(v), false, false);
    return f(__int_as_float(r[0]), __int_as_float(r[1]));
  }
  return v;
}
// of the lanes that differ in bits 1 .. N / 2: a row's chunks
template <int N>
__device__ __forceinline__ float chunk_sum(float v) {
  if constexpr (N > 1) v += dpp_mov<kDppQuadSwap1>(v);
  if constexpr (N > 2) v += dpp_mov<kDppQuadSwap2>(v);
  if constexpr (N > 4) v += dpp_mov<0x1B>(dpp_mov<0x141>(v));
  if constexpr (N > 8) v += dpp_mov<kDppRowRor8>(v);
  if constexpr (N > 16) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_int(v), __float_as_int(v), false, false);
    v = __int_as_float(r[0]) + __int_as_float(r[1]);
  }
  if constexpr (N > 32) v = both_halves_sum(v);
  return v;
}

// sixteen bytes as they were loaded: elements of 16 bits would take a register each across the loop
typedef unsigned Words __attribute__((ext_vector_type(4)));
typedef Words AnyWords __attribute__((aligned(2)));
template <typename T>
__device__ __forceinline__ float word_at(const Words &w, int e) {
  if constexpr (sizeof(T) == 4) return __uint_as_float(w[e]);
  return __uint_as_float(e & 1 ? w[e / 2] & 0xFFFF0000u : w[e / 2] << 16);
}

// Tiles of up to NR rows of one key head.  A wave reads NL chunks of 16 bytes a lane of keys and of values at a time, whole rows by
// CH neighbouring lanes, and multiplies them where they are: a score is summed over its CH lanes, a value's products stay in
// the lane that has its features until the end.  The next keys are on their way while this tile's values are multiplied, and
// the other way round.  Nothing is staged in LDS, so that three to four times the waves of the step kernel have loads on
// their way, and a weight is not rounded.  SHARE: as in the step kernel.  A matrix unit's fp32 product takes the same cycles
// for one row as for 32 (4096 for 32 keys of 64 features, here about 600 a row).  Bound by memory: a token of each of 64
// sentences of up to 2000 positions, 16 heads of 128 in fp32, 133 us, 5.3 TB/s (by the step kernel 281); 768 of up to 200, 8
// heads of 64, 35 us (82); 16 over up to 9000, 16 heads of 192 in bf16, 148 us (by tiles of 128 rows 637).  Four rows in
// bf16 are better left to the matrix units where they fit (16 tokens of 4 a key head over 32768 positions 460 us, 364).
template <typename T, int DP, int NR, bool PAGED, bool SHARE>
__global__ void __launch_bounds__(256, NR == 1 ? 4 : 2) row_kernel(MhaArgs a, StepPlan plan) {
  constexpr int ES = sizeof(T), EPC = 16 / ES, CH = DP / EPC, RSTEP = 64 / CH, NL = ES == 2 && !PAGED ? 4 : 8, KT = NL * RSTEP;
  typedef Vec<T, EPC> V;  // of a matrix in bf16 half of that: eight addresses and their rows do not fit the registers
  __shared__ __attribute__((aligned(16))) float sums[SHARE ? 4 : 1][SHARE ? NR : 1][SHARE ? DP : 1];
  __shared__ float2 ends[4][NR];
  __shared__ int2 found[4];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const unsigned w = plan.first + xcd_remap(blockIdx.x, gridDim.x), job = SHARE ? w : w * 4 + wave;
  if (job >= plan.jobs) return;
  const int part = (int)(job % (unsigned)plan.parts), tile = (int)(job / (unsigned)plan.parts % (unsigned)plan.tiles);
  const int bh = (int)(job / (unsigned)plan.parts / (unsigned)plan.tiles), b = bh / a.Hk, h = bh - b * a.Hk;
  const RowSpan span = row_span<PAGED>(a, b, h == 0 && tile == 0 && part == 0 && lane == 0);
  const int r0 = tile * NR, R = span.n * a.G - r0;  // of the rows, those from r0
  if (R <= 0) return;
  int lo, hi, lo2, hi2;  // keys that some row sees: [lo, hi2); that all see: [lo2, hi)
  seen_keys<PAGED>(a, span, r0 / a.G, lo, hi);
  seen_keys<PAGED>(a, span, (r0 + min(NR, R) - 1) / a.G, lo2, hi2);
  const int chunk = lane % CH, group = lane / CH;
  const bool feature = chunk * EPC < a.Dh;
  // ---- the rows' features in this lane
  float q[NR][EPC], acc[NR][EPC], m[NR], l[NR];
  int qlo[NR], qhi[NR];
#pragma unroll
  for (int r = 0; r < NR; ++r) {
    const int rr = r0 + min(r, R - 1), i = rr / a.G, hq = h * a.G + rr - i * a.G;
    seen_keys<PAGED>(a, span, i, qlo[r], qhi[r]);
    typename V::Raw v = {};
    if (feature) v = V::raw_any((const T *)a.q + ((long long)b * a.S + i) * a.ldq + (long long)hq * a.Dh + chunk * EPC);
#pragma unroll
    for (int e = 0; e < EPC; ++e) {
      q[r][e] = (float)v.v[e];
      acc[r][e] = 0.f;
    }
    m[r] = kNegInf;
    l[r] = 0.f;
  }
  const float *mask = !PAGED && a.mask ? a.mask + (long long)b * a.Sk : nullptr;
  if (!PAGED && mask && plan.edges) {
    const int2 e = plan.edges[b];
    lo = e.x;
    hi2 = e.y;
  } else if (!PAGED && mask) {  // the first and the last valid position
    mask_ends<SHARE ? 4 : 8>(mask, a.Sk, SHARE ? threadIdx.x : lane, SHARE ? 256 : 64, lo, hi2);
    lo = wave_ext<int, false>(lo);
    hi2 = wave_ext<int, true>(hi2);
    if (SHARE) {
      if (lane == 0) found[wave] = make_int2(lo, hi2);
      __syncthreads();
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const int2 e = found[v];
        lo = min(lo, e.x);
        hi2 = max(hi2, e.y);
      }
    }
  }
  lo &= ~(KT - 1);
  int nt = hi2 > lo ? (hi2 - lo + KT - 1) / KT : 0;  // tiles of keys, this part's of them
  {
    const int per = (nt + plan.parts - 1) / plan.parts;
    const int t0 = min(nt, part * per);
    nt = min(nt, t0 + per) - t0;
    lo += t0 * KT;
  }
  // ---- keys and values: RSTEP rows a load, which lie in one page
  const int last = hi2 - 1, rowb = a.Dh * ES, plog = a.page_log2, pmask = (1 << plog) - 1, col = feature ? chunk * 16 : 0;
  const unsigned page_bytes = ((unsigned)a.Hk << plog) * rowb;
  const int32_t *const table = PAGED ? a.table + (long long)b * a.n_blocks : nullptr;
  const long long ldk = a.ldk * ES, ldv = a.ldv * ES;
  const char *const kbase = (const char *)a.k + (PAGED ? ((long long)h << plog) * rowb : (long long)b * a.Sk * ldk + h * rowb);
  const char *const vbase = (const char *)a.v + (PAGED ? ((long long)h << plog) * rowb : (long long)b * a.Sk * ldv + h * rowb);
  int pg[NL], next[NL], bad = 0;
  float valid = 1.f;
  unsigned long long there = ~0ull, there_next = ~0ull;  // keys of a tile that are there and not masked
  auto look = [&](int k0) {  // what the tile at k0 will need
    if (PAGED) {
#pragma unroll
      for (int x = 0; x < NL; ++x) next[x] = table[min(k0 + x * RSTEP, last) >> plog];
    } else if (mask) {
      valid = mask[min(k0 + lane, last)];
    }
  };
  auto begin = [&](int k0) {
    if (PAGED) {
#pragma unroll
      for (int x = 0; x < NL; ++x) {
        pg[x] = min(max(next[x], 0), a.n_pages - 1);
        bad |= pg[x] ^ next[x];
      }
    } else {
      there_next = __ballot(lane >= KT || (k0 + lane <= last && (!mask || valid != 0.f)));
    }
  };
  auto load = [&](Words(&to)[NL], int k0, const char *base, long long ld) {
#pragma unroll
    for (int x = 0; x < NL; ++x) {
      if (PAGED) {  // positions behind the last key are read too, inside its page
        const unsigned long long at =
            (unsigned long long)(unsigned)pg[x] * page_bytes + (unsigned)((k0 + x * RSTEP) & pmask) * rowb;
        to[x] = *(const Words *)(base + at + (unsigned)(group * rowb + col));
      } else {  // rows behind the last key stand for it
        const int j = min(k0 + x * RSTEP + group, last);
        to[x] = *(const AnyWords *)(base + j * ld + col);
      }
    }
  };
  Words kr[NL], vr[NL];
  const int every = SHARE ? 4 : 1;
  int t = SHARE ? wave : 0;
  const int t_first = t;
  if (t < nt) {
    look(lo + t * KT);
    begin(lo + t * KT);
    load(kr, lo + t * KT, kbase, ldk);
    load(vr, lo + t * KT, vbase, ldv);
    look(lo + (t + every) * KT);
  }
  for (; t < nt; t += every) {
    const int k0 = lo + t * KT, k1 = k0 + every * KT;
    const bool more = t + every < nt;
    there = there_next;
    float s[NR][NL];
    if (rowb != DP * ES && !feature) {  // columns that only pad have read the first one
#pragma unroll
      for (int x = 0; x < NL; ++x) kr[x] = 0u;
    }
#pragma unroll
    for (int x = 0; x < NL; ++x) {
      if (ES == 2) asm volatile("" : "+v"(kr[x]));  // or they cross the loop as floats, and spill
      float k[EPC];
#pragma unroll
      for (int e = 0; e < EPC; ++e) k[e] = word_at<T>(kr[x], e);
#pragma unroll
      for (int r = 0; r < NR; ++r) {
        float d = 0.f;
#pragma unroll
        for (int e = 0; e < EPC; ++e) d = fmaf(q[r][e], k[e], d);
        s[r][x] = chunk_sum<CH>(d);
      }
    }
    if (more) {
      begin(k1);
      load(kr, k1, kbase, ldk);
    }
    // ---- keys that a row does not see
    unsigned hidden[NR] = {};  // by load
    const bool some = PAGED ? k0 + KT > hi || k0 < lo2 : there != ~0ull;
    if (some) {
#pragma unroll
      for (int r = 0; r < NR; ++r)
#pragma unroll
        for (int x = 0; x < NL; ++x) {
          const int kk = x * RSTEP + group;
          const bool ok = PAGED ? k0 + kk >= qlo[r] && k0 + kk < qhi[r] : (there >> kk) & 1;
          if (!ok) {
            s[r][x] = kNegInf;
            hidden[r] |= 1u << x;
          }
        }
    }
    // ---- weights: the maximum moves where a score passes it by 2^8, as in the step kernel.  It is one of the scores before the
    // scale, so that differences to it are exact near it, whatever the scores' size
    auto larger = [](float x, float y) { return fmaxf(x, y); };
#pragma unroll
    for (int r = 0; r < NR; ++r) {
      float mx = s[r][0];
#pragma unroll
      for (int x = 1; x < NL; ++x) mx = fmaxf(mx, s[r][x]);
      mx = across<CH>(mx, larger);
      if (__any((mx - m[r]) * a.scale > 8.f)) {
        const float mn = fmaxf(m[r], mx), c = m[r] == kNegInf ? 0.f : __builtin_amdgcn_exp2f((m[r] - mn) * a.scale);
        m[r] = mn;
        l[r] *= c;
#pragma unroll
        for (int e = 0; e < EPC; ++e) acc[r][e] *= c;
      }
      const float use = m[r] == kNegInf ? 0.f : m[r];
#pragma unroll
      for (int x = 0; x < NL; ++x) {
        s[r][x] = __builtin_amdgcn_exp2f((s[r][x] - use) * a.scale);
        l[r] += s[r][x];
      }
    }
    // ---- values: one that a row does not see has no part in it, whatever it is
    if (some) {
#pragma unroll
      for (int x = 0; x < NL; ++x) {
        if (ES == 2) asm volatile("" : "+v"(vr[x]));
#pragma unroll
        for (int r = 0; r < NR; ++r)
#pragma unroll
          for (int e = 0; e < EPC; ++e) {
            const float v = (hidden[r] >> x) & 1 ? 0.f : word_at<T>(vr[x], e);
            acc[r][e] = fmaf(s[r][x], v, acc[r][e]);
          }
      }
    } else {
#pragma unroll
      for (int x = 0; x < NL; ++x) {
        if (ES == 2) asm volatile("" : "+v"(vr[x]));
#pragma unroll
        for (int e = 0; e < EPC; ++e) {
          const float v = word_at<T>(vr[x], e);
#pragma unroll
          for (int r = 0; r < NR; ++r) acc[r][e] = fmaf(s[r][x], v, acc[r][e]);
        }
      }
    }
    if (more) {
      load(vr, k1, vbase, ldv);
      look(k1 + every * KT);
    }
  }
  if (PAGED && t_first < nt && bad) atomicOr(a.err, kErrPage);
  // ---- results
  auto plus = [](float x, float y) { return x + y; };
#pragma unroll
  for (int r = 0; r < NR; ++r) {
    l[r] = across<CH>(l[r], plus);
#pragma unroll
    for (int e = 0; e < EPC; ++e) acc[r][e] = across<CH>(acc[r][e], plus);
  }
  if constexpr (SHARE) {
    if (lane == 0) {
#pragma unroll
      for (int r = 0; r < NR; ++r) ends[wave][r] = make_float2(m[r], l[r]);
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < NR; ++r) {
      float mm = kNegInf, ll = 0.f;
#pragma unroll
      for (int v = 0; v < 4; ++v) mm = fmaxf(mm, ends[v][r].x);
      const float use = mm == kNegInf ? 0.f : mm;
      auto factor = [&](float x) { return x == kNegInf ? 1.f : __builtin_amdgcn_exp2f((x - use) * a.scale); };  // sums without a maximum: zeros, or NaN
#pragma unroll
      for (int v = 0; v < 4; ++v) ll = fmaf(ends[v][r].y, factor(ends[v][r].x), ll);
      const float c = factor(m[r]);
      if (lane < CH) {
#pragma unroll
        for (int e = 0; e < EPC; e += 4)
          *(float4 *)&sums[wave][r][chunk * EPC + e] = make_float4(acc[r][e] * c, acc[r][e + 1] * c, acc[r][e + 2] * c, acc[r][e + 3] * c);
      }
      m[r] = mm;
      l[r] = ll;
    }
    __syncthreads();
    if (wave != 0) return;
    if (lane < CH) {
#pragma unroll
      for (int r = 0; r < NR; ++r)
#pragma unroll
        for (int e = 0; e < EPC; ++e)
          acc[r][e] = (sums[0][r][chunk * EPC + e] + sums[1][r][chunk * EPC + e]) + (sums[2][r][chunk * EPC + e] + sums[3][r][chunk * EPC + e]);
    }
  }
  if (lane >= CH || !feature) return;
  const long long rows = (long long)a.B * a.Hq * a.S;
  const Parts parts = parts_of(a.ws, rows, plan.parts);
  const long long prow = part * rows + (long long)bh * a.S * a.G + r0;
#pragma unroll
  for (int r = 0; r < NR; ++r) {
    if (r >= R) break;
    const int i = (r0 + r) / a.G, hq = h * a.G + r0 + r - i * a.G;
    if (plan.parts > 1) {
      // the sums relative to the maximum times the scale, rounded: less what that is off by, where it is not all that there is;
      // none where it is minus infinity
      const float ms = m[r] * a.scale, left = ms == kNegInf && m[r] != kNegInf ? 0.f : 1.f;
      const float c = fabsf(ms) < kFarScore ? __builtin_amdgcn_exp2f(fmaf(m[r], a.scale, -ms)) : left;
      float *po = parts.o + (prow + r) * a.Dh + chunk * EPC;
#pragma unroll
      for (int e = 0; e < EPC; e += 4)
        *(float4 *)(po + e) = make_float4(acc[r][e] * c, acc[r][e + 1] * c, acc[r][e + 2] * c, acc[r][e + 3] * c);
      if (lane == 0) parts.ml[prow + r] = make_float2(ms, l[r] * c);
    } else {
      const float inv = l[r] == 0.f ? 0.f : 1.f / l[r];
#pragma unroll
      for (int e = 0; e < EPC; ++e) acc[r][e] = times_or_zero(acc[r][e], inv);
      V::put_any((T *)a.y + ((long long)b * a.S + i) * a.ldy + (long long)hq * a.Dh + chunk * EPC, acc[r]);
    }
  }
}

template <typename T, int DP, int NR, bool PAGED>
hipError_t launch_rows_of(const MhaArgs &a, StepPlan plan, bool share, hipStream_t st) {
  const long long jobs = (long long)a.B * a.Hk * plan.tiles * plan.parts, all = share ? jobs : (jobs + 3) / 4;
  plan.jobs = (unsigned)jobs;
  const long long most = 1 << 22;  // workgroups of a launch
  for (long long first = 0; first < all; first += most) {
    plan.first = (int)first;
    const dim3 grid((unsigned)(all - first < most ? all - first : most)), block(256);
    if (share)
      hipLaunchKernelGGL((row_kernel<T, DP, NR, PAGED, true>), grid, block, 0, st, a, plan);
    else
      hipLaunchKernelGGL((row_kernel<T, DP, NR, PAGED, false>), grid, block, 0, st, a, plan);
  }
  return hipGetLastError();
}

template <typename T, int NR, bool PAGED>
hipError_t launch_rows_as(const MhaArgs &a, const StepPlan &plan, bool share, hipStream_t st) {
  if constexpr (few_rows(NR, 128, sizeof(T) == 4)) {
    if (a.Dh <= 64) return launch_rows_of<T, 64, NR, PAGED>(a, plan, share, st);
    if (a.Dh <= 128) return launch_rows_of<T, 128, NR, PAGED>(a, plan, share, st);
  }
  return launch_rows_of<T, 256, NR, PAGED>(a, plan, share, st);
}

// rows of which few_rows holds
template <typename T>
hipError_t launch_rows_typed(const MhaArgs &a, const StepPlan &plan, bool share, hipStream_t st) {
  const bool one = (long long)a.S * a.G == 1;
  if (a.table) return one ? launch_rows_as<T, 1, true>(a, plan, share, st) : launch_rows_as<T, kRowRows, true>(a, plan, share, st);
  return one ? launch_rows_as<T, 1, false>(a, plan, share, st) : launch_rows_as<T, kRowRows, false>(a, plan, share, st);
}

hipError_t launch_rows_bf16(const MhaArgs &a, const StepPlan &plan, bool share, hipStream_t st);
hipError_t launch_rows_f32(const MhaArgs &a, const StepPlan &plan, bool share, hipStream_t st);

}  // namespace mt
