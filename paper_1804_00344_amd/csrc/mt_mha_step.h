// Attention of few query rows: kernel and launch, instantiated by mt_mha_step_*.hip.
#pragma once

#include "mt_mha_tile.h"

namespace mt {

constexpr int kStepRows = 32;

// workgroups of the step kernel that a unit holds
constexpr int step_unit(int Dh, bool f32) { return Dh <= 64 ? (f32 ? 2 : 3) : f32 ? 1 : 2; }

// What a launch of the step kernel has decided
struct StepPlan {
  int tiles;  // of kStepRows rows of a sequence's key head
  int parts;  // the key axis is cut into
  int first;  // workgroup of this launch
  unsigned jobs;  // rows' tiles of all key heads and parts: below 2^31
  bool falling;   // whether a row's tiles differ much in their keys, over several rounds of workgroups
  const int2 *edges;  // of each sentence's mask: its first valid position, one past its last; or NULL: not yet known
};

// Tiles of 32 rows of one key head (as in the tile kernel) and 32 keys at a time, each wave with its own part of LDS and
// no barriers.  SHARE: the four waves of a workgroup take the tiles of keys in turn and join their sums at the end, for
// short latency; else each wave has its own rows, for many of them.  Bound by memory where the cache is long (16 tokens over
// 32768 positions, 8 key heads of 128 in bf16: 367 us, 5.9 TB/s; by tiles of 128 rows 412), by one tile's latency where it is not.
// The 32 columns of a product that one token leaves empty cost nothing then (matrix units 8% busy).
template <typename T, int DP, bool PAGED, bool SHARE>
__global__ void __launch_bounds__(256, step_unit(DP, sizeof(T) == 4)) step_kernel(MhaArgs a, StepPlan plan) {
  constexpr int KT = 32, TB = KT * DP * (int)sizeof(T), DB = DP / 32;
  __shared__ __attribute__((aligned(1024))) char lds[4 * 2 * TB];
  __shared__ float2 ends[4][32];
  __shared__ int2 found[4];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 31;
  // a key head's jobs are neighbours on one XCD; or, falling: the last tiles of all heads, which see the most keys, come first,
  // and no XCD has all of a long sequence's
  const bool falling = PAGED && plan.falling;
  const unsigned w = plan.first + (falling ? blockIdx.x : xcd_remap(blockIdx.x, gridDim.x)), job = SHARE ? w : w * 4 + wave;
  if (job >= plan.jobs) return;
  const int part = (int)(job % (unsigned)plan.parts), u = (int)(job / (unsigned)plan.parts), heads = a.B * a.Hk;
  const int bh = falling ? (u + u / heads) % heads : u / plan.tiles, tile = falling ? plan.tiles - 1 - u / heads : u - bh * plan.tiles;
  const int b = bh / a.Hk, h = bh - b * a.Hk;
  const RowSpan span = row_span<PAGED>(a, b, h == 0 && tile == 0 && part == 0 && lane == 0);
  const int R = span.n * a.G, r0 = tile * kStepRows;
  if (r0 >= R) return;
  const int i_first = r0 / a.G, i_last = min(r0 + kStepRows - 1, R - 1) / a.G;
  int lo, hi, lo2, hi2;  // keys that some row sees: [lo, hi2); that all see: [lo2, hi)
  seen_keys<PAGED>(a, span, i_first, lo, hi);
  seen_keys<PAGED>(a, span, i_last, lo2, hi2);
  // ---- this lane's query
  const int r = r0 + col;
  const bool live = r < R;
  const int qi = (live ? r : R - 1) / a.G, hq = h * a.G + (live ? r : R - 1) - qi * a.G;
  int qlo, qhi;
  seen_keys<PAGED>(a, span, qi, qlo, qhi);
  Rows<T, DP> me;
  me.start((const T *)a.q + ((long long)b * a.S + qi) * a.ldq + (long long)hq * a.Dh, live, a.Dh);
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
  // ---- tiles of keys
  char *const buf = lds + wave * 2 * TB;
  Mover<T, DP, PAGED, KT, 64> mv;
  bool odd = false;
  const int every = SHARE ? 4 : 1;
  int t = SHARE ? wave : 0;
  if (t < nt) {
    mv.start(a, b, h, lane, hi2 - 1, mask);
    mv.look(lo + t * KT);
    mv.fetch(lo + t * KT, every * KT);
  }
  for (; t < nt; t += every) {
    const int k0 = lo + t * KT;
    const bool mixed = k0 + KT > hi || k0 < lo2;
    odd |= mv.put(k0, buf, mixed);
    const unsigned seen = (unsigned)mv.seen;
    // the wave's own LDS accesses are served in order
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    if (t + every < nt) mv.fetch(k0 + every * KT, every * KT);
    f32x16 s[1] = {me.scores(buf, 0)};
    if (PAGED ? mixed : seen != ~0u) hide<PAGED>(s[0], k0, qlo, qhi, seen);
    me.weights(s, a.scale);
    me.values(buf + TB, 0, s[0]);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
  if (PAGED && (SHARE ? wave : 0) < nt && mv.bad) atomicOr(a.err, kErrPage);
  if (PAGED && __any(odd)) {  // values that are no numbers where some rows see them and others not: those that do
    for (t = SHARE ? wave : 0; t < nt; t += every) {
      const int k0 = lo + t * KT;
      if (k0 + KT <= hi && k0 >= lo2) continue;
      mv.put_again(k0, buf);
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
      me.odd_values(buf + TB, 0, k0 + 4 * (lane >> 5) - qlo, max(qhi - qlo, 0));
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
  }
  me.l = both_halves_sum(me.l);
  // ---- results
  const long long rows = (long long)a.B * a.Hq * a.S;
  const Parts parts = parts_of(a.ws, rows, plan.parts);
  const long long prow = part * rows + (long long)bh * a.S * a.G;
  const bool cut = plan.parts > 1;
  T *const y = (T *)a.y + ((long long)b * a.S + qi) * a.ldy + (long long)hq * a.Dh;
  float *const po = parts.o + (prow + r) * a.Dh;
  if (!SHARE) {
    if (live) {
      if (cut)
        me.put_part(po, parts.ml + prow + r, a.Dh);
      else
        me.put(y, a.Dh);
    }
  } else {
    if (lane < 32) ends[wave][lane] = make_float2(me.m, me.l);
    __syncthreads();
    float m = kNegInf, l = 0.f;
#pragma unroll
    for (int v = 0; v < 4; ++v) m = fmaxf(m, ends[v][col].x);
    const float use = m == kNegInf ? 0.f : m;
    auto factor = [&](float x) { return x == kNegInf ? 1.f : __builtin_amdgcn_exp2f(x - use); };  // sums without a maximum: zeros, or NaN
#pragma unroll
    for (int v = 0; v < 4; ++v) l = fmaf(ends[v][col].y, factor(ends[v][col].x), l);
    // a wave's sums take its own part of LDS: group g of four features of a lane at (64 g + lane) * 16
    const float c = factor(me.m);
    float4 *const own = (float4 *)buf;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int e = 0; e < 16; e += 4)
        own[(d * 4 + e / 4) * 64 + lane] = make_float4(me.o[d][e] * c, me.o[d][e + 1] * c, me.o[d][e + 2] * c, me.o[d][e + 3] * c);
    static_assert(DB * 4 * 64 * 16 <= 2 * TB, "the sums fit into the wave's part");
    __syncthreads();
    const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
    for (int x = 0; x < DB; ++x) {  // this wave's quarter of the groups
      const int g = wave * DB + x, f = g * 8 + 4 * (lane >> 5);
      float v[4] = {};
#pragma unroll
      for (int o = 0; o < 4; ++o) {
        const float4 q = ((const float4 *)(lds + o * 2 * TB))[g * 64 + lane];
        v[0] += q.x, v[1] += q.y, v[2] += q.z, v[3] += q.w;
      }
      if (!live || f >= a.Dh) continue;
      if (cut) {
        *(float4 *)(po + f) = make_float4(v[0], v[1], v[2], v[3]);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = times_or_zero(v[e], inv);
        Vec<T, 4>::put_any(y + f, v);
      }
    }
    if (cut && live && wave == 0 && lane < 32) parts.ml[prow + r] = make_float2(m, l);
  }
}

template <typename T, int DP, bool PAGED>
hipError_t launch_steps_of(const MhaArgs &a, StepPlan plan, bool share, hipStream_t st) {
  const long long jobs = (long long)a.B * a.Hk * plan.tiles * plan.parts, all = share ? jobs : (jobs + 3) / 4;
  plan.jobs = (unsigned)jobs;
  const long long most = 1 << 22;  // workgroups of a launch
  for (long long first = 0; first < all; first += most) {
    plan.first = (int)first;
    const dim3 grid((unsigned)(all - first < most ? all - first : most)), block(256);
    if (share)
      hipLaunchKernelGGL((step_kernel<T, DP, PAGED, true>), grid, block, 0, st, a, plan);
    else
      hipLaunchKernelGGL((step_kernel<T, DP, PAGED, false>), grid, block, 0, st, a, plan);
  }
  return hipGetLastError();
}

template <typename T, bool PAGED>
hipError_t launch_steps_as(const MhaArgs &a, const StepPlan &plan, bool share, hipStream_t st) {
  if (a.Dh <= 64) return launch_steps_of<T, 64, PAGED>(a, plan, share, st);
  return launch_steps_of<T, 128, PAGED>(a, plan, share, st);  // of wider heads a tile in flight would not fit a wave's registers
}

hipError_t launch_steps_bf16(const MhaArgs &a, const StepPlan &plan, bool share, hipStream_t st);
hipError_t launch_steps_f32(const MhaArgs &a, const StepPlan &plan, bool share, hipStream_t st);

}  // namespace mt
