// Attention of query heads over keys and values in pages of a cache, or in rows of another length under a mask:
//   y = sum_j softmax_j(scale q.k_j) v_j over the keys that a query sees.
// Here: how a call is split over the chip, and the join of the parts of a key axis that is cut.
#include <algorithm>

#include "mt_mha_row.h"

namespace mt {

namespace {
constexpr int kMaxSort = 1024;
}  // namespace

MhaPlan mha_plan(int Hq, int Hk, int Dh, int B, int S, long long n_keys, int window, bool f32, int num_cu) {
  MhaPlan p;
  const long long rows = (long long)S * (Hq / Hk), heads = (long long)B * Hk;
  if (window && n_keys > (long long)window + S) n_keys = (long long)window + S;  // keys that a row's queries see
  // The key axis is cut until there are enough workgroups; where there are many parts, each has 256 keys at least.  Tiles of
  // 128 rows want what a unit's registers hold, some computing scores while others take exponentials (300 positions over 9000,
  // 32 heads of 128: two a unit 84 us, one 132; 700 over 9000, 32 heads of 64: three 93, two 121; 2048 over 20000, 8 heads of
  // 64: 132 and 127); tiles of 32 want one, as the parts have to be joined (a token over 20000, 32 heads of 128 in 8 groups: 26
  // us, two 30; 6 x 100 queries over 900, 8 heads of 64: 14 us, two 17), but two where long sequences of one tile would get few
  // parts (16 tokens over 10 to 20000 positions 165 -> 116 us, all of 20000 228 -> 231); the vector units want what fits (16
  // tokens of up to 4000 in fp32, 4 groups of 4 heads of 128: one 52 us, two 38; in bf16 of up to 9000, 16 heads of 192: one
  // 304, two 187, four 148).
  // Few parts may be shorter, down to 128 keys (64 of wide heads): 4 queries over 843 positions, 48 heads of 128 in 16 groups, 29
  // -> 23 us in fp32 and 14.7 -> 13.0 in bf16; 200 positions of 4 heads of 192 behind 600 in bf16 28 -> 21; a token over 16242,
  // 8 heads of 128 in 2 groups in bf16: 63 parts 20 us, 126 25.  In bf16 short axes are not worth the join (30 positions over
  // 430, 8 heads of 64: one part 8.3 us, three 11.5).
  const long long coarse = std::max(1ll, n_keys / 256);
  const long long fine = std::max(coarse, std::min(n_keys / (Dh > 128 ? 64 : 128), 32ll));
  auto parts = [&](long long wgs, int a_unit, long long most) {
    const long long want = a_unit * num_cu / wgs;
    return (int)(want < 1 ? 1 : want < most ? want : most);
  };
  const int tile_unit = Dh <= 64 ? 3 : Dh <= 128 ? 2 : 1;
  const long long big = heads * ((rows + kTileRows - 1) / kTileRows);
  // Tiles of 128 rows read the keys a quarter as often as those of 32, which fill the chip and end sooner where there is
  // less to do (heads of 64: 1000 positions of 8 heads 27 us by 128, 13 by 32; 200 over 2000 of 32 heads 32 and 25, of 128
  // heads 53 and 66; heads of 128: 300 over 9000 of 8 heads 75 and 92).
  p.step = Dh <= 128 && (rows <= kStepRows || big * parts(big, tile_unit, coarse) < num_cu || (big < num_cu && n_keys <= (Dh <= 64 ? 4096 : 2048)));
  p.few = few_rows(rows, Dh, f32);
  if (f32 && Dh > 128 && !p.few) {
    // tiles of 128 rows take as long for one row as for all, a round of workgroups as long as some 24 rows a unit by the vector
    // units (200 positions of 4 heads of 192: 78 us by tiles, 23 by rows; 402 x 21 of 2 heads of 224 75 and 42; 400 of 16 heads
    // of 160 in 4 groups, in parts, 66 and 140; in bf16 tiles are as fast, 16 x 12 queries over 300, 8 heads of 256, 27 and 27)
    const long long cut = parts(big, 1, fine), rounds = (big * cut + num_cu - 1) / num_cu;
    p.few = heads * rows * cut < 24ll * num_cu * rounds;
  }
  p.step |= p.few;
  const int per = p.few ? kRowRows : p.step ? kStepRows : kTileRows;
  p.tiles = (int)((rows + per - 1) / per);
  const int unit = !p.step ? tile_unit : !p.few ? (p.tiles == 1 && heads * 4 >= num_cu ? 2 : 1) : rows == 1 ? 4 : 2;
  p.parts = parts(heads * p.tiles, unit, !f32 && Dh <= 128 && n_keys < 512 ? coarse : fine);
  if (!p.step && B > 2 && n_keys > 2ll * S) {
    // Several sequences are often of different lengths: up to twice the parts, where joining them is little beside the products
    // and the rounds do not get longer (12 x 166 positions of 16 heads of 64 in fp32 behind up to 1664: ragged 108 -> 78 us, all
    // alike 205 -> 207; 3 x 500 of 16 heads of 128 in bf16 behind up to 6000: 104 -> 66 and 132 -> 127)
    const long long wgs = heads * p.tiles, slots = (long long)num_cu * unit;
    const long long few_joined = std::max(n_keys / (f32 ? 448 : 1024), n_keys / (16 * rows));
    const auto rounds = [&](long long n) { return (wgs * n + slots - 1) / slots; };
    for (long long n = std::min<long long>(parts(wgs, 2 * unit, coarse), few_joined); n > p.parts; --n)
      if (rounds(n) * p.parts <= rounds(p.parts) * n) p.parts = (int)n;
  }
  // the waves of a workgroup share a row's keys where there are few rows, or long ones (256 tokens of 16 heads over up to 2000
  // 146 -> 131 us; 768 of 8 over up to 512 41 -> 49)
  p.share = heads * p.tiles < 8 * num_cu || n_keys >= 1024;
  if (p.step && !p.few && n_keys < 1024) {  // not where most waves would find no keys, in several rounds
    // (182 x 8 queries over 15, 32 heads of 128 in 8 groups: fp32 77 -> 32 us, bf16 22 -> 13; 200 x 12 over 40, 8 heads of 64, fp32 34 -> 18)
    const long long jobs = heads * p.tiles * p.parts, at_once = num_cu * step_unit(Dh, f32), kt = (n_keys + 31) / 32;
    p.share &= (jobs + at_once - 1) / at_once * ((kt + 3) / 4) <= (jobs + 4 * at_once - 1) / (4 * at_once) * kt;
  }
  // Under a mask over several rounds of workgroups: the longest sentence last would leave most units waiting for it, and
  // every workgroup would look for its sentence's end (8 ragged sentences of up to 2048 x 2048, 16 heads of 64: 101 us as
  // they come, 87 sorted, with the two launches that find the order).  Over pages the ends are known, and sorting 16
  // ragged prompts of up to 2048 gained as often as it lost (86 to 108 us, sorted 92).
  p.sort = !p.step && B >= 4 && B <= kMaxSort && heads * p.tiles * p.parts >= 4 * num_cu;
  // a launch more, where a workgroup alone would take long (12 queries of 8 heads over 30000 positions 29.5 -> 25.7 us, over
  // 10000 16.2 and 15.7, 4 x 10 over 2351 13.0 -> 14.6)
  p.ends = p.sort || n_keys >= 8192;
  return p;
}

namespace {

// The first valid position of each sentence and one past its last: a workgroup each
__global__ void __launch_bounds__(1024) edges_kernel(const float *mask, int S, int2 *edges) {
  __shared__ int lo[16], hi[16];
  const float *m = mask + (long long)blockIdx.x * S;
  int first, last;
  mask_ends<4>(m, S, threadIdx.x, 1024, first, last);
  first = wave_ext<int, false>(first);
  last = wave_ext<int, true>(last);
  const int w = threadIdx.x >> 6;
  if ((threadIdx.x & 63) == 0) lo[w] = first, hi[w] = last;
  __syncthreads();
  if (threadIdx.x != 0) return;
  for (int i = 1; i < 16; ++i) first = min(first, lo[i]), last = max(last, hi[i]);
  edges[blockIdx.x] = make_int2(first, last);
}

// The sentences by their work: a thread each, whose place is the number of those before it
__global__ void __launch_bounds__(kMaxSort) order_kernel(MhaArgs a, const int2 *edges, int *order) {
  __shared__ float work[kMaxSort];
  const int b = threadIdx.x;
  float mine = 0.f;
  if (b < a.B) {
    const int2 e = edges[b];
    mine = (float)row_span<false>(a, b, false).n * max(0, e.y - e.x);
    work[b] = mine;
  }
  __syncthreads();
  if (b >= a.B) return;
  int place = 0;
  for (int o = 0; o < a.B; ++o) place += work[o] > mine || (work[o] == mine && o < b);
  order[place] = b;
}

// The parts of a row together: sums relative to the largest of the parts' maxima.  A wave per row, NF features a lane.
template <typename T, int NF>
__global__ void __launch_bounds__(256) join_kernel(MhaArgs a, int n_parts) {
  const long long rows = (long long)a.B * a.Hq * a.S;
  const long long row = blockIdx.x * 4ll + (threadIdx.x >> 6);
  if (row >= rows) return;
  const int lane = threadIdx.x & 63;
  const long long per = (long long)a.S * a.G, bh = row / per;
  const int rr = (int)(row - bh * per), i = rr / a.G, b = (int)(bh / a.Hk), hq = (int)(bh - (long long)b * a.Hk) * a.G + rr - i * a.G;
  const int n0 = a.n_new ? a.n_new[b] : a.S;
  // the parts hold a sequence's rows one after the other: those of its n queries
  if (i >= min(max(n0, 0), a.S)) return;
  const Parts p = parts_of(a.ws, rows, n_parts);
  // a part per lane for the maxima and factors, a feature per lane for the sums, whose loads do not wait for each other
  float m = kNegInf;
  for (int s0 = 0; s0 < n_parts; s0 += 64) m = fmaxf(m, s0 + lane < n_parts ? p.ml[(s0 + lane) * rows + row].x : kNegInf);
  m = wave_max(m);
  const float use = m == kNegInf ? 0.f : m;
  float l = 0.f, acc[NF] = {};
  int d[NF];
#pragma unroll
  for (int f = 0; f < NF; ++f) d[f] = min(lane + 64 * f, a.Dh - 1);
  for (int s0 = 0; s0 < n_parts; s0 += 64) {
    float2 ml = make_float2(kNegInf, 0.f);
    if (s0 + lane < n_parts) ml = p.ml[(s0 + lane) * rows + row];
    // sums without a maximum are zeros or no numbers; a part that has seen nothing has not written its sums
    const float c = ml.x == kNegInf ? 1.f : __builtin_amdgcn_exp2f(ml.x - use);
    l += wave_sum(ml.y * c);
    const unsigned long long there = __ballot(ml.y != 0.f);
    constexpr int U = 8;
    for (int s1 = 0; s1 < min(64, n_parts - s0); s1 += U) {
      float v[U][NF];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const float *o = p.o + (min(s0 + s1 + u, n_parts - 1) * rows + row) * a.Dh;
#pragma unroll
        for (int f = 0; f < NF; ++f) v[u][f] = o[d[f]];
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const float w = lane_f(c, s1 + u);
        const bool ok = (there >> (s1 + u)) & 1;
#pragma unroll
        for (int f = 0; f < NF; ++f) acc[f] = ok ? fmaf(v[u][f], w, acc[f]) : acc[f];
      }
    }
  }
  T *y = (T *)a.y + ((long long)b * a.S + i) * a.ldy + (long long)hq * a.Dh;
#pragma unroll
  for (int f = 0; f < NF; ++f)
    if (lane + 64 * f < a.Dh) Store<T>::put(y + lane + 64 * f, l == 0.f ? 0.f : acc[f] / l);
}

template <typename T>
void launch_join(const MhaArgs &a, int n_parts, hipStream_t st) {
  const dim3 grid((unsigned)(((long long)a.B * a.Hq * a.S + 3) / 4)), block(256);
  if (a.Dh <= 64)
    hipLaunchKernelGGL((join_kernel<T, 1>), grid, block, 0, st, a, n_parts);
  else if (a.Dh <= 128)
    hipLaunchKernelGGL((join_kernel<T, 2>), grid, block, 0, st, a, n_parts);
  else
    hipLaunchKernelGGL((join_kernel<T, 4>), grid, block, 0, st, a, n_parts);
}

}  // namespace

size_t mha_workspace_bytes(int Hq, int Hk, int Dh, bool f32, int B, int S, long long n_keys, int window, int num_cu) {
  size_t most = 256;  // of both attentions: only that over pages has the window
  for (int w : {window, 0}) {
    const MhaPlan p = mha_plan(Hq, Hk, Dh, B, S, n_keys, w, f32, num_cu);
    size_t n = p.parts > 1 ? (parts_bytes((long long)B * Hq * S, p.parts, Dh) + 255) / 256 * 256 : 256;
    if (p.ends) n += (size_t)kMaxSort * 4 + ((size_t)B * 8 + 255) / 256 * 256;  // behind the parts: places and edges
    if (n > most) most = n;
  }
  return most;
}

hipError_t launch_mha(const MhaArgs &a, hipStream_t st) {
  const MhaPlan p = mha_plan(a.Hq, a.Hk, a.Dh, a.B, a.S, a.table ? (long long)a.n_blocks << a.page_log2 : a.Sk, a.window,
                        !a.bf16_io, a.num_cu);
  int *order = nullptr;
  int2 *edges = nullptr;
  if (p.ends && a.mask) {
    const size_t at = p.parts > 1 ? (parts_bytes((long long)a.B * a.Hq * a.S, p.parts, a.Dh) + 255) / 256 * 256 : 0;
    order = (int *)((char *)a.ws + at);
    edges = (int2 *)(order + kMaxSort);
    hipLaunchKernelGGL(edges_kernel, dim3(a.B), dim3(1024), 0, st, a.mask, a.Sk, edges);
    if (p.sort)
      hipLaunchKernelGGL(order_kernel, dim3(1), dim3(kMaxSort), 0, st, a, edges, order);
    else
      order = nullptr;
  }
  hipError_t e;
  const bool causal = a.table && !a.window && 2ll * a.S >= (long long)a.n_blocks << a.page_log2;  // tiles see different numbers of keys
  if (p.step) {
    // 10 x 591 positions of 3 heads of 128 in fp32 79 -> 71 us, ragged 48 -> 39; behind 700 others, 8 x 64 of 8 heads of 64,
    // where all tiles see as many, 20 -> 24
    const bool falling = causal && (long long)a.B * a.Hk * p.tiles * p.parts > a.num_cu;
    const StepPlan s{p.tiles, p.parts, 0, 0, falling, edges};
    if (p.few)
      e = a.bf16_io ? launch_rows_bf16(a, s, p.share, st) : launch_rows_f32(a, s, p.share, st);
    else
      e = a.bf16_io ? launch_steps_bf16(a, s, p.share, st) : launch_steps_f32(a, s, p.share, st);
  } else {
    TilePlan t{p.tiles, p.parts, 0, false, order, edges};
    t.fold = causal;
    e = a.bf16_io ? launch_tiles_bf16(a, t, st) : launch_tiles_f32(a, t, st);
  }
  if (e != hipSuccess || p.parts == 1) return e;
  a.bf16_io ? launch_join<bf16>(a, p.parts, st) : launch_join<float>(a, p.parts, st);
  return hipGetLastError();
}

}  // namespace mt
