// Selective state space scan over prompts and single tokens.  Per channel d with states n:
//   D_t = softplus(dt_t + dt_bias[d]),  h_t[n] = exp(D_t A[d,n]) h_{t-1}[n] + D_t x_t B_t[n],
//   y_t = (sum_n C_t[n] h_t[n] + skip[d] x_t) * silu(z_t).
#include <algorithm>
#include <cmath>

#include "mt_layer_dev.h"

namespace mt {

namespace {

constexpr int kThreads = 256;

// log(1 + e^v) = max(v, 0) + log1p(e^-|v|), log1p(e) = 2 atanh(s), s = e / (2 + e) <= 1/3: accurate for
// small e too, where 1 + e would round e away.  atanh(s) / s is a polynomial of degree 4 in s^2, fitted
// at Chebyshev nodes of [0, 1/9]: within 2^-26.9.
__device__ __forceinline__ float softplus(float v) {
  const float e = exp_acc(-fabsf(v));
  const float s = e * rcp_fast(2.0f + e), q = s * s;
  float p = 0.14087328f;
  p = fmaf(p, q, 0.13980709f);
  p = fmaf(p, q, 0.20012426f);
  p = fmaf(p, q, 0.33333158f);
  p = fmaf(p, q, 1.0f);
  return fmaf(s + s, p, fmaxf(v, 0.0f));
}

// The value of another lane of a row.  All lanes of these patterns exist, and saying so (bound_ctrl) lets the
// compiler make the move part of the instruction that uses it.
template <int CTRL>
__device__ __forceinline__ float lane_mov(float v) {
  return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), CTRL, 0xF, 0xF, true));
}

// Sum over the L neighbouring lanes of a channel (a power of two), the result in each
template <int L>
__device__ __forceinline__ float group_sum(float v) {
  if constexpr (L >= 2) v += lane_mov<kDppQuadSwap1>(v);
  if constexpr (L >= 4) v += lane_mov<kDppQuadSwap2>(v);
  if constexpr (L >= 8) v += lane_mov<0x141>(v);   // row_half_mirror: the other four lanes of eight
  if constexpr (L >= 16) v += lane_mov<0x140>(v);  // row_mirror: the other eight of sixteen
  if constexpr (L >= 32) v += __shfl_xor(v, 16, 64);
  if constexpr (L >= 64) v += __shfl_xor(v, 32, 64);
  return v;
}

// NS states from p (n of them exist, the others are zero)
template <int NS>
__device__ __forceinline__ void load_states(const float *p, int n, bool wide, float (&h)[NS]) {
  if (wide) {
#pragma unroll
    for (int i = 0; i < NS; i += 4) {
      float4 q = make_float4(0.f, 0.f, 0.f, 0.f);
      if (i < n) q = *(const float4 *)(p + i);
      h[i] = q.x; h[i + 1] = q.y; h[i + 2] = q.z; h[i + 3] = q.w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < NS; ++i) h[i] = i < n ? p[i] : 0.f;
  }
}
template <int NS>
__device__ __forceinline__ void store_states(float *p, int n, bool wide, const float (&h)[NS]) {
  if (wide) {
#pragma unroll
    for (int i = 0; i < NS; i += 4)
      if (i < n) *(float4 *)(p + i) = make_float4(h[i], h[i + 1], h[i + 2], h[i + 3]);
  } else {
#pragma unroll
    for (int i = 0; i < NS; ++i)
      if (i < n) p[i] = h[i];
  }
}

struct ScanPlan {
  int lanes;              // lanes per channel
  int chunks, chunk_len;  // pieces of the axis
  int waves, ngr;         // of a workgroup: waves with channels, groups of their channels
  int ordered;            // prompts in the order of longest_first
  float *part;            // [B][chunks - 1][D][Np] state of each piece started from zero
  float *dsum;            // [B][chunks - 1][D] sum of D_t over it
};

// the value of lane j of each group of J lanes
template <int J>
__device__ __forceinline__ float bcast(float v, int j) {
  if constexpr (J == 1) return v;
  if constexpr (J == 2) return j == 0 ? lane_mov<0xA0>(v) : lane_mov<0xF5>(v);
  switch (j) {
    case 0: return lane_mov<0x00>(v);
    case 1: return lane_mov<0x55>(v);
    case 2: return lane_mov<0xAA>(v);
    default: return lane_mov<0xFF>(v);
  }
}
// lane j of each group of J receives the sum over its channel's L lanes of y[j]
template <int L, int J>
__device__ __forceinline__ float transpose_sum(float (&y)[J], int sub) {
  if constexpr (L >= 16)
#pragma unroll
    for (int j = 0; j < J; ++j) y[j] += lane_mov<0x140>(y[j]);  // row_mirror: lane 15 - l
  if constexpr (L >= 8)
#pragma unroll
    for (int j = 0; j < J; ++j) y[j] += lane_mov<0x141>(y[j]);  // row_half_mirror: lane 7 - l
  if constexpr (J == 1) {
    return y[0];
  } else {
    const bool o1 = sub & 1, o2 = sub & 2;
    const float a = (o1 ? y[1] : y[0]) + lane_mov<kDppQuadSwap1>(o1 ? y[0] : y[1]);
    if constexpr (J == 2) {
      return a;
    } else {
      const float b = (o1 ? y[3] : y[2]) + lane_mov<kDppQuadSwap1>(o1 ? y[2] : y[3]);
      return (o2 ? b : a) + lane_mov<kDppQuadSwap2>(o2 ? a : b);
    }
  }
}

// positions of B and C staged together: two tiles of 64 / LPC groups fit into 64 KiB
constexpr int tile_positions(int NS) { return NS <= 8 ? 8 : 4; }

// elements of B and C of the next tile that a thread holds in registers
constexpr int scan_stage(int Np) { return Np > 16 ? Np / 16 : 1; }

// The z-th of up to 64 prompts in the order long (more than half of S), middle (more than a quarter),
// short: workgroups are dispatched in the order of z, and a long prompt that starts last ends last.
__device__ __forceinline__ int longest_first(const int32_t *len, int B, int S, int z) {
  const int l = threadIdx.x & 63, n = l < B ? len[l] : 0;
  const bool c0 = l < B && n > S / 2, c1 = l < B && !c0 && n > S / 4, c2 = l < B && !c0 && !c1;
  const uint64_t m0 = __ballot(c0), m1 = __ballot(c1), m2 = __ballot(c2), below = (1ull << l) - 1;
  const int place = c0 ? __popcll(m0 & below) : c1 ? __popcll(m0) + __popcll(m1 & below)
                                                   : __popcll(m0 | m1) + __popcll(m2 & below);
  return __ffsll(__ballot(l < B && place == z)) - 1;
}

// A workgroup takes the channels of its threads / LPC in one piece of a prompt; LPC lanes share a channel,
// NS states each.  The work per position and channel (softplus, gate, skip) is spread over the lanes:
// lane j of each J = min(LPC, 4) does it for the j-th of J positions.  B and C of the next tile and x,
// dt and z of its positions are on their way while a tile is computed.  A tile is always computed whole:
// behind the end the steps D_t are zero, which keeps the state as it is.
// Bound by the vector units, active in 80% (first pass) and 85% (second) of the cycles of 1 x 8192 x 2048 x 16
// (62 and 84 us): an exp2 takes 10 to 11 cycles and does not overlap the products, 3 each, and an
// eighth of the instructions taken out (lane moves within the products, no copies for the output) gave 4%.
// MANY: B and C of a tile, of several groups or many states, are more than a thread holds in scan_stage
// registers.  All 256 threads stage them then, also those of waves without channels, at distances that are
// the same for all threads.  2 x 500 x 1024 x 16 of 1024 groups took 317 us with the staging of one
// group and takes 174, 23 x 1595 x 16 x 16 of 8 groups 79 and 37, 2 x 721 x 16 x 128 of 4 groups 50 and 36; the
// other way round, this staging for one group, 64 x 80 x 2048 x 16 took 32 in place of 29.  Two groups at 32
// states lose by it: 7 x 97 x 330 x 24 of 3 groups 16 and 18.
// PAD: some of the Np states do not exist.  Their A and B are zero, but an infinite D_t x_t times that B, or an
// infinite D_t times that A, is NaN and would be part of y from there on, so they are set to zero at every position
// (16 x 300 x 1024 x 24 50.7 -> 52.3 us, 4 x 600 x 1024 x 100 142 -> 148; a test per four positions in place of it
// 56.5 and 151).  The first pass leaves them: the join clears them.
template <typename T, int NS, int LPC, bool FINAL, bool MANY, bool PAD>
__global__ void __launch_bounds__(256, NS == 4 ? 4 : NS == 8 ? 3 : 2) scan_kernel(ScanArgs a, ScanPlan pl) {
  constexpr int J = LPC < 4 ? LPC : 4, Np = NS * LPC, kTile = tile_positions(NS), SLOTS = kTile / J;
  constexpr int STAGE = MANY ? (Np <= 64 ? 4 : 8) : scan_stage(Np);  // elements a thread holds for the next tile
  extern __shared__ __attribute__((aligned(16))) float lds[];
  const int tid = threadIdx.x, nthr = MANY ? 256 : blockDim.x, sub = tid % LPC, n0 = sub * NS, tj = sub % J;
  const int cpb = (MANY ? pl.waves * 64 : nthr) / LPC, c0 = blockIdx.x * cpb;
  const int d = min(c0 + tid / LPC, a.D - 1);
  const bool owner = c0 + tid / LPC < a.D;
  const bool works = !MANY || ((tid >> 6) < pl.waves && c0 + (tid & ~63) / LPC < a.D);  // the wave has channels
  const int per = a.D / a.G, g0 = c0 / per, gi = d / per - g0;
  const int chunk = blockIdx.y;
  constexpr int nw = FINAL ? 2 : 1;        // the first pass reads B only
  constexpr int grpl = kTile * nw * Np;    // floats of a group's tile
  const int bufl = pl.ngr * grpl;          // and of all groups'
  const bool wide = a.N % 4 == 0, gated = a.z != nullptr;
  const long long ldz = gated ? a.ldz : a.ldx;
  const int nn = min(NS, a.N - n0);        // states of this lane that exist
  float A2[NS];
#pragma unroll
  for (int i = 0; i < NS; ++i) A2[i] = a.A2[(size_t)d * Np + n0 + i];
  const float dtb = a.dt_bias[d], skip = a.skip[d];

  // A tile in LDS: [group][position][B, C][Np], states that do not exist zero.
  // Not MANY: element k of a thread, number tid + k nthr of the tile: its position (none if there is no
  // such element) and its source.
  const T *e_src[STAGE];
  int e_t[STAGE];
  if constexpr (!MANY) {
#pragma unroll
    for (int k = 0; k < STAGE; ++k) {
      const int e = tid + k * nthr, n = e % Np, w = e / Np % nw, g = g0 + e / grpl;
      e_t[k] = e / (Np * nw) % kTile;
      e_src[k] = (const T *)(w ? a.cm : a.bm) + (long long)e_t[k] * a.ldbc + (long long)g * a.N + n;
      if (e >= bufl || n >= a.N || g >= a.G) e_t[k] = 1 << 30;
    }
  }
  // MANY: passes of 256 elements, one per thread: R passes per group, or GP groups per pass.  The place of a
  // thread's elements within a group and their distances are the same in every pass.
  constexpr int R = grpl / 256, GP = R ? 1 : 256 / grpl, ROW = Np * nw, TSTEP = ROW <= 256 ? 256 / ROW : 1;
  const int passes = R ? pl.ngr * R : (pl.ngr + GP - 1) / GP;
  const int en = ROW <= 256 ? tid % Np : tid, et = ROW <= 256 ? tid % grpl / ROW : 0, eg = R ? 0 : tid / grpl;
  const T *const eb = (const T *)a.bm + (long long)g0 * a.N + en, *const ec = (const T *)a.cm + (long long)g0 * a.N + en;
  const T *const esrc = (ROW <= 256 && tid / Np % nw ? ec : eb) + (long long)et * a.ldbc;
  auto element = [&](int k, long long o, int left) -> T {  // of pass k; left: positions of the prompt from the tile on
    const int g = R ? k / (R ? R : 1) : eg + k * GP, q = R ? k % (R ? R : 1) : 0;
    const int t = ROW <= 256 ? et + q * TSTEP : q / nw;
    if (en >= a.N || g >= pl.ngr || g0 + g >= a.G || t >= left) return (T)0.f;
    const T *src = ROW <= 256 ? esrc + (long long)(q * TSTEP) * a.ldbc : (q % nw ? ec : eb) + (long long)t * a.ldbc;
    return src[o + (long long)g * a.N];
  };
  const bool pre = !MANY || passes <= STAGE;
  for (int bz = blockIdx.z; bz < a.B; bz += gridDim.z) {
    int b = bz;
    if (pl.ordered) b = __builtin_amdgcn_readfirstlane(longest_first(a.len, a.B, a.S, bz));
    int len = a.S;
    if (a.len) {
      len = a.len[b];
      if (len < 0 || len > a.S) {
        if (blockIdx.x == 0 && chunk == 0 && tid == 0) atomicOr(a.err, 4);
        len = len < 0 ? 0 : a.S;
      }
    }
    const int t0 = chunk * pl.chunk_len;
    if (t0 >= len && chunk > 0) continue;
    const int t1 = min(t0 + pl.chunk_len, len);
    const long long r0 = (long long)b * a.S;
    T xr[SLOTS], dr[SLOTS], zr[SLOTS], er[STAGE];
    const long long rl = r0 + (t0 < t1 ? scan_first_row(t0, tj, t1) : 0);  // this lane's first row
    const T *px = (const T *)a.x + rl * a.ldx + d, *pd = (const T *)a.dt + rl * a.lddt + d;
    // without a gate its loads are those of x again and its factor is 1: no branch in the loop
    const T *pz = gated ? (const T *)a.z + rl * a.ldz + d : px;
    T *py = (T *)a.y + (r0 + t0 + (J > 1 ? tj : 0)) * a.ldy + d;
    // this lane's next row (slots and tiles in order, ts the tile's first position); behind the end the
    // last row of the lane again, so no row at or behind t1 is read (whole: see scan_whole_tile)
    auto fetch_row = [&](bool whole, int ts, int i) {
      xr[i] = *px;
      dr[i] = *pd;
      if (FINAL) zr[i] = *pz;
      const bool in = scan_next_row(whole, ts, i, J, tj, t1);
      px += in ? J * a.ldx : 0;
      pd += in ? J * a.lddt : 0;
      if (FINAL) pz += in ? J * ldz : 0;
    };
    const long long ob = (r0 + t0) * a.ldbc;
    auto fetch_bc = [&](int ts) {
      const long long o = ob + (ts - t0) * a.ldbc;
#pragma unroll
      for (int k = 0; k < STAGE; ++k) {
        if constexpr (MANY) {
          if (k < passes) er[k] = element(k, o, t1 - ts);
        } else {
          er[k] = (T)0.f;
          if (e_t[k] < t1 - ts) er[k] = e_src[k][o];
        }
      }
    };
    auto stage_bc = [&](int ts, float *buf) {
      if (pre) {
#pragma unroll
        for (int k = 0; k < STAGE; ++k)
          if (tid + k * nthr < bufl) buf[tid + k * nthr] = (float)er[k];
      } else {
        for (int k0 = 0; k0 < passes; k0 += STAGE) {
          T e[STAGE];
#pragma unroll
          for (int k = 0; k < STAGE; ++k) e[k] = element(k0 + k, ob + (ts - t0) * a.ldbc, t1 - ts);
#pragma unroll
          for (int k = 0; k < STAGE; ++k)
            if (tid + (k0 + k) * 256 < bufl) buf[tid + (k0 + k) * 256] = (float)e[k];
        }
      }
    };
    float h[NS];
#pragma unroll
    for (int i = 0; i < NS; ++i) h[i] = 0.f;
    if (FINAL && chunk > 0)  // as scan_join_kernel left it
      load_states<NS>(pl.part + (((long long)b * (pl.chunks - 1) + chunk - 1) * a.D + d) * Np + n0, NS, true, h);
    else if (FINAL && a.state_in)
      load_states<NS>(a.state_in + ((long long)b * a.D + d) * a.N + n0, nn, wide, h);
    float ds = 0.f;
    __syncthreads();  // the last tile of another prompt
    if (t0 < t1) {
      if (works) {
#pragma unroll
        for (int i = 0; i < SLOTS; ++i) fetch_row(false, t0, i);
      }
      if (pre) fetch_bc(t0);
      stage_bc(t0, lds);
    }
    // the positions of a tile.  WHOLE: neither they nor the lanes' rows after it come to the end
    auto compute = [&](auto whole, int ts, const float *buf) {
      constexpr bool WHOLE = decltype(whole)::value;
#pragma unroll
      for (int i = 0; i < SLOTS; ++i) {
        const bool in = WHOLE || ts + i * J + tj < t1;
        const float xv = (float)xr[i], zv = FINAL ? (float)zr[i] : 0.f;
        float dl = softplus((float)dr[i] + dtb);
        fetch_row(WHOLE, ts + kTile, i);
        dl = in ? dl : 0.f;
        const float dx = in ? dl * xv : 0.f;
        float y[J];
#pragma unroll
        for (int j = 0; j < J; ++j) {
          const float *bq = buf + (i * J + j) * nw * Np, *cq = bq + Np;
          float b[NS], c[NS];  // read at once: by turns with the states 4 x 600 x 1024 x 100 took 160 us, so 147
#pragma unroll
          for (int n = 0; n < NS; ++n) {
            b[n] = bq[n];
            if (FINAL) c[n] = cq[n];
          }
          const float dlj = bcast<J>(dl, j), dxj = bcast<J>(dx, j);
          float ys[2], e[NS];
#pragma unroll
          for (int n = 0; n < NS; ++n) e[n] = dlj * A2[n];
#pragma unroll
          for (int n = 0; n < NS; ++n) {
            h[n] = fmaf(__builtin_amdgcn_exp2f(e[n]), h[n], dxj * b[n]);
            if (PAD) h[n] = n < nn ? h[n] : 0.f;
            if constexpr (FINAL) ys[n & 1] = n < 2 ? c[n] * h[n] : fmaf(c[n], h[n], ys[n & 1]);
          }
          if constexpr (FINAL) {
            y[j] = ys[0] + ys[1];
            asm volatile("" : "+v"(y[j]));
          }
          // the next position's B and C are read when this one's states and output are done: the compiler
          // would otherwise read those of many positions at once and spill, or copy the states for the
          // output (2 x 500 x 512 x 256: 161 us without the output's tie, 117 with it)
#pragma unroll
          for (int n = 0; n < NS; ++n)
            asm volatile("" : "+v"(h[n])::"memory");
        }
        if constexpr (FINAL) {
          const float yv = fmaf(skip, xv, transpose_sum<LPC, J>(y, sub)), g = silu(zv);
          // lanes past the last channel, and the lanes of a channel past its first J, hold the value
          // of another lane and store it again
          if (in) *py = (T)(yv * (gated ? g : 1.f));
          py += J * a.ldy;
        } else {
          ds += dl;
        }
      }
    };
    int p = 0;
    for (int ts = t0; ts < t1; ts += kTile) {
      __syncthreads();  // this tile is staged, and nobody reads the other buffer any more
      const bool more = ts + kTile < t1;
      if (more && pre) fetch_bc(ts + kTile);
      const float *buf = lds + p * bufl + gi * grpl + n0;
      if (!works) {
      } else if (scan_whole_tile(ts, kTile, J, t1)) {
        compute(std::true_type(), ts, buf);
      } else {
        compute(std::false_type(), ts, buf);
      }
      p ^= 1;
      if (more) stage_bc(ts + kTile, lds + p * bufl);
    }
    if constexpr (FINAL) {
      if (works && owner && a.state_out && t1 == len && nn > 0)
        store_states<NS>(a.state_out + ((long long)b * a.D + d) * a.N + n0, nn, wide, h);
    } else {
      const long long o = (long long)b * (pl.chunks - 1) + chunk;
      ds = group_sum<J>(ds);
      if (works && owner) {
        store_states<NS>(pl.part + (o * a.D + d) * Np + n0, NS, true, h);
        if (sub == 0) pl.dsum[o * a.D + d] = ds;
      }
    }
  }
}

// Joins the pieces: part[c] becomes the state after pieces 0 .. c.  A thread takes one state of a
// channel and requests sixteen pieces' values at a time: the pass is a chain of those round trips (64
// pieces of 2048 x 16 states: 7.8 us; eight at a time with four states per thread took 4.5 more).
__global__ void __launch_bounds__(256) scan_join_kernel(ScanArgs a, ScanPlan pl) {
  constexpr int R = 16;
  const long long id = (long long)blockIdx.x * 256 + threadIdx.x;
  const int d = (int)(id / a.Np), n = (int)(id - (long long)d * a.Np);
  if (d >= a.D) return;
  const float A2 = a.A2[id];
  const int nc = pl.chunks - 1;
  for (int b = blockIdx.y; b < a.B; b += gridDim.y) {
    int len = a.len ? a.len[b] : a.S;
    len = len < 0 ? 0 : len > a.S ? a.S : len;
    const int live = min(nc, (len - 1) / pl.chunk_len);  // pieces that another one follows
    float h = a.state_in && n < a.N ? a.state_in[((long long)b * a.D + d) * a.N + n] : 0.f;
    float *part = pl.part + (long long)b * nc * a.D * a.Np + id;
    const float *dsum = pl.dsum + (long long)b * nc * a.D + d;
    const long long sp = (long long)a.D * a.Np;
    for (int c0 = 0; c0 < live; c0 += R) {
      float s[R], w[R];
#pragma unroll
      for (int i = 0; i < R; ++i) {
        const int c = min(c0 + i, live - 1);
        s[i] = part[c * sp];
        w[i] = dsum[(long long)c * a.D];
      }
#pragma unroll
      for (int i = 0; i < R; ++i) {
        if (c0 + i >= live) break;
        // an infinite state outlasts a finite sum of steps, also where its power is below the smallest float
        const float f = fabsf(h) == INFINITY && w[i] < INFINITY ? 1.f : __builtin_amdgcn_exp2f(w[i] * A2);
        h = fmaf(f, h, s[i]);
        if (n >= a.N) h = 0.f;  // a state that does not exist: see PAD
        part[(c0 + i) * sp] = h;
      }
    }
  }
}

// One token of a hypothesis: LPC lanes share a channel, four states each.  Bound by the states' traffic:
// each is read and written once, 16 bytes a lane (two and four hypotheses per thread were no faster).
// WIDE: a lane's four states, and its B and C at any alignment, are one access (N a multiple of 4; 768 x 2048 x
// 16 element by element: 83 us).  STREAM: the new states are stored past the L2.  For states larger than the L2s
// together that is the faster form wherever something else runs between two steps: 768 x 2048 x 16 takes 39 us
// (5.5 TB/s; calls in a graph) against 54 from the same states again, and 49 against 57 with a 154 MB matrix of
// logits written between a step and the next; only steps back to back, which find their states in the last-level
// cache, lose (50 against 38).
template <typename T, int LPC, bool WIDE, bool STREAM>
__global__ void __launch_bounds__(kThreads) scan_step_kernel(ScanArgs a) {
  constexpr int NS = 4, CPB = kThreads / LPC;
  const int tid = threadIdx.x, sub = tid % LPC, n0 = sub * NS;
  const int c = blockIdx.x * CPB + tid / LPC, d = min(c, a.D - 1);
  const int g = d / (a.D / a.G);
  const int nn = min(NS, a.N - n0);
  const bool gated = a.z != nullptr;
  for (int m = blockIdx.y; m < a.B; m += gridDim.y) {
    int row = m;
    if (a.row) {
      row = a.row[m];
      if (row < 0 || row >= a.n_rows) {
        if (blockIdx.x == 0 && tid == 0) atomicOr(a.err, 2);
        row = row < 0 ? 0 : a.n_rows - 1;
      }
    }
    float h[NS], bv[NS], cv[NS];
    load_states<NS>(a.state_in + ((long long)row * a.D + d) * a.N + n0, nn, WIDE, h);
    const float xv = (float)((const T *)a.x)[(long long)m * a.ldx + d];
    const float dv = (float)((const T *)a.dt)[(long long)m * a.lddt + d];
    const float zv = gated ? (float)((const T *)a.z)[(long long)m * a.ldz + d] : 0.f;
    const float4 A2 = *(const float4 *)(a.A2 + (size_t)d * a.Np + n0);
    const float dtb = a.dt_bias[d], skip = a.skip[d];
    const long long o = (long long)m * a.ldbc + (long long)g * a.N + n0;
    if constexpr (WIDE) {
      typename Vec<T, NS>::Raw b4{}, c4{};
      if (nn > 0) {
        b4 = Vec<T, NS>::raw_any((const T *)a.bm + o);
        c4 = Vec<T, NS>::raw_any((const T *)a.cm + o);
      }
#pragma unroll
      for (int i = 0; i < NS; ++i) {
        bv[i] = (float)b4.v[i];
        cv[i] = (float)c4.v[i];
      }
    } else {
#pragma unroll
      for (int i = 0; i < NS; ++i) {
        bv[i] = i < nn ? (float)((const T *)a.bm)[o + i] : 0.f;
        cv[i] = i < nn ? (float)((const T *)a.cm)[o + i] : 0.f;
      }
    }
    const float dl = softplus(dv + dtb), dx = dl * xv;
    const float A[NS] = {A2.x, A2.y, A2.z, A2.w};
    float yv = 0.f;
#pragma unroll
    for (int i = 0; i < NS; ++i) {
      h[i] = fmaf(__builtin_amdgcn_exp2f(dl * A[i]), h[i], dx * bv[i]);
      // states that only pad are not part of the sum: infinite dl and dx times zero are NaN
      if (WIDE || i < nn) yv = fmaf(cv[i], h[i], yv);
    }
    if (WIDE && nn <= 0) yv = 0.f;
    yv = fmaf(skip, xv, group_sum<LPC>(yv));
    if (gated) yv *= silu(zv);
    if (c < a.D) {
      float *so = a.state_out + ((long long)m * a.D + d) * a.N + n0;
      if (STREAM && nn > 0)
        Vec<float, NS>::template put<true>(so, h);
      else if (nn > 0)
        store_states<NS>(so, nn, WIDE, h);
      if (sub == 0) ((T *)a.y)[(long long)m * a.ldy + d] = (T)yv;
    }
  }
}

// groups that n neighbouring channels can touch
int scan_groups(int n, int per, int G) { return std::min({G, n, per % n == 0 ? 1 : (n - 1) / per + 2}); }

// Lanes of a channel: four states each, more where they exceed a row of 16 lanes.  (16 states per lane, one
// lane a channel, spilled or left a SIMD two waves: 1 x 8192 x 2048 x 16 176 us and more; eight per lane
// 156, four 158; 64 x 80 ragged 39 and 33, before the prompts were ordered and B and C of a position read at once.)
int scan_lanes(int Np) { return std::min(Np / 4, 16); }

// Pieces of the axis, by the time they are expected to take: with k waves on a SIMD a wave's position takes
// hypot(0.135, 0.077 k) us, with more than four states per lane hypot(0.11, 0.077 k) for each four, and a
// piece's start as much as six positions (fitted to 2048 channels x 16 states, 8192 positions, k = 1 to 8,
// and to 500 to 600 positions of 100 and 256 states).  Cutting the axis adds a first pass over it (0.75 of the
// second's time) and the join.  Measured, 1 x 8192 x 2048 x 16 in one piece 1343 us, in 16 pieces 187, 32: 152,
// 64: 148, 128: 154; 64 x 80 x 2048 x 16 whole 28, in two pieces 62; 7 x 97 x 330 x 24 whole 22, in 7 pieces
// 18.5; 4 x 600 x 1024 x 100 whole 160, in 16 pieces 199; 2 x 500 x 512 x 256 whole 292, in 8 pieces 92, 16
// (which the rule takes): 99, 32: 116.
ScanPlan scan_plan(int B, int S, int D, int N, int num_cu) {
  const int Np = scan_padded_states(N);
  ScanPlan best{};
  best.lanes = scan_lanes(Np);
  const int ns = Np / best.lanes, tile = tile_positions(ns);
  const double waves = (double)B * ((D * (long long)best.lanes + 63) / 64) / (num_cu * 4);
  double best_us = 1e30;
  for (int chunks = 1; chunks <= 256; chunks *= 2) {
    const int len = chunks == 1 ? S : ((S + chunks - 1) / chunks + tile - 1) / tile * tile;
    const int n = (S + len - 1) / len;
    const double us = (len + 6) * (ns / 4) * std::hypot(ns > 4 ? 0.11 : 0.135, 0.077 * std::max(1.0, waves * n)) *
                          (n > 1 ? 1.75 : 1.0) + (n > 1 ? 6.0 + 0.05 * n : 0.0);
    if (us < best_us) {
      best_us = us;
      best.chunk_len = len;
      best.chunks = n;
    }
  }
  return best;
}

template <typename T, int NS, int LPC>
hipError_t run_scan(const ScanArgs &a, ScanPlan pl, hipStream_t st) {
  const int per = a.D / a.G;
  // a workgroup's channels: fewer where their groups' B and C would not fit into LDS twice
  size_t lds;
  for (pl.waves = std::min(4, (a.D * LPC + 63) / 64);; --pl.waves) {
    pl.ngr = scan_groups(pl.waves * 64 / LPC, per, a.G);
    lds = (size_t)pl.ngr * a.Np * 8 * tile_positions(NS) * 2;
    if (lds <= 65536 || pl.waves == 1) break;
  }
  const bool many = pl.ngr * a.Np * 2 * tile_positions(NS) > scan_stage(a.Np) * pl.waves * 64;
  const int cpb = pl.waves * 64 / LPC;
  const dim3 first((unsigned)((a.D + cpb - 1) / cpb), pl.chunks - 1, (unsigned)std::min(a.B, 32768)),
      second(first.x, pl.chunks, first.z), threads(many ? 256 : pl.waves * 64);
#define MT_SCAN(FINAL, MANY, PAD, GRID, LDS) \
  hipLaunchKernelGGL((scan_kernel<T, NS, LPC, FINAL, MANY, PAD>), GRID, threads, LDS, st, a, pl)
  if (pl.chunks > 1) {
    if (many)
      MT_SCAN(false, true, false, first, lds / 2);
    else
      MT_SCAN(false, false, false, first, lds / 2);
    hipLaunchKernelGGL(scan_join_kernel, dim3((unsigned)(((long long)a.D * a.Np + 255) / 256), first.z), dim3(256), 0, st, a,
                       pl);
  }
  const bool pad = a.N != a.Np;
  if (many && pad)
    MT_SCAN(true, true, true, second, lds);
  else if (many)
    MT_SCAN(true, true, false, second, lds);
  else if (pad)
    MT_SCAN(true, false, true, second, lds);
  else
    MT_SCAN(true, false, false, second, lds);
#undef MT_SCAN
  return hipGetLastError();
}

template <typename T>
hipError_t scan_by_states(const ScanArgs &a, const ScanPlan &pl, hipStream_t st) {
  switch (a.Np) {
    case 4: return run_scan<T, 4, 1>(a, pl, st);
    case 8: return run_scan<T, 4, 2>(a, pl, st);
    case 16: return run_scan<T, 4, 4>(a, pl, st);
    case 32: return run_scan<T, 4, 8>(a, pl, st);
    case 64: return run_scan<T, 4, 16>(a, pl, st);
    case 128: return run_scan<T, 8, 16>(a, pl, st);
    default: return run_scan<T, 16, 16>(a, pl, st);
  }
}

template <typename T, int LPC>
hipError_t run_step(const ScanArgs &a, hipStream_t st) {
  constexpr int CPB = kThreads / LPC;
  const dim3 grid((a.D + CPB - 1) / CPB, (unsigned)std::min(a.B, 32768));
  const bool wide = a.N % 4 == 0;
  if (wide && (double)a.B * a.D * a.N * 4 > 32e6)
    hipLaunchKernelGGL((scan_step_kernel<T, LPC, true, true>), grid, dim3(kThreads), 0, st, a);
  else if (wide)
    hipLaunchKernelGGL((scan_step_kernel<T, LPC, true, false>), grid, dim3(kThreads), 0, st, a);
  else
    hipLaunchKernelGGL((scan_step_kernel<T, LPC, false, false>), grid, dim3(kThreads), 0, st, a);
  return hipGetLastError();
}

template <typename T>
hipError_t step_by_states(const ScanArgs &a, hipStream_t st) {
  switch (a.Np) {
    case 4: return run_step<T, 1>(a, st);
    case 8: return run_step<T, 2>(a, st);
    case 16: return run_step<T, 4>(a, st);
    case 32: return run_step<T, 8>(a, st);
    case 64: return run_step<T, 16>(a, st);
    case 128: return run_step<T, 32>(a, st);
    default: return run_step<T, 64>(a, st);
  }
}

}  // namespace

int scan_walk_rows(int len, int tile, int J, int tj) {
  const int slots = tile / J;
  int held[8];  // the positions in the lane's registers
  int row = scan_first_row(0, tj, len), last = 0;
  bool own = true;
  auto fetch = [&](bool whole, int ts, int i) {
    held[i] = row;
    last = std::max(last, row);
    if (scan_next_row(whole, ts, i, J, tj, len)) row += J;
  };
  for (int i = 0; i < slots; ++i) fetch(false, 0, i);
  for (int ts = 0; ts < len; ts += tile)
    for (int i = 0; i < slots; ++i) {
      const int t = ts + i * J + tj;
      own = own && (t >= len || held[i] == t);
      fetch(scan_whole_tile(ts, tile, J, len), ts + tile, i);
    }
  return own ? last : -1;
}

int scan_padded_states(int N) {
  int p = 4;
  while (p < N) p *= 2;
  return p;
}

int scan_pieces(int B, int S, int D, int N, int num_cu) { return scan_plan(B, S, D, N, num_cu).chunks; }

size_t scan_workspace_bytes(int B, int S, int D, int N, int num_cu) {
  const ScanPlan p = scan_plan(B, S, D, N, num_cu);
  const size_t n = (size_t)B * (p.chunks - 1) * D;
  return n * 4 * (scan_padded_states(N) + 1) + 256;
}

hipError_t launch_scan(const ScanArgs &a, hipStream_t st) {
  ScanPlan p = scan_plan(a.B, a.S, a.D, a.N, a.num_cu);
  const size_t n = (size_t)a.B * (p.chunks - 1) * a.D;
  p.ordered = a.len && a.B > 1 && a.B <= 64 && p.chunks == 1;
  p.part = (float *)a.ws;
  p.dsum = p.part + n * a.Np;
  return a.bf16_io ? scan_by_states<bf16>(a, p, st) : scan_by_states<float>(a, p, st);
}

hipError_t launch_scan_step(const ScanArgs &a, hipStream_t st) {
  return a.bf16_io ? step_by_states<bf16>(a, st) : step_by_states<float>(a, st);
}

}  // namespace mt
