// Selective state space scan over prompts and single tokens.  Per channel d with states n:
//   D_t = softplus(dt_t + dt_bias[d]),  h_t[n] = exp(D_t A[d,n]) h_{t-1}[n] + D_t x_t B_t[n],
//   y_t = (sum_n C_t[n] h_t[n] + skip[d] x_t) * silu(z_t).
#include <algorithm>

#include "mt_layer_dev.h"

namespace mt {

namespace {

constexpr int kThreads = 256;

// log(1 + e^v) = max(v, 0) + log1p(e^-|v|), log1p(e) = 2 atanh(s), s = e / (2 + e) <= 1/3, by the
// atanh series to s^17 (its remainder is below 2^-27 of the sum): accurate for small e too, where
// 1 + e would round e away.
__device__ __forceinline__ float softplus(float v) {
  const float e = exp_acc(-fabsf(v));
  const float s = e * rcp_fast(2.0f + e), q = s * s;
  float p = 1.0f / 17.0f;
  p = fmaf(p, q, 1.0f / 15.0f);
  p = fmaf(p, q, 1.0f / 13.0f);
  p = fmaf(p, q, 1.0f / 11.0f);
  p = fmaf(p, q, 1.0f / 9.0f);
  p = fmaf(p, q, 1.0f / 7.0f);
  p = fmaf(p, q, 1.0f / 5.0f);
  p = fmaf(p, q, 1.0f / 3.0f);
  p = fmaf(p, q, 1.0f);
  return fmaxf(v, 0.0f) + 2.0f * s * p;
}

// Sum over the L neighbouring lanes of a channel (a power of two), the result in each
template <int L>
__device__ __forceinline__ float group_sum(float v) {
  if constexpr (L >= 2) v += dpp_mov<kDppQuadSwap1>(v);
  if constexpr (L >= 4) v += dpp_mov<kDppQuadSwap2>(v);
  if constexpr (L >= 8) v += dpp_mov<0x141>(v);   // row_half_mirror: the other four lanes of eight
  if constexpr (L >= 16) v += dpp_mov<0x140>(v);  // row_mirror: the other eight of sixteen
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
  int chunks, chunk_len;  // pieces of the axis
  int tile, ngr;          // positions of B and C staged together, groups of a workgroup's channels
  float *part;            // [B][chunks - 1][D][Np] state of each piece started from zero
  float *dsum;            // [B][chunks - 1][D] sum of D_t over it
};

template <typename T, int NS, int LPC, bool FINAL>
__global__ void __launch_bounds__(kThreads) scan_kernel(ScanArgs a, ScanPlan pl) {
  constexpr int CPB = kThreads / LPC;
  extern __shared__ __attribute__((aligned(16))) float lds[];
  const int tid = threadIdx.x, sub = tid % LPC, n0 = sub * NS;
  const int c0 = blockIdx.x * CPB;
  const int d = min(c0 + tid / LPC, a.D - 1);
  const bool owner = c0 + tid / LPC < a.D;
  const int per = a.D / a.G;
  const int g0 = c0 / per, ngr = min((c0 + CPB - 1) / per, a.G - 1) - g0 + 1, gi = d / per - g0;
  const int tile = pl.tile, chunk = blockIdx.y;
  const int tfl = pl.ngr * a.Np;  // floats of B (and of C) per position
  const bool wide = a.N % 4 == 0;
  const int nn = min(NS, a.N - n0);  // states of this lane that exist
  float A2[NS];
#pragma unroll
  for (int i = 0; i < NS; ++i) A2[i] = a.A2[(size_t)d * a.Np + n0 + i];
  const float dtb = a.dt_bias[d], skip = a.skip[d];
  for (int i = tid; i < tile * tfl * 2; i += kThreads) lds[i] = 0.f;

  for (int b = blockIdx.z; b < a.B; b += gridDim.z) {
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
    float h[NS];
#pragma unroll
    for (int i = 0; i < NS; ++i) h[i] = 0.f;
    float ds = 0.f;
    if constexpr (FINAL) {
      if (a.state_in) load_states<NS>(a.state_in + ((long long)b * a.D + d) * a.N + n0, nn, wide, h);
      for (int c = 0; c < chunk; ++c) {
        const long long o = (long long)b * (pl.chunks - 1) + c;
        float s[NS];
        load_states<NS>(pl.part + (o * a.D + d) * a.Np + n0, NS, true, s);
        const float q = pl.dsum[o * a.D + d];
#pragma unroll
        for (int i = 0; i < NS; ++i) h[i] = fmaf(__builtin_amdgcn_exp2f(q * A2[i]), h[i], s[i]);
      }
    }
    for (int ts = t0; ts < t1; ts += tile) {
      const int nt = min(tile, t1 - ts);
      __syncthreads();
      const int ne = ngr * a.N;
      for (int e = tid; e < nt * ne; e += kThreads) {
        const int t = e / ne, r = e - t * ne, g = r / a.N, n = r - g * a.N;
        const long long o = (r0 + ts + t) * a.ldbc + (long long)(g0 + g) * a.N + n;
        lds[(t * 2) * tfl + g * a.Np + n] = (float)((const T *)a.bm)[o];
        if constexpr (FINAL) lds[(t * 2 + 1) * tfl + g * a.Np + n] = (float)((const T *)a.cm)[o];
      }
      __syncthreads();
      for (int t = 0; t < nt; ++t) {
        const long long r = r0 + ts + t;
        const float xv = (float)((const T *)a.x)[r * a.ldx + d];
        const float dl = softplus((float)((const T *)a.dt)[r * a.lddt + d] + dtb);
        const float dx = dl * xv;
        const float *bp = lds + (t * 2) * tfl + gi * a.Np + n0, *cp = bp + tfl;
        float yv = 0.f;
#pragma unroll
        for (int i = 0; i < NS; ++i) {
          h[i] = fmaf(__builtin_amdgcn_exp2f(dl * A2[i]), h[i], dx * bp[i]);
          if constexpr (FINAL) yv = fmaf(cp[i], h[i], yv);
        }
        if constexpr (FINAL) {
          yv = fmaf(skip, xv, group_sum<LPC>(yv));
          if (a.z) yv *= silu((float)((const T *)a.z)[r * a.ldz + d]);
          if (owner && sub == 0) ((T *)a.y)[r * a.ldy + d] = (T)yv;
        } else {
          ds += dl;
        }
      }
    }
    if constexpr (FINAL) {
      if (owner && a.state_out && t1 == len && nn > 0)
        store_states<NS>(a.state_out + ((long long)b * a.D + d) * a.N + n0, nn, wide, h);
    } else {
      const long long o = (long long)b * (pl.chunks - 1) + chunk;
      if (owner) {
        store_states<NS>(pl.part + (o * a.D + d) * a.Np + n0, NS, true, h);
        if (sub == 0) pl.dsum[o * a.D + d] = ds;
      }
    }
  }
}

// One token of a hypothesis
template <typename T, int LPC>
__global__ void __launch_bounds__(kThreads) scan_step_kernel(ScanArgs a) {
  constexpr int NS = 4, CPB = kThreads / LPC;
  const int tid = threadIdx.x, sub = tid % LPC, n0 = sub * NS;
  const int c = blockIdx.x * CPB + tid / LPC, d = min(c, a.D - 1);
  const int g = d / (a.D / a.G);
  const int nn = min(NS, a.N - n0);
  const bool wide = a.N % 4 == 0;
  for (int m = blockIdx.y; m < a.B; m += gridDim.y) {
    int row = m;
    if (a.row) {
      row = a.row[m];
      if (row < 0 || row >= a.n_rows) {
        if (blockIdx.x == 0 && tid == 0) atomicOr(a.err, 2);
        row = row < 0 ? 0 : a.n_rows - 1;
      }
    }
    float h[NS];
    load_states<NS>(a.state_in + ((long long)row * a.D + d) * a.N + n0, nn, wide, h);
    const float xv = (float)((const T *)a.x)[(long long)m * a.ldx + d];
    const float dl = softplus((float)((const T *)a.dt)[(long long)m * a.lddt + d] + a.dt_bias[d]);
    const float dx = dl * xv;
    const long long o = (long long)m * a.ldbc + (long long)g * a.N + n0;
    float yv = 0.f;
#pragma unroll
    for (int i = 0; i < NS; ++i) {
      if (i < nn) {
        const float bv = (float)((const T *)a.bm)[o + i], cv = (float)((const T *)a.cm)[o + i];
        h[i] = fmaf(__builtin_amdgcn_exp2f(dl * a.A2[(size_t)d * a.Np + n0 + i]), h[i], dx * bv);
        yv = fmaf(cv, h[i], yv);
      }
    }
    yv = fmaf(a.skip[d], xv, group_sum<LPC>(yv));
    if (a.z) yv *= silu((float)((const T *)a.z)[(long long)m * a.ldz + d]);
    if (c < a.D) {
      if (nn > 0) store_states<NS>(a.state_out + ((long long)m * a.D + d) * a.N + n0, nn, wide, h);
      if (sub == 0) ((T *)a.y)[(long long)m * a.ldy + d] = (T)yv;
    }
  }
}

// lanes per channel of the prompt form
int scan_lanes(int Np) { return Np <= 16 ? 1 : Np / 16; }

ScanPlan scan_plan(int B, int S, int D, int N, int num_cu) {
  ScanPlan p{};
  const int Np = scan_padded_states(N), lanes = scan_lanes(Np);
  const long long waves = (long long)B * ((D * (long long)lanes + 255) / 256) * 4;
  const long long want = (long long)num_cu * 8;
  const long long chunks = std::max(1ll, std::min({want / waves, (long long)S / 64, 32ll}));
  p.chunk_len = (int)((S + chunks - 1) / chunks + 15) / 16 * 16;
  p.chunks = (S + p.chunk_len - 1) / p.chunk_len;
  return p;
}

template <typename T, int NS, int LPC>
hipError_t run_scan(const ScanArgs &a, ScanPlan pl, hipStream_t st) {
  constexpr int CPB = kThreads / LPC;
  const int per = a.D / a.G;
  pl.ngr = std::min(a.G, (CPB - 1) / per + 2);
  const int per_pos = pl.ngr * a.Np * 2 * 4;
  pl.tile = std::max(1, std::min(16, 32768 / per_pos));
  const size_t lds = (size_t)pl.tile * per_pos;
  const unsigned gx = (unsigned)((a.D + CPB - 1) / CPB), gz = (unsigned)std::min(a.B, 32768);
  if (pl.chunks > 1)
    hipLaunchKernelGGL((scan_kernel<T, NS, LPC, false>), dim3(gx, pl.chunks - 1, gz), dim3(kThreads), lds, st, a, pl);
  hipLaunchKernelGGL((scan_kernel<T, NS, LPC, true>), dim3(gx, pl.chunks, gz), dim3(kThreads), lds, st, a, pl);
  return hipGetLastError();
}

template <typename T>
hipError_t scan_by_states(const ScanArgs &a, const ScanPlan &pl, hipStream_t st) {
  switch (a.Np) {
    case 4: return run_scan<T, 4, 1>(a, pl, st);
    case 8: return run_scan<T, 8, 1>(a, pl, st);
    case 16: return run_scan<T, 16, 1>(a, pl, st);
    case 32: return run_scan<T, 16, 2>(a, pl, st);
    case 64: return run_scan<T, 16, 4>(a, pl, st);
    case 128: return run_scan<T, 16, 8>(a, pl, st);
    default: return run_scan<T, 16, 16>(a, pl, st);
  }
}

template <typename T, int LPC>
hipError_t run_step(const ScanArgs &a, hipStream_t st) {
  constexpr int CPB = kThreads / LPC;
  hipLaunchKernelGGL((scan_step_kernel<T, LPC>), dim3((a.D + CPB - 1) / CPB, (unsigned)std::min(a.B, 32768)),
                     dim3(kThreads), 0, st, a);
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

int scan_padded_states(int N) {
  int p = 4;
  while (p < N) p *= 2;
  return p;
}

size_t scan_workspace_bytes(int B, int S, int D, int N, int num_cu) {
  const ScanPlan p = scan_plan(B, S, D, N, num_cu);
  const size_t n = (size_t)B * (p.chunks - 1) * D;
  return n * 4 * (scan_padded_states(N) + 1) + 256;
}

hipError_t launch_scan(const ScanArgs &a, hipStream_t st) {
  ScanPlan p = scan_plan(a.B, a.S, a.D, a.N, a.num_cu);
  const size_t n = (size_t)a.B * (p.chunks - 1) * a.D;
  p.part = (float *)a.ws;
  p.dsum = p.part + n * a.Np;
  return a.bf16_io ? scan_by_states<bf16>(a, p, st) : scan_by_states<float>(a, p, st);
}

hipError_t launch_scan_step(const ScanArgs &a, hipStream_t st) {
  return a.bf16_io ? step_by_states<bf16>(a, st) : step_by_states<float>(a, st);
}

}  // namespace mt
