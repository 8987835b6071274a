// Norms of the heads of queries and keys, their rotation by position, and the store of keys and values into the
// pages of a cache, in one pass:  n = x / sqrt(mean(x^2) + eps) g,  (u, w) -> (u cos - w sin, w cos + u sin).
#include "mt_layer_dev.h"
#include "mt_mha.h"

namespace mt {

namespace {

// What a row's lengths say: the position of its first new one and their number (clamped, reported by one lane)
__device__ __forceinline__ void row_lengths(const AppendArgs &a, int b, bool tell, int &first, int &n) {
  const int cap = a.n_blocks << a.page_log2, l0 = a.len[b], n0 = a.n_new ? a.n_new[b] : a.S;
  const int l = min(max(l0, 0), cap);
  n = min(max(n0, 0), a.S);
  if (tell && (l != l0 || n != n0)) atomicOr(a.err, kErrLen);
  first = l - n;
}

// A head takes LP lanes (a power of two) of VEC features each, one 16-byte access per lane; a workgroup takes TOK
// rows, whose angles its threads form first (in 64 bits, as turns: the product keeps 2^-22 of a turn at position
// 2^30) and all heads of the row share.  Partners of a rotation pass through LDS within the head's lanes.
template <typename T, int LP, int TOK>
__global__ void __launch_bounds__(256) append_kernel(AppendArgs a) {
  constexpr int VEC = 16 / sizeof(T);
  typedef Vec<T, VEC> V;
  __shared__ float cs[TOK][2][128];
  __shared__ __attribute__((aligned(16))) float part[256 * VEC];
  const long long row0 = (long long)blockIdx.x * TOK, rows = (long long)a.B * a.S;
  const int half = a.rot / 2, H = a.Hq + 2 * a.Hk;
  for (int e = threadIdx.x; e < TOK * half; e += 256) {
    const int t = e / half, i = e - t * half;
    const long long row = row0 + t;
    if (row >= rows) break;
    int first, n;
    row_lengths(a, (int)(row / a.S), false, first, n);
    const double v = (double)(first + (int)(row % a.S)) * a.turns[i];
    float s, c;
    sincospif(2.0f * (float)(v - rint(v)), &s, &c);
    cs[t][0][i] = c;
    cs[t][1][i] = s;
  }
  __syncthreads();
  const int chunk = threadIdx.x & (LP - 1), d0 = chunk * VEC;
  float *const mine = part + threadIdx.x * VEC, *const head = part + (threadIdx.x & ~(LP - 1)) * VEC;
  const bool whole = half % VEC == 0;  // a lane's partners are one lane's
  for (int u = threadIdx.x / LP; u < TOK * H; u += 256 / LP) {
    const int t = u / H, h = u - t * H;
    const long long row = row0 + t;
    if (row >= rows) break;
    const int b = (int)(row / a.S), i = (int)(row % a.S);
    int first, n;
    row_lengths(a, b, i == 0 && h == 0 && chunk == 0, first, n);
    if (i >= n) continue;
    const bool in_head = d0 < a.Dh;  // the others only take part in the sum
    const int pos = first + i;
    const int kind = h < a.Hq ? 0 : h < a.Hq + a.Hk ? 1 : 2, hk = h - a.Hq - (kind == 2 ? a.Hk : 0);
    if (pos < 0) {  // before the row's beginning: no position
      if (kind == 0 && in_head) {
        const float zero[VEC] = {};
        V::put_any((T *)a.qo + row * a.ldqo + h * a.Dh + d0, zero);
      }
      continue;
    }
    const T *src = kind == 0   ? (const T *)a.q + row * a.ldq + h * a.Dh
                   : kind == 1 ? (const T *)a.k + row * a.ldk + hk * a.Dh
                               : (const T *)a.v + row * a.ldv + hk * a.Dh;
    typename V::Raw in = {};
    if (in_head) in = V::raw_any(src + d0);
    T *dst = nullptr;
    if (kind != 0) {
      int pg = a.table[(long long)b * a.n_blocks + (pos >> a.page_log2)];
      if ((unsigned)pg >= (unsigned)a.n_pages) {
        if (chunk == 0) atomicOr(a.err, kErrPage);
        pg = pg < 0 ? 0 : a.n_pages - 1;
      }
      dst = (T *)(kind == 1 ? a.kp : a.vp) +
            ((((long long)pg * a.Hk + hk) << a.page_log2) + (pos & ((1 << a.page_log2) - 1))) * a.Dh + d0;
    }
    if (kind == 2) {
      if (in_head) *(typename V::Raw *)dst = in;
      continue;
    }
    float x[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) x[e] = (float)in.v[e];
    if (a.norm) {
      float ss = 0.f;
#pragma unroll
      for (int e = 0; e < VEC; ++e) ss = fmaf(x[e], x[e], ss);
#pragma unroll
      for (int o = 1; o < LP; o <<= 1) ss += __shfl_xor(ss, o);
      const float r = rsqrtf(ss / (float)a.Dh + a.eps);
      const float *g = kind == 0 ? a.gq : a.gk;
#pragma unroll
      for (int e = 0; e < VEC; ++e) x[e] = in_head ? x[e] * r * g[d0 + e] : 0.f;
    }
    if (d0 < a.rot) {
      if (a.rot_pairs) {
#pragma unroll
        for (int e = 0; e < VEC; e += 2) {
          if (d0 + e < a.rot) {
            const float c = cs[t][0][(d0 + e) >> 1], s = cs[t][1][(d0 + e) >> 1], p = x[e], w = x[e + 1];
            x[e] = p * c - w * s;
            x[e + 1] = w * c + p * s;
          }
        }
      } else {
        // the lanes of a head are of one wave, whose LDS accesses are served in order
#pragma unroll
        for (int e = 0; e < VEC; e += 4) *(float4 *)(mine + e) = make_float4(x[e], x[e + 1], x[e + 2], x[e + 3]);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        float p[VEC];
        if (whole) {
          const float *from = head + (d0 < half ? d0 + half : d0 - half);
#pragma unroll
          for (int e = 0; e < VEC; e += 4) {
            const float4 f = *(const float4 *)(from + e);
            p[e] = f.x; p[e + 1] = f.y; p[e + 2] = f.z; p[e + 3] = f.w;
          }
        } else {
#pragma unroll
          for (int e = 0; e < VEC; ++e) {
            const int d = d0 + e;
            p[e] = d < a.rot ? head[d < half ? d + half : d - half] : 0.f;
          }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          const int d = d0 + e;
          if (d < a.rot) {
            const int i2 = d < half ? d : d - half;
            const float s = cs[t][1][i2];
            x[e] = x[e] * cs[t][0][i2] + p[e] * (d < half ? -s : s);
          }
        }
      }
    }
    if (!in_head) continue;
    if (kind == 0)
      V::put_any((T *)a.qo + row * a.ldqo + h * a.Dh + d0, x);
    else
      V::put(dst, x);
  }
}

template <typename T, int LP>
hipError_t by_rows(const AppendArgs &a, hipStream_t st) {
  const long long rows = (long long)a.B * a.S;
  // several rows of a workgroup share nothing but its start: only where there are enough of them
  if (rows >= 16ll * a.num_cu)
    hipLaunchKernelGGL((append_kernel<T, LP, 4>), dim3((unsigned)((rows + 3) / 4)), dim3(256), 0, st, a);
  else
    hipLaunchKernelGGL((append_kernel<T, LP, 1>), dim3((unsigned)rows), dim3(256), 0, st, a);
  return hipGetLastError();
}

template <typename T>
hipError_t by_lanes(const AppendArgs &a, hipStream_t st) {
  const int lanes = (a.Dh * (int)sizeof(T) + 15) / 16;
  if (lanes <= 1) return by_rows<T, 1>(a, st);
  if (lanes <= 2) return by_rows<T, 2>(a, st);
  if (lanes <= 4) return by_rows<T, 4>(a, st);
  if (lanes <= 8) return by_rows<T, 8>(a, st);
  if (lanes <= 16) return by_rows<T, 16>(a, st);
  if (lanes <= 32) return by_rows<T, 32>(a, st);
  return by_rows<T, 64>(a, st);
}

}  // namespace

hipError_t launch_append(const AppendArgs &a, hipStream_t st) {
  return a.bf16_io ? by_lanes<bf16>(a, st) : by_lanes<float>(a, st);
}

}  // namespace mt
