// Norms of the heads of queries and keys, their rotation by position, and the store of keys and values into the
// pages of a cache, in one pass:  n = x / sqrt(mean(x^2) + eps) g,  (u, w) -> (u cos - w sin, w cos + u sin).
#include "mt_layer_dev.h"
#include "mt_mha.h"

namespace mt {

namespace {

// v of lane ^ O within groups of more than O lanes
template <int O>
__device__ __forceinline__ float lane_xor(float v) {
  if constexpr (O == 1) return dpp_mov<kDppQuadSwap1>(v);
  if constexpr (O == 2) return dpp_mov<kDppQuadSwap2>(v);
  if constexpr (O == 4) return dpp_mov<0x1B>(dpp_mov<0x141>(v));  // eight lanes reversed, then each four
  if constexpr (O == 8) return dpp_mov<kDppRowRor8>(v);
  if constexpr (O == 16) return __shfl_xor(v, 16);
  if constexpr (O == 32) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_int(v), __float_as_int(v), false, false);
    return __int_as_float((threadIdx.x & 32) ? r[0] : r[1]);
  }
  return 0.f;
}

template <int O, int LP, int U>
__device__ __forceinline__ void head_sums(float (&v)[U]) {
  if constexpr (O < LP) {
    float other[U];
#pragma unroll
    for (int u = 0; u < U; ++u) other[u] = lane_xor<O>(v[u]);
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] += other[u];
    head_sums<O * 2, LP, U>(v);
  }
}

template <typename T, bool STREAM, int VEC>
__device__ __forceinline__ void put_rows(T *p, const float (&x)[VEC]) {
  if constexpr (STREAM)
    Vec<T, VEC>::template put<true>(p, x);
  else
    Vec<T, VEC>::put_any(p, x);
}

// A head takes LP lanes (a power of two) of VEC features each, one 16-byte access per lane, and a lane U heads at a
// time, step by step together: one, as more waves bring more loads on their way than more heads of a lane do (8 x 4096 x
// 48 heads of 128 in bf16: one 157 us, 5.1 TB/s, two 166, four 210).  The loops over them stay for the order that the compiler
// makes of them: written out for one, calls of few positions took 1 to 4% longer (151 tokens of 80 heads of 128 5.5 -> 5.9 us).
// A workgroup takes TOK positions of a row, whose angles its threads form first and all heads share: in 64 bits, as turns, so that the factor and the product are off by 2^-53 of
// themselves each and what is left of the last turn by 2^-26 of one (1.6 roundings of 32 bits, in radians).  Partners of a rotation
// come from the lane half a head away where the lanes are a whole head, else through LDS.
template <typename T, int LP, int TOK, bool STREAM>
__global__ void __launch_bounds__(256) append_kernel(AppendArgs a, int per_row, int base) {
  constexpr int VEC = 16 / sizeof(T), U = 1, HEADS = 256 / LP;
  typedef Vec<T, VEC> V;
  __shared__ __attribute__((aligned(16))) float cs[TOK][2][128];
  __shared__ __attribute__((aligned(16))) float part[256 * VEC];
  const int w = base + blockIdx.x, b = w / per_row, i0 = (w - b * per_row) * TOK;
  const int cap = a.n_blocks << a.page_log2, l0 = a.len[b], n0 = a.n_new ? a.n_new[b] : a.S;
  const int len = min(max(l0, 0), cap), n = min(max(n0, 0), a.S), first = len - n;
  if (i0 == 0 && threadIdx.x == 0 && (len != l0 || n != n0)) atomicOr(a.err, kErrLen);
  const int toks = min(TOK, n - i0);
  if (toks <= 0) return;
  const int half = a.rot / 2, H = a.Hq + a.Hk, pmask = (1 << a.page_log2) - 1;
  const int chunk = threadIdx.x & (LP - 1), d0 = chunk * VEC, h0 = threadIdx.x / LP;
  const bool in_head = d0 < a.Dh;  // the others only take part in the sums
  const long long row0 = (long long)b * a.S + i0;
  // first feature of a position in the pages, of key head 0
  bool bad = false;
  auto place = [&](int pos) {
    const int pg = a.table[(long long)b * a.n_blocks + (pos >> a.page_log2)];
    bad |= (unsigned)pg >= (unsigned)a.n_pages;
    return ((((long long)min(max(pg, 0), a.n_pages - 1) * a.Hk) << a.page_log2) + (pos & pmask)) * a.Dh;
  };
  const long long head_step = (long long)a.Dh << a.page_log2;
  struct Task {
    int t, h;
  };
  auto next = [&](Task &k, int heads) {
    k.h += HEADS;
    while (k.h >= heads && k.t < toks) {
      k.h -= heads;
      ++k.t;
    }
  };
  // ---- values: copies
  {
    Task k{0, h0};
    while (k.h >= a.Hk && k.t < toks) {
      k.h -= a.Hk;
      ++k.t;
    }
    while (k.t < toks) {
      typename V::Raw in[U];
      long long to[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int pos = first + i0 + k.t;
        to[u] = -1;
        if (k.t < toks && in_head && pos >= 0) {
          in[u] = V::raw_any((const T *)a.v + (row0 + k.t) * a.ldv + k.h * a.Dh + d0);
          to[u] = place(pos) + k.h * head_step + d0;
        }
        next(k, a.Hk);
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (to[u] >= 0) V::template store<STREAM>((T *)a.vp + to[u], in[u]);
    }
  }
  for (int e = threadIdx.x; e < toks * half; e += 256) {
    const int t = e / half, i = e - t * half;
    const double v = (double)(first + i0 + t) * a.turns[i];
    float s, c;
    sincospif(2.0f * (float)(v - rint(v)), &s, &c);
    cs[t][0][i] = c;
    cs[t][1][i] = s;
  }
  float gq[VEC], gk[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) gq[e] = a.gq[d0 + e], gk[e] = a.gk[d0 + e];  // 256 of each are there
  __syncthreads();
  float *const mine = part + threadIdx.x * VEC, *const head = part + h0 * LP * VEC;
  const bool whole = half % VEC == 0, swaps = a.rot == LP * VEC && LP > 1;
  Task k{0, h0};
  while (k.h >= H && k.t < toks) {
    k.h -= H;
    ++k.t;
  }
  while (k.t < toks) {
    Task task[U];
    float x[U][VEC];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      task[u] = k;
      typename V::Raw in = {};
      if (k.t < toks && in_head) {
        const T *src = k.h < a.Hq ? (const T *)a.q + (row0 + k.t) * a.ldq + k.h * a.Dh
                                  : (const T *)a.k + (row0 + k.t) * a.ldk + (k.h - a.Hq) * a.Dh;
        in = V::raw_any(src + d0);
      }
#pragma unroll
      for (int e = 0; e < VEC; ++e) x[u][e] = (float)in.v[e];
      next(k, H);
    }
    if (a.norm) {
      float ss[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        ss[u] = 0.f;
#pragma unroll
        for (int e = 0; e < VEC; ++e) ss[u] = fmaf(x[u][e], x[u][e], ss[u]);
      }
      head_sums<1, LP, U>(ss);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const float r = rsqrtf(fmaf(ss[u], a.inv_Dh, a.eps));
        const bool q = task[u].h < a.Hq;
#pragma unroll
        for (int e = 0; e < VEC; ++e) x[u][e] = x[u][e] * r * (q ? gq[e] : gk[e]);
      }
    }
    if (a.rot && a.rot_pairs) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int t = min(task[u].t, toks - 1);
#pragma unroll
        for (int e = 0; e < VEC; e += 2) {
          if (d0 + e < a.rot) {
            const float c = cs[t][0][(d0 + e) >> 1], s = cs[t][1][(d0 + e) >> 1], p = x[u][e], w = x[u][e + 1];
            x[u][e] = p * c - w * s;
            x[u][e + 1] = w * c + p * s;
          }
        }
      }
    } else if (swaps) {
      const bool low = chunk < LP / 2;
      const int i2 = (chunk & (LP / 2 - 1)) * VEC;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int t = min(task[u].t, toks - 1);
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          const float p = lane_xor<(LP > 1 ? LP / 2 : 1)>(x[u][e]), s = cs[t][1][i2 + e];
          x[u][e] = x[u][e] * cs[t][0][i2 + e] + p * (low ? -s : s);
        }
      }
    } else if (a.rot) {
      // the lanes of a head are of one wave, whose LDS accesses are served in order
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int t = min(task[u].t, toks - 1);
#pragma unroll
        for (int e = 0; e < VEC; e += 4) *(float4 *)(mine + e) = make_float4(x[u][e], x[u][e + 1], x[u][e + 2], x[u][e + 3]);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        if (d0 >= a.rot) {
        } else if (whole) {
          const bool low = d0 < half;
          const float *from = head + (low ? d0 + half : d0 - half);
          const int i2 = low ? d0 : d0 - half;
#pragma unroll
          for (int e = 0; e < VEC; ++e) {
            const float s = cs[t][1][i2 + e];
            x[u][e] = x[u][e] * cs[t][0][i2 + e] + from[e] * (low ? -s : s);
          }
        } else {
#pragma unroll
          for (int e = 0; e < VEC; ++e) {
            const int d = d0 + e;
            if (d < a.rot) {
              const int i2 = d < half ? d : d - half;
              const float p = head[d < half ? d + half : i2], s = cs[t][1][i2];
              x[u][e] = x[u][e] * cs[t][0][i2] + (d < half ? -p : p) * s;
            }
          }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (task[u].t >= toks || !in_head) continue;
      const int pos = first + i0 + task[u].t;
      if (pos < 0) {  // before the row's beginning: no position
#pragma unroll
        for (int e = 0; e < VEC; ++e) x[u][e] = 0.f;
      }
      if (task[u].h < a.Hq)
        put_rows<T, STREAM>((T *)a.qo + (row0 + task[u].t) * a.ldqo + task[u].h * a.Dh + d0, x[u]);
      else if (pos >= 0)
        V::template put<STREAM>((T *)a.kp + place(pos) + (task[u].h - a.Hq) * head_step + d0, x[u]);
    }
  }
  if (bad) atomicOr(a.err, kErrPage);
}

template <typename T, int LP, int TOK, bool STREAM>
void launch_as(const AppendArgs &a, hipStream_t st) {
  const int per_row = (a.S + TOK - 1) / TOK, all = a.B * per_row, most = 1 << 22;  // workgroups of a launch
  for (int base = 0; base < all; base += most)
    hipLaunchKernelGGL((append_kernel<T, LP, TOK, STREAM>), dim3((unsigned)(all - base < most ? all - base : most)), dim3(256), 0, st,
                       a, per_row, base);
}

template <typename T, int LP>
hipError_t by_rows(const AppendArgs &a, hipStream_t st) {
  const bool aligned = (uintptr_t)a.qo % 16 == 0 && a.ldqo % (16 / (int)sizeof(T)) == 0;
  const AppendForm f = append_form(a.B, a.S, a.Hq, a.Hk, a.Dh, sizeof(T), aligned, a.num_cu);
  if (f.stream)
    launch_as<T, LP, 4, true>(a, st);
  else if (f.tokens == 16)
    launch_as<T, LP, 16, false>(a, st);
  else if (f.tokens == 4)
    launch_as<T, LP, 4, false>(a, st);
  else
    launch_as<T, LP, 1, false>(a, st);
  return hipGetLastError();
}

// lanes of a head
int head_lanes(int Dh, int esize) {
  int n = 1;
  while (n * 16 < Dh * esize) n *= 2;
  return n;
}

template <typename T>
hipError_t by_lanes(const AppendArgs &a, hipStream_t st) {
  switch (head_lanes(a.Dh, sizeof(T))) {
    case 1: return by_rows<T, 1>(a, st);
    case 2: return by_rows<T, 2>(a, st);
    case 4: return by_rows<T, 4>(a, st);
    case 8: return by_rows<T, 8>(a, st);
    case 16: return by_rows<T, 16>(a, st);
    case 32: return by_rows<T, 32>(a, st);
  }
  return by_rows<T, 64>(a, st);
}

}  // namespace

// Several positions of a workgroup share its start and keep loads on their way: only where there are enough of them, and
// as many as fill its lanes (87 x 1507 of 2 heads of 64: 4 positions 152 us, 16 97).  Aligned results larger than the
// L2s together are stored past them (8 x 4096 x 48 heads of 128 in bf16: 164 -> 159 us).
AppendForm append_form(int B, int S, int Hq, int Hk, int Dh, int esize, bool aligned, int num_cu) {
  const long long rows = (long long)B * S;
  const int lanes = (Hq + Hk) * head_lanes(Dh, esize);
  if (rows < 16ll * num_cu || S < 4) return {1, false};
  if (aligned && (double)rows * (Hq + 2 * Hk) * Dh * esize > 32e6 && lanes > 128) return {4, true};
  return {lanes <= 128 && rows >= 64ll * num_cu && S >= 16 ? 16 : 4, false};
}

hipError_t launch_append(const AppendArgs &a, hipStream_t st) {
  return a.bf16_io ? by_lanes<bf16>(a, st) : by_lanes<float>(a, st);
}

}  // namespace mt
