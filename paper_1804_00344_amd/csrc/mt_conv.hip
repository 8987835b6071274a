// Causal depthwise convolution of width W <= 8 over prompts and single tokens:
// y[t, d] = act(b[d] + sum_j w[d, j] x[t - W + 1 + j, d]).
//
// Memory-bound: every input is used W times, from registers.  A thread takes VEC neighbouring channels (16 bytes
// where the channels divide into them; rows at odd elements too, 4 x 8192 x 2048 bf16 53 us, channel by channel
// 76) over RUN positions: it requests all their inputs and the W - 1 before them at once, then computes.  Threads
// are numbered channel first, so a wave's accesses are consecutive for any channel count.  A prompt's first
// thread of a channel reads the state before it and is the one that writes the state after it.
#include "mt_layer_dev.h"

namespace mt {

namespace {

template <typename T, int VEC, int W>
__device__ __forceinline__ void load_taps(const ConvArgs &a, int d, float (&w)[W][VEC], float (&b)[VEC]) {
#pragma unroll
  for (int v = 0; v < VEC; ++v) {
    b[v] = a.b[d + v];
#pragma unroll
    for (int j = 0; j < W; ++j) w[j][v] = a.w[(size_t)j * a.D + d + v];
  }
}

template <typename T, int VEC, int W, int RUN, bool STREAM>
__global__ void __launch_bounds__(256) conv_kernel(ConvArgs a) {
  using V = Vec<T, VEC>;
  const int dv = a.D / VEC;
  const int runs = (a.S + RUN - 1) / RUN;
  const long long id = (long long)blockIdx.x * 256 + threadIdx.x;
  if (id >= (long long)runs * dv) return;
  const int run = (int)(id / dv), d = (int)(id - (long long)run * dv) * VEC;
  float w[W][VEC], bias[VEC];
  load_taps<T, VEC, W>(a, d, w, bias);
  for (int b = blockIdx.y; b < a.B; b += gridDim.y) {
    int len = a.S;
    if (a.len) {
      len = a.len[b];
      if (len < 0 || len > a.S) {
        if (id == 0) atomicOr(a.err, 4);
        len = len < 0 ? 0 : a.S;
      }
    }
    const T *x = (const T *)a.x + (long long)b * a.S * a.ldx + d;
    T *y = (T *)a.y + (long long)b * a.S * a.ldy + d;
    const T *st = a.state_in ? (const T *)a.state_in + (long long)b * (W - 1) * a.D + d : nullptr;
    // the input at position t >= 1 - W of this prompt
    auto input = [&](int t) -> typename V::Raw {
      if (t >= 0) return V::raw_any(x + (long long)t * a.ldx);
      if (st) return V::raw(st + (long long)(t + W - 1) * a.D);
      return {};
    };
    const int t0 = run * RUN, t1 = t0 + RUN < len ? t0 + RUN : len;
    if (t0 < t1) {
      typename V::Raw in[RUN + W - 1];  // positions t0 - W + 1 .. t0 + RUN - 1, behind the end the last one
#pragma unroll
      for (int j = 0; j + 1 < W; ++j) in[j] = input(t0 - W + 1 + j);
#pragma unroll
      for (int i = 0; i < RUN; ++i) in[W - 1 + i] = V::raw_any(x + (long long)min(t0 + i, t1 - 1) * a.ldx);
#pragma unroll
      for (int i = 0; i < RUN; ++i) {
        float o[VEC];
#pragma unroll
        for (int v = 0; v < VEC; ++v) {
          o[v] = bias[v];
#pragma unroll
          for (int j = 0; j < W; ++j) o[v] = fmaf(w[j][v], (float)in[i + j].v[v], o[v]);
          if (a.silu) o[v] = silu(o[v]);
        }
        if (t0 + i >= t1) continue;
        if constexpr (STREAM)
          V::template put<true>(y + (long long)(t0 + i) * a.ldy, o);
        else
          V::put_any(y + (long long)(t0 + i) * a.ldy, o);
      }
    }
    if (run == 0 && W > 1 && a.state_out) {
      T *so = (T *)a.state_out + (long long)b * (W - 1) * a.D + d;
#pragma unroll
      for (int j = 0; j + 1 < W; ++j) *(typename V::Raw *)(so + (long long)j * a.D) = input(len - W + 1 + j);
    }
  }
}

// One token of a hypothesis: its state row is read whole before its new one is written (they may be
// the same one).  A few bytes per thread and no reuse: 768 x 2048, W = 4, bf16 7.5 us (25 MB of traffic, a
// launch's latency and 4.9 us at a copy's rate), one row 2.7.
template <typename T, int VEC, int W>
__global__ void __launch_bounds__(256) conv_step_kernel(ConvArgs a) {
  using V = Vec<T, VEC>;
  const int dv = a.D / VEC;
  const long long id = (long long)blockIdx.x * 256 + threadIdx.x;
  const int m = (int)(id / dv), d = (int)(id - (long long)m * dv) * VEC;
  if (m >= a.B) return;
  int row = m;
  if (a.row) {
    row = a.row[m];
    if (row < 0 || row >= a.n_rows) {
      if (d == 0) atomicOr(a.err, 2);
      row = row < 0 ? 0 : a.n_rows - 1;
    }
  }
  typename V::Raw in[W];
  if constexpr (W > 1) {
    const T *st = (const T *)a.state_in + (long long)row * (W - 1) * a.D + d;
#pragma unroll
    for (int j = 0; j + 1 < W; ++j) in[j] = V::raw(st + (long long)j * a.D);
  }
  in[W - 1] = V::raw_any((const T *)a.x + (long long)m * a.ldx + d);
  float w[W][VEC], o[VEC];
  load_taps<T, VEC, W>(a, d, w, o);
#pragma unroll
  for (int v = 0; v < VEC; ++v) {
#pragma unroll
    for (int j = 0; j < W; ++j) o[v] = fmaf(w[j][v], (float)in[j].v[v], o[v]);
    if (a.silu) o[v] = silu(o[v]);
  }
  V::put_any((T *)a.y + (long long)m * a.ldy + d, o);
  if constexpr (W > 1) {
    T *so = (T *)a.state_out + (long long)m * (W - 1) * a.D + d;
#pragma unroll
    for (int j = 0; j + 1 < W; ++j) *(typename V::Raw *)(so + (long long)j * a.D) = in[j + 1];
  }
}

template <typename T, int VEC, int W, int RUN, bool STREAM>
hipError_t run_prompts(const ConvArgs &a, hipStream_t st) {
  const long long n = ((a.S + RUN - 1) / RUN * (long long)(a.D / VEC) + 255) / 256;
  hipLaunchKernelGGL((conv_kernel<T, VEC, W, RUN, STREAM>), dim3((unsigned)n, (unsigned)(a.B < 32768 ? a.B : 32768)),
                     dim3(256), 0, st, a);
  return hipGetLastError();
}

// Runs of 8 positions once those of 4 fill the chip four times over (4 x 8192 x 2048, W = 4: 60 us, runs of 4
// and 16: 71 and 62; 3 x 61 x 333: 3.1 us with runs of 4, 6.5 with one position after the other).
// Aligned outputs larger than the L2s together are stored past them (60 -> 56 us); smaller ones stay for
// the product that reads them.
template <typename T, int VEC, int W>
hipError_t run_conv(const ConvArgs &a, bool step, hipStream_t st) {
  const long long dv = a.D / VEC;
  if (step) {
    hipLaunchKernelGGL((conv_step_kernel<T, VEC, W>), dim3((unsigned)((a.B * dv + 255) / 256)), dim3(256), 0, st, a);
    return hipGetLastError();
  }
  const double n = (double)a.B * a.S * dv;  // vectors
  const bool aligned = (uintptr_t)a.y % 16 == 0 && a.ldy % VEC == 0;
  if (VEC > 1 && aligned && n * 16 > 32e6) return run_prompts<T, VEC, W, 8, VEC != 1>(a, st);
  if (n >= 4.0 * 64 * 16 * a.num_cu) return run_prompts<T, VEC, W, 8, false>(a, st);
  return run_prompts<T, VEC, W, 4, false>(a, st);
}

template <typename T, int VEC>
hipError_t by_width(const ConvArgs &a, bool step, hipStream_t st) {
  switch (a.W) {
    case 1: return run_conv<T, VEC, 1>(a, step, st);
    case 2: return run_conv<T, VEC, 2>(a, step, st);
    case 3: return run_conv<T, VEC, 3>(a, step, st);
    case 4: return run_conv<T, VEC, 4>(a, step, st);
    case 5: return run_conv<T, VEC, 5>(a, step, st);
    case 6: return run_conv<T, VEC, 6>(a, step, st);
    case 7: return run_conv<T, VEC, 7>(a, step, st);
    default: return run_conv<T, VEC, 8>(a, step, st);
  }
}

template <typename T>
hipError_t by_vector(const ConvArgs &a, bool step, hipStream_t st) {
  constexpr int VEC = 16 / sizeof(T);
  return a.D % VEC == 0 ? by_width<T, VEC>(a, step, st) : by_width<T, 1>(a, step, st);
}

}  // namespace

hipError_t launch_conv(const ConvArgs &a, hipStream_t st) {
  return a.bf16_io ? by_vector<bf16>(a, false, st) : by_vector<float>(a, false, st);
}
hipError_t launch_conv_step(const ConvArgs &a, hipStream_t st) {
  return a.bf16_io ? by_vector<bf16>(a, true, st) : by_vector<float>(a, true, st);
}

}  // namespace mt
