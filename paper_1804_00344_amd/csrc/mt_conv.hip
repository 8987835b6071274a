// Causal depthwise convolution of width W <= 8 over prompts and single tokens:
// y[t, d] = act(b[d] + sum_j w[d, j] x[t - W + 1 + j, d]).
//
// Memory-bound: every input is used W times, from registers.  A thread takes VEC neighbouring
// channels (16 bytes where the rows are aligned for it) over a run of kRun positions and keeps the
// last W - 1 inputs in registers, so the inputs are read (1 + (W - 1) / kRun) times, the second time
// mostly from the caches.  Threads are numbered channel first, so a wave's accesses are consecutive
// for any channel count.  A prompt's first thread of a channel reads the state before it and is the
// one that writes the state after it.
#include "mt_layer_dev.h"

namespace mt {

namespace {

constexpr int kRun = 16;

template <typename T, int VEC, int W>
__device__ __forceinline__ void load_taps(const ConvArgs &a, int d, float (&w)[W][VEC], float (&b)[VEC]) {
#pragma unroll
  for (int v = 0; v < VEC; ++v) {
    b[v] = a.b[d + v];
#pragma unroll
    for (int j = 0; j < W; ++j) w[j][v] = a.w[(size_t)j * a.D + d + v];
  }
}

template <typename T, int VEC, int W>
__global__ void __launch_bounds__(256) conv_kernel(ConvArgs a) {
  using V = Vec<T, VEC>;
  const int dv = a.D / VEC;
  const int runs = (a.S + kRun - 1) / kRun;
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
    auto input = [&](int t, float (&f)[VEC]) {
      typename V::Raw r;
      if (t >= 0)
        r = V::raw(x + (long long)t * a.ldx);
      else if (st)
        r = V::raw(st + (long long)(t + W - 1) * a.D);
      else
        r = {};
#pragma unroll
      for (int v = 0; v < VEC; ++v) f[v] = (float)r.v[v];
    };
    const int t0 = run * kRun, t1 = t0 + kRun < len ? t0 + kRun : len;
    if (t0 < t1) {
      float h[W][VEC];  // h[j]: the input of tap j
#pragma unroll
      for (int j = 0; j + 1 < W; ++j) input(t0 - W + 1 + j, h[j + 1]);
      for (int t = t0; t < t1; ++t) {
#pragma unroll
        for (int j = 0; j + 1 < W; ++j)
#pragma unroll
          for (int v = 0; v < VEC; ++v) h[j][v] = h[j + 1][v];
        input(t, h[W - 1]);
        float o[VEC];
#pragma unroll
        for (int v = 0; v < VEC; ++v) {
          o[v] = bias[v];
#pragma unroll
          for (int j = 0; j < W; ++j) o[v] = fmaf(w[j][v], h[j][v], o[v]);
          if (a.silu) o[v] = silu(o[v]);
        }
        V::put(y + (long long)t * a.ldy, o);
      }
    }
    if (run == 0 && W > 1 && a.state_out) {
      T *so = (T *)a.state_out + (long long)b * (W - 1) * a.D + d;
#pragma unroll
      for (int j = 0; j + 1 < W; ++j) {
        float f[VEC];
        input(len - W + 1 + j, f);
        V::put(so + (long long)j * a.D, f);
      }
    }
  }
}

// One token of a hypothesis: its state row is read whole before its new one is written (they may be
// the same one).
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
  in[W - 1] = V::raw((const T *)a.x + (long long)m * a.ldx + d);
  float w[W][VEC], o[VEC];
  load_taps<T, VEC, W>(a, d, w, o);
#pragma unroll
  for (int v = 0; v < VEC; ++v) {
#pragma unroll
    for (int j = 0; j < W; ++j) o[v] = fmaf(w[j][v], (float)in[j].v[v], o[v]);
    if (a.silu) o[v] = silu(o[v]);
  }
  V::put((T *)a.y + (long long)m * a.ldy + d, o);
  if constexpr (W > 1) {
    T *so = (T *)a.state_out + (long long)m * (W - 1) * a.D + d;
#pragma unroll
    for (int j = 0; j + 1 < W; ++j) *(typename V::Raw *)(so + (long long)j * a.D) = in[j + 1];
  }
}

template <typename T, int VEC, int W>
hipError_t run_conv(const ConvArgs &a, bool step, hipStream_t st) {
  const long long dv = a.D / VEC;
  if (step) {
    const long long n = (a.B * dv + 255) / 256;
    hipLaunchKernelGGL((conv_step_kernel<T, VEC, W>), dim3((unsigned)n), dim3(256), 0, st, a);
  } else {
    const long long n = ((a.S + kRun - 1) / kRun * dv + 255) / 256;
    hipLaunchKernelGGL((conv_kernel<T, VEC, W>), dim3((unsigned)n, (unsigned)(a.B < 32768 ? a.B : 32768)), dim3(256),
                       0, st, a);
  }
  return hipGetLastError();
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
  const bool wide = a.D % VEC == 0 && a.ldx % VEC == 0 && a.ldy % VEC == 0 && ((uintptr_t)a.x | (uintptr_t)a.y) % 16 == 0;
  return wide ? by_width<T, VEC>(a, step, st) : by_width<T, 1>(a, step, st);
}

}  // namespace

hipError_t launch_conv(const ConvArgs &a, hipStream_t st) {
  return a.bf16_io ? by_vector<bf16>(a, false, st) : by_vector<float>(a, false, st);
}
hipError_t launch_conv_step(const ConvArgs &a, hipStream_t st) {
  return a.bf16_io ? by_vector<bf16>(a, true, st) : by_vector<float>(a, true, st);
}

}  // namespace mt
