// Matrix products in 8-bit integers: rows x [M, K] quantised within the call, columns at load, each
// with one scale: y = (qx q) s_n s_m + bias.
//
// Both operands lie in fragment order: blocks of 32 rows (columns) x 32 k of 1 KiB, lane l of a wave
// holding row l % 32 and k-values 16 (l / 32) .. + 15 in 16 bytes, all k of a row block together:
// [block][Kp / 32][64 lanes][16].  This is one operand of a 32 x 32 x 32 MFMA, so a block moves to LDS
// by one direct load of a wave and from LDS to registers by one 16-byte read per lane, both without
// bank conflicts and without any arithmetic on addresses.
#include <algorithm>

#include "mt_layer_dev.h"

namespace mt {

namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));

constexpr float kTiny = 0x1p-100f;  // a row whose largest magnitude is below it is all zeros

// scale factor and scale of a row from the bits of its largest magnitude (a NaN or an infinity,
// whose bits exceed every finite value's, makes the scale NaN)
__device__ __forceinline__ void row_scales(uint32_t amax, float &r, float &s) {
  const float a = __uint_as_float(amax);
  r = a >= kTiny ? 127.0f / a : 0.0f;
  s = a >= kTiny ? a / 127.0f : 0.0f;
  if (amax >= 0x7f800000u) {
    r = 0.0f;
    s = __uint_as_float(0x7fc00000u);
  }
}
__device__ __forceinline__ int quant(float v, float r) { return (int)rintf(v * r); }
__device__ __forceinline__ int pack4(int a, int b, int c, int d) {
  return (a & 255) | (b & 255) << 8 | (c & 255) << 16 | d << 24;
}
// byte offset of (row, 16-value group kg) in fragment order with KB = Kp / 32 blocks of k
__device__ __forceinline__ size_t frag_offset(int row, int kg, int KB) {
  return ((size_t)(row >> 5) * KB + (kg >> 1)) * 1024 + (kg & 1) * 512 + (row & 31) * 16;
}

// 16 values of a row from k0 on, zero from K on
template <typename T>
__device__ __forceinline__ void load16(const T *row, int k0, int K, bool wide, float (&f)[16]) {
  if (wide && k0 + 16 <= K) {
    constexpr int E = 16 / sizeof(T);
#pragma unroll
    for (int i = 0; i < 16; i += E) {
      const typename Vec<T, E>::Raw q = Vec<T, E>::raw(row + k0 + i);
#pragma unroll
      for (int j = 0; j < E; ++j) f[i + j] = (float)q.v[j];
    }
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i) f[i] = k0 + i < K ? (float)row[k0 + i] : 0.f;
  }
}

// One wave per row: its largest magnitude, then its values in 8 bits.  Groups of k past K and rows past
// M of the last blocks are left as they are: they meet zero columns or rows that are not stored.
template <typename T>
__global__ void __launch_bounds__(256) quant_rows_kernel(I8Problem p, int wide) {
  const int lane = threadIdx.x & 63, m = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (m >= p.M) return;
  const T *row = (const T *)p.x + (long long)m * p.ldx;
  const int ng = (p.K + 15) / 16, KB = p.Kp / 32;
  uint32_t mx = 0;
  for (int g = lane; g < ng; g += 64) {
    float f[16];
    load16<T>(row, g * 16, p.K, wide, f);
#pragma unroll
    for (int i = 0; i < 16; ++i) mx = max(mx, __float_as_uint(f[i]) & 0x7fffffffu);
  }
  mx = wave_ext<uint32_t, true>(mx);
  float r, s;
  row_scales(mx, r, s);
  if (lane == 0) p.xs[m] = s;
  for (int g = lane; g < ng; g += 64) {
    float f[16];
    load16<T>(row, g * 16, p.K, wide, f);
    i32x4 q;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      q[i] = pack4(quant(f[4 * i], r), quant(f[4 * i + 1], r), quant(f[4 * i + 2], r), quant(f[4 * i + 3], r));
    *(i32x4 *)(p.xq + frag_offset(m, g, KB)) = q;
  }
}

// ---- packing of the columns at load ----
__global__ void __launch_bounds__(256) col_max_kernel(const float *W, int K, int N, int Np, uint32_t *amax) {
  const int n = blockIdx.x * 256 + threadIdx.x;
  uint32_t mx = 0;
  if (n < N)
    for (int k = 0; k < K; ++k) mx = max(mx, __float_as_uint(W[(size_t)k * N + n]) & 0x7fffffffu);
  amax[n] = mx;
}
__global__ void __launch_bounds__(256) pack_cols_kernel(const float *W, int K, int N, int KB, const uint32_t *amax,
                                                        int8_t *wq) {
  const int n = blockIdx.x * 256 + threadIdx.x;
  float r, sc;
  row_scales(amax[n], r, sc);
  for (int g = blockIdx.y; g < KB * 2; g += gridDim.y) {
    i32x4 q;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      int v[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int k = g * 16 + i * 4 + j;
        v[j] = n < N && k < K ? quant(W[(size_t)k * N + n], r) : 0;
      }
      q[i] = pack4(v[0], v[1], v[2], v[3]);
    }
    *(i32x4 *)(wq + frag_offset(n, g, KB)) = q;
  }
}
// the scales, over the magnitudes they come from
__global__ void __launch_bounds__(256) col_scale_kernel(float *s, int *bad) {
  const int n = blockIdx.x * 256 + threadIdx.x;
  const uint32_t mx = __float_as_uint(s[n]);
  float r, sc;
  row_scales(mx, r, sc);
  s[n] = sc;
  if (mx >= 0x7f800000u) *bad = 1;
}

// ---- tiles ----

constexpr int waitcnt(int vm, int lgkm) { return (vm & 15) | (vm >> 4) << 14 | 7 << 4 | lgkm << 8; }

// A workgroup of WM x WN waves computes a tile of 32 MF WM rows by 32 NF WN columns, k in stages of 64
// through a ring of ST stages in LDS that direct loads fill ST - 1 stages ahead.
template <int MF, int NF, int WM, int WN, int ST, bool BF>
__global__ void __launch_bounds__(64 * WM * WN) i8_tile_kernel(I8Problem p, int tilesM, int tilesN) {
  constexpr int AB = MF * WM, BB = NF * WN;       // blocks of 32 rows and columns
  constexpr int STAGE = (AB + BB) * 2 * 1024;     // a stage: two blocks of k of each
  constexpr int NL = (AB + BB) * 2 / (WM * WN);   // direct loads of a wave per stage
  static_assert((AB + BB) * 2 % (WM * WN) == 0, "every wave issues the same number of loads");
  __shared__ __attribute__((aligned(1024))) char lds[ST * STAGE];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wm = wave / WN, wn = wave % WN;
  const int KB = p.Kp / 32, stages = KB / 2;
  const int w = xcd_remap(blockIdx.x, gridDim.x);
  // tiles in groups of up to eight row tiles, columns slowest within a group: the tiles that run
  // together share both operands in their XCD's L2
  const int gsz = 8 * tilesN, grp = w / gsz, gm = min(8, tilesM - grp * 8);
  const int tm = grp * 8 + (w - grp * gsz) % gm, tn = (w - grp * gsz) / gm;
  const char *ga = (const char *)p.xq + (size_t)tm * AB * KB * 1024 + lane * 16;
  const char *gb = (const char *)p.wq + (size_t)tn * BB * KB * 1024 + lane * 16;
  auto load = [&](int s) {
    char *dst = lds + (s % ST) * STAGE;
    const int sk = s < stages ? s : stages - 1;  // past the end: a load that nobody reads
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int f = wave * NL + i, blk = f >> 1;  // blocks 0 .. AB-1 of rows, then of columns
      const char *src = (blk < AB ? ga + (size_t)blk * KB * 1024 : gb + (size_t)(blk - AB) * KB * 1024) +
                        (size_t)(sk * 2 + (f & 1)) * 1024;
      __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)src,
                                       (__attribute__((address_space(3))) void *)(dst + f * 1024), 16, 0, 0);
    }
  };
  i32x16 acc[MF][NF];
#pragma unroll
  for (int i = 0; i < MF; ++i)
#pragma unroll
    for (int j = 0; j < NF; ++j) acc[i][j] = (i32x16)(0);
  i32x4 fa[2][MF], fb[2][NF];
  auto read = [&](int s, int h) {  // block of k number h of stage s
    const char *src = lds + (s % ST) * STAGE + lane * 16 + h * 1024;
#pragma unroll
    for (int i = 0; i < MF; ++i) fa[h][i] = *(const i32x4 *)(src + (wm * MF + i) * 2048);
#pragma unroll
    for (int j = 0; j < NF; ++j) fb[h][j] = *(const i32x4 *)(src + (AB + wn * NF + j) * 2048);
  };
  auto mma = [&](int h) {
#pragma unroll
    for (int i = 0; i < MF; ++i)
#pragma unroll
      for (int j = 0; j < NF; ++j)
        acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fa[h][i], fb[h][j], acc[i][j], 0, 0, 0);
  };
#pragma unroll
  for (int s = 0; s < ST; ++s) load(s);
  __builtin_amdgcn_s_waitcnt(waitcnt((ST - 1) * NL, 15));
  __builtin_amdgcn_s_barrier();
  read(0, 0);
  for (int s = 0; s < stages; ++s) {
    read(s, 1);
    __builtin_amdgcn_sched_barrier(0);
    mma(0);
    // every wave holds all of stage s in registers and its part of stage s + 1 has arrived: past the
    // barrier that stage can be read and this one's buffer filled again
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt(waitcnt((ST - 2) * NL, 0));
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    load(s + ST);
    read(s + 1 < stages ? s + 1 : s, 0);
    __builtin_amdgcn_sched_barrier(0);
    mma(1);
  }
  // no direct load may still be on its way when the workgroup gives its LDS back
  __builtin_amdgcn_s_waitcnt(waitcnt(0, 0));
  // ---- lane holds rows 8 (r / 4) + 4 (lane / 32) + r % 4, column lane % 32 of each block ----
  const int m0 = (tm * AB + wm * MF) * 32 + 4 * (lane >> 5), n0 = (tn * BB + wn * NF) * 32 + (lane & 31);
  float sw[NF], bias[NF];
#pragma unroll
  for (int j = 0; j < NF; ++j) {
    sw[j] = p.ws[n0 + j * 32];
    bias[j] = p.bias && n0 + j * 32 < p.N ? p.bias[n0 + j * 32] : 0.f;
  }
#pragma unroll
  for (int i = 0; i < MF; ++i) {
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int m = m0 + i * 32 + 8 * (r >> 2) + (r & 3);
      if (m >= p.M) continue;
      const float sx = p.xs[m];
#pragma unroll
      for (int j = 0; j < NF; ++j) {
        const int n = n0 + j * 32;
        if (n >= p.N) continue;
        const float v = fmaf((float)acc[i][j][r] * sw[j], sx, bias[j]);
        if constexpr (BF)
          ((bf16 *)p.y)[(long long)m * p.ldy + n] = (bf16)v;
        else
          ((float *)p.y)[(long long)m * p.ldy + n] = v;
      }
    }
  }
}

template <int MF, int NF, int WM, int WN, int ST>
hipError_t run_tiles(const I8Problem &p, hipStream_t st) {
  const int tm = (p.M + 32 * MF * WM - 1) / (32 * MF * WM), tn = (p.N + 32 * NF * WN - 1) / (32 * NF * WN);
  if (p.y_bf16)
    hipLaunchKernelGGL((i8_tile_kernel<MF, NF, WM, WN, ST, true>), dim3((unsigned)(tm * tn)), dim3(64 * WM * WN), 0, st,
                       p, tm, tn);
  else
    hipLaunchKernelGGL((i8_tile_kernel<MF, NF, WM, WN, ST, false>), dim3((unsigned)(tm * tn)), dim3(64 * WM * WN), 0,
                       st, p, tm, tn);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_i8_product(const I8Problem &p, hipStream_t st) {
  const int ev = p.x_bf16 ? 8 : 4;
  const int wide = (uintptr_t)p.x % 16 == 0 && p.ldx % ev == 0;
  const unsigned rows = (unsigned)((p.M + 3) / 4);
  if (p.x_bf16)
    hipLaunchKernelGGL(quant_rows_kernel<bf16>, dim3(rows), dim3(256), 0, st, p, wide);
  else
    hipLaunchKernelGGL(quant_rows_kernel<float>, dim3(rows), dim3(256), 0, st, p, wide);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  return run_tiles<2, 2, 2, 2, 3>(p, st);
}

hipError_t launch_i8_pack(const float *W, int K, int N, int Kp, int Np, int8_t *wq, float *s, int *bad,
                          hipStream_t st) {
  const int nb = Np / 256, KB = Kp / 32;
  hipLaunchKernelGGL(col_max_kernel, dim3(nb), dim3(256), 0, st, W, K, N, Np, (uint32_t *)s);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(pack_cols_kernel, dim3(nb, std::min(KB * 2, 64)), dim3(256), 0, st, W, K, N, KB,
                     (const uint32_t *)s, wq);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  hipLaunchKernelGGL(col_scale_kernel, dim3(nb), dim3(256), 0, st, s, bad);
  return hipGetLastError();
}

}  // namespace mt
