// Matrix products in 8-bit integers: rows x [M, K] quantised within the call, columns at load, each
// with one scale: y = (qx q) s_n s_m + bias.
//
// Both operands lie in fragment order: blocks of 32 rows (columns) x 32 k of 1 KiB, lane l of a wave
// holding row l % 32 and k-values 16 (l / 32) .. + 15 in 16 bytes, all k of a row block together:
// [block][Kp / 32][64 lanes][16].  This is one operand of a 32 x 32 x 32 MFMA, so a block moves to LDS
// by one direct load of a wave and from LDS to registers by one 16-byte read per lane, both without
// bank conflicts and without any arithmetic on addresses.
#include <algorithm>
#include <cmath>

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

// 8 values of a row from k0 on, zero from K on
template <typename T>
struct Row8 {  // whole vectors at any alignment: element by element 4 x 3711 x 3000 fp32 took 16 us, so 11
  static constexpr int E = 16 / sizeof(T);
  typename Vec<T, E>::Raw v[8 / E];
  __device__ __forceinline__ void load(const T *row, int k0, int K) {
    if (k0 + 8 <= K) {
#pragma unroll
      for (int i = 0; i < 8 / E; ++i) v[i] = Vec<T, E>::raw_any(row + k0 + i * E);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i / E].v[i % E] = k0 + i < K ? row[k0 + i] : (T)0.f;
    }
  }
  __device__ __forceinline__ float at(int i) const { return (float)v[i / E].v[i % E]; }
  __device__ __forceinline__ uint32_t magnitude() const {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(at(i)) & 0x7fffffffu);
    return m;
  }
  __device__ __forceinline__ int2 packed(float r) const {
    return make_int2(pack4(quant(at(0), r), quant(at(1), r), quant(at(2), r), quant(at(3), r)),
                     pack4(quant(at(4), r), quant(at(5), r), quant(at(6), r), quant(at(7), r)));
  }
  // the eight 8-bit values at their place of row m
  __device__ __forceinline__ void store(int8_t *xq, int m, int k0, int KB, float r) const {
    *(int2 *)(xq + frag_offset(m, k0 >> 4, KB) + (k0 & 8)) = packed(r);
  }
};

// One wave per row, eight neighbouring values per lane and pass: the row's largest magnitude, then its
// values in 8 bits.  A row of up to 512 R values is read once and waits in registers (longer ones, R = 0,
// are read twice).  Bound by traffic: 8192 x 4096 bf16 22 us (4.6 TB/s).  Values of k past K and rows past M
// of the last blocks are left as they are: they meet zero columns or rows that are not stored.
template <typename T, int R>
__global__ void __launch_bounds__(256) quant_rows_kernel(I8Problem p) {
  const int lane = threadIdx.x & 63, m = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (m >= p.M) return;
  const T *row = (const T *)p.x + (long long)m * p.ldx;
  const int KB = p.Kp / 32;
  uint32_t mx = 0;
  float r, s;
  if constexpr (R > 0) {
    Row8<T> q[R];
#pragma unroll
    for (int i = 0; i < R; ++i) q[i].load(row, (i * 64 + lane) * 8, p.K);
#pragma unroll
    for (int i = 0; i < R; ++i) mx = max(mx, q[i].magnitude());
    row_scales(wave_ext<uint32_t, true>(mx), r, s);
#pragma unroll
    for (int i = 0; i < R; ++i)
      if ((i * 64 + lane) * 8 < p.K) q[i].store(p.xq, m, (i * 64 + lane) * 8, KB, r);
  } else {
    Row8<T> q;
    for (int k = lane * 8; k < p.K; k += 512) {
      q.load(row, k, p.K);
      mx = max(mx, q.magnitude());
    }
    row_scales(wave_ext<uint32_t, true>(mx), r, s);
    for (int k = lane * 8; k < p.K; k += 512) {
      q.load(row, k, p.K);
      q.store(p.xq, m, k, KB, r);
    }
  }
  if (lane == 0) p.xs[m] = s;
}

template <typename T>
hipError_t run_quant(const I8Problem &p, hipStream_t st) {
  const dim3 grid((unsigned)((p.M + 3) / 4)), block(256);
  if (p.K <= 512)
    hipLaunchKernelGGL((quant_rows_kernel<T, 1>), grid, block, 0, st, p);
  else if (p.K <= 1024)
    hipLaunchKernelGGL((quant_rows_kernel<T, 2>), grid, block, 0, st, p);
  else if (p.K <= 2048)
    hipLaunchKernelGGL((quant_rows_kernel<T, 4>), grid, block, 0, st, p);
  else if (p.K <= 4096)
    hipLaunchKernelGGL((quant_rows_kernel<T, 8>), grid, block, 0, st, p);
  else
    hipLaunchKernelGGL((quant_rows_kernel<T, 0>), grid, block, 0, st, p);
  return hipGetLastError();
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
// through a ring of ST stages in LDS that direct loads fill ST - 1 stages ahead.  8192 x 4096 x 8192 bf16 takes
// 250 us (2.2 P operations/s) and is bound by power: with the MFMAs busy in 59% of the cycles the clock
// falls from 2.4 to 1.8 GHz.  768 x 512 x 50000 fp32: 42 to 47 us, bound by the 154 MB of its results.
template <int MF, int NF, int WM, int WN, int ST, bool BF, bool STREAM>
__global__ void __launch_bounds__(64 * WM * WN) i8_tile_kernel(I8Problem p, int tilesM, int tilesN) {
  constexpr int AB = MF * WM, BB = NF * WN;       // blocks of 32 rows and columns
  constexpr int STAGE = (AB + BB) * 2 * 1024;     // a stage: two blocks of k of each
  constexpr int NL = (AB + BB) * 2 / (WM * WN);   // direct loads of a wave per stage
  static_assert((AB + BB) * 2 % (WM * WN) == 0, "every wave issues the same number of loads");
  __shared__ __attribute__((aligned(1024))) char lds[ST * STAGE + 2 * BB * 32 * 4];
  float *const cols = (float *)(lds + ST * STAGE);  // scales and biases of the tile's columns
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wm = wave / WN, wn = wave % WN;
  const int KB = p.Kp / 32, stages = KB / 2;
  const int w = xcd_remap(blockIdx.x, gridDim.x);
  // tiles in groups of up to eight row tiles, columns slowest within a group: the tiles that run
  // together share both operands in their XCD's L2
  const int gsz = 8 * tilesN, grp = w / gsz, gm = min(8, tilesM - grp * 8);
  const int tm = grp * 8 + (w - grp * gsz) % gm, tn = (w - grp * gsz) / gm;
  const char *ga = (const char *)p.xq + (size_t)tm * AB * KB * 1024 + lane * 16;
  const char *gb = (const char *)p.wq + (size_t)tn * BB * KB * 1024 + lane * 16;
  auto load = [&](int s, int i) {  // the i-th direct load of this wave for stage s
    char *dst = lds + (s % ST) * STAGE;
    const int sk = s < stages ? s : stages - 1;  // past the end: a load that nobody reads
    const int f = wave * NL + i, blk = f >> 1;   // blocks 0 .. AB-1 of rows, then of columns
    const char *src = (blk < AB ? ga + (size_t)blk * KB * 1024 : gb + (size_t)(blk - AB) * KB * 1024) +
                      (size_t)(sk * 2 + (f & 1)) * 1024;
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)src,
                                     (__attribute__((address_space(3))) void *)(dst + f * 1024), 16, 0, 0);
  };
  // a column's scale and bias per thread, on their way while the products run (read by each wave after them
  // 768 x 512 x 50000 took 50 us, so 47; as an LDS array of its own it makes the compiler wait for the
  // direct loads in every stage)
  static_assert(BB * 32 <= 64 * WM * WN, "a thread per column");
  const bool has_col = threadIdx.x < BB * 32;
  const float col_scale = has_col ? p.ws[tn * BB * 32 + threadIdx.x] : 0.f;
  const float col_bias = has_col && p.bias ? p.bias[tn * BB * 32 + threadIdx.x] : 0.f;
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
  // the MFMAs of block h of k, the wave's loads i0 .. i1-1 for stage s spread among them: right after the
  // barrier all waves' loads would queue before their first MFMA
  auto mma = [&](int h, int s, int i0, int i1) {
    constexpr int every = MF * NF / ((NL + 1) / 2) > 0 ? MF * NF / ((NL + 1) / 2) : 1;
#pragma unroll
    for (int q = 0; q < MF * NF; ++q) {
      const int i = q / NF, j = q % NF;
      acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fb[h][j], fa[h][i], acc[i][j], 0, 0, 0);
      if (q % every == 0 && i0 + q / every < i1) {
        __builtin_amdgcn_sched_barrier(0);
        load(s, i0 + q / every);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  };
#pragma unroll
  for (int s = 0; s < ST; ++s)
#pragma unroll
    for (int i = 0; i < (s + 1 < ST ? NL : NL / 2); ++i) load(s, i);
  __builtin_amdgcn_s_waitcnt(waitcnt((ST - 2) * NL + NL / 2, 15));
  __builtin_amdgcn_s_barrier();
  read(0, 0);
  for (int s = 0; s < stages; ++s) {
    // the first block's reads were issued a block of MFMAs ago; waited for here, the ones that follow
    // are not waited for with them
    __builtin_amdgcn_s_waitcnt(waitcnt(63, 0));
    read(s, 1);
    __builtin_amdgcn_sched_barrier(0);
    mma(0, s + ST - 1, NL / 2, NL);
    // every wave holds all of stage s in registers and its part of stage s + 1 has arrived: past the
    // barrier that stage can be read and this one's buffer filled again
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt(waitcnt((ST - 2) * NL, 0));
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    read(s + 1 < stages ? s + 1 : s, 0);
    __builtin_amdgcn_sched_barrier(0);
    mma(1, s + ST, 0, NL / 2);
  }
  if (has_col) {
    cols[threadIdx.x] = col_scale;
    cols[BB * 32 + threadIdx.x] = col_bias;
  }
  // no direct load may still be on its way when the ring is used for the results (or given back)
  __builtin_amdgcn_s_waitcnt(waitcnt(0, 0));
  __builtin_amdgcn_s_barrier();
  // ---- the columns are the MFMAs' first operand, so a lane holds row lane % 32 and columns 8 (r / 4) +
  // 4 (lane / 32) + r % 4 of each block: four neighbours at a time.  They pass through the wave's part
  // of LDS (32 rows at a time, 16-byte chunks of a row permuted by its number against bank conflicts) to
  // be stored as whole vectors of consecutive columns.
  typedef typename std::conditional<BF, bf16, float>::type Y;
  constexpr int ES = sizeof(Y), ROWB = NF * 32 * ES, CPR = ROWB / 16, EPC = 16 / ES;  // chunks of a row, elements
  static_assert(WM * WN * 32 * ROWB <= ST * STAGE, "the results of 32 rows of every wave fit into the ring");
  char *own = lds + wave * 32 * ROWB;
  const int n0 = (tn * BB + wn * NF) * 32, lr = lane & 31;
#pragma unroll
  for (int i = 0; i < MF; ++i) {
    const int mb = (tm * AB + wm * MF + i) * 32;
    const float sx = p.xs[min(mb + lr, p.M - 1)];
#pragma unroll
    for (int j = 0; j < NF; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int nq = j * 32 + 8 * q + 4 * (lane >> 5);
        const float4 sw = *(const float4 *)(cols + wn * NF * 32 + nq);
        const float4 bias = *(const float4 *)(cols + (BB + wn * NF) * 32 + nq);
        float v[4];
        v[0] = fmaf((float)acc[i][j][4 * q] * sw.x, sx, bias.x);
        v[1] = fmaf((float)acc[i][j][4 * q + 1] * sw.y, sx, bias.y);
        v[2] = fmaf((float)acc[i][j][4 * q + 2] * sw.z, sx, bias.z);
        v[3] = fmaf((float)acc[i][j][4 * q + 3] * sw.w, sx, bias.w);
        const int byte = nq * ES;
        Vec<Y, 4>::put((Y *)(own + lr * ROWB + (((byte >> 4) ^ (lr % CPR)) << 4) + (byte & 15)), v);
      }
    __builtin_amdgcn_s_waitcnt(waitcnt(63, 0));  // the wave's own part: no barrier
    __builtin_amdgcn_wave_barrier();
    Y *const yb = (Y *)p.y + (long long)mb * p.ldy + n0;
#pragma unroll
    for (int u = 0; u < 32 * CPR / 64; ++u) {
      const int c = lane + u * 64;
      const int r = c / CPR, k = c % CPR, n = n0 + k * EPC;
      const typename Vec<Y, EPC>::Raw v = *(const typename Vec<Y, EPC>::Raw *)(own + r * ROWB + ((k ^ (r % CPR)) << 4));
      if (mb + r >= p.M) continue;
      Y *dst = yb + (long long)r * p.ldy + k * EPC;
      if (n + EPC <= p.N) {
        if constexpr (STREAM)
          Vec<Y, EPC>::template store<true>(dst, v);
        else
          Vec<Y, EPC>::store_any(dst, v);
      } else {
        for (int e = 0; e < EPC; ++e)
          if (n + e < p.N) dst[e] = v.v[e];
      }
    }
    __builtin_amdgcn_s_waitcnt(waitcnt(63, 0));
    __builtin_amdgcn_wave_barrier();
  }
}

template <int MF, int NF, int WM, int WN, int ST>
hipError_t run_tiles(const I8Problem &p, hipStream_t st) {
  const int tm = (p.M + 32 * MF * WM - 1) / (32 * MF * WM), tn = (p.N + 32 * NF * WN - 1) / (32 * NF * WN);
  const dim3 grid((unsigned)(tm * tn)), block(64 * WM * WN);
  // aligned results larger than the L2s together are stored past them: 768 x 512 x 50000 fp32 71 -> 53 us
  const bool aligned = (uintptr_t)p.y % 16 == 0 && p.ldy % (p.y_bf16 ? 8 : 4) == 0;
  const bool stream = aligned && (double)p.M * p.N * (p.y_bf16 ? 2 : 4) > 32e6;
#define MT_TILES(BF, S) hipLaunchKernelGGL((i8_tile_kernel<MF, NF, WM, WN, ST, BF, S>), grid, block, 0, st, p, tm, tn)
  if (p.y_bf16 && stream)
    MT_TILES(true, true);
  else if (p.y_bf16)
    MT_TILES(true, false);
  else if (stream)
    MT_TILES(false, true);
  else
    MT_TILES(false, false);
#undef MT_TILES
  return hipGetLastError();
}

// ---- one to four rows ----

// A pass over the weights in one launch: a wave takes 32 columns and one of KW parts of k, eight blocks of k
// on their way at a time, straight into registers.  Every workgroup quantises the rows itself, one per wave,
// into LDS ([16 values of k][row][16 bytes]); the row's loads are issued before the weights', so that they
// return first.  The parts are summed in LDS, in whole numbers.  Bound by the weights' traffic and
// the latency of a launch (1 x 512 x 50000 fp32: see the rule below).
template <typename T, int R>
__global__ void __launch_bounds__(256) i8_few_kernel(I8Problem p, int KW) {
  constexpr int U = 8;
  extern __shared__ __attribute__((aligned(16))) char lds[];
  __shared__ float xs[4];
  __shared__ int red[3][16][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, KB = p.Kp / 32, M = p.M;
  const int part = wave % KW, blk = blockIdx.x * (4 / KW) + wave / KW;
  const int nblk = (p.N + 31) / 32;
  const int per = (KB + KW - 1) / KW, k0 = min(part * per, KB), k1 = min(k0 + per, KB);
  Row8<T> q[R];
  if (wave < M) {
#pragma unroll
    for (int i = 0; i < R; ++i) q[i].load((const T *)p.x + wave * p.ldx, (i * 64 + lane) * 8, p.K);
  }
  const char *wp = (const char *)p.wq + (size_t)min(blk, nblk - 1) * KB * 1024 + lane * 16;
  i32x4 fb[U];
#pragma unroll
  for (int u = 0; u < U; ++u) fb[u] = *(const i32x4 *)(wp + (size_t)min(k0 + u, KB - 1) * 1024);
  if (wave < M) {
    uint32_t mx = 0;
    float r, s;
#pragma unroll
    for (int i = 0; i < R; ++i) mx = max(mx, q[i].magnitude());
    row_scales(wave_ext<uint32_t, true>(mx), r, s);
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int k = (i * 64 + lane) * 8;
      if (k < p.Kp) *(int2 *)(lds + ((k >> 4) * M + wave) * 16 + (k & 8)) = q[i].packed(r);
    }
    if (lane == 0) xs[wave] = s;
  }
  __syncthreads();
  // lanes of rows past the last read row 0: their results are not stored
  const char *xp = lds + ((lane >> 5) * M + ((lane & 31) < M ? lane & 31 : 0)) * 16;
  i32x16 acc = (i32x16)(0);
  for (int k = k0; k < k1; k += U) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (k + u >= k1) break;
      const i32x4 fa = *(const i32x4 *)(xp + (k + u) * 2 * M * 16), b = fb[u];
      fb[u] = *(const i32x4 *)(wp + (size_t)min(k + u + U, KB - 1) * 1024);
      acc = __builtin_amdgcn_mfma_i32_32x32x32_i8(b, fa, acc, 0, 0, 0);
    }
  }
  if (KW > 1) {
    if (part > 0) {
#pragma unroll
      for (int r = 0; r < 16; ++r) red[wave - 1][r][lane] = acc[r];
    }
    __syncthreads();
    if (part > 0) return;
    for (int w = 1; w < KW; ++w)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[r] += red[wave + w - 1][r][lane];
  }
  // lane holds row lane % 32, columns 8 (r / 4) + 4 (lane / 32) + r % 4
  const int m = lane & 31;
  if (blk >= nblk || m >= M) return;
  const float sx = xs[m];
#pragma unroll
  for (int c = 0; c < 4; ++c)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int n = blk * 32 + 8 * c + 4 * (lane >> 5) + e;
      if (n >= p.N) continue;
      const float v = fmaf((float)acc[4 * c + e] * p.ws[n], sx, p.bias ? p.bias[n] : 0.f);
      if (p.y_bf16)
        ((bf16 *)p.y)[(long long)m * p.ldy + n] = (bf16)v;
      else
        ((float *)p.y)[(long long)m * p.ldy + n] = v;
    }
}

constexpr int kFewRows = 4, kFewK = 4096;

template <typename T>
hipError_t run_few(const I8Problem &p, hipStream_t st) {
  const int nblk = (p.N + 31) / 32, KB = p.Kp / 32;
  int KW = 1;  // parts of k: until there are eight waves per unit, of at least two blocks
  while (KW < 4 && (long long)nblk * KW < 8ll * p.num_cu && KB / (KW * 2) >= 2) KW *= 2;
  const dim3 grid((unsigned)((nblk + 4 / KW - 1) / (4 / KW))), block(256);
  const size_t lds = (size_t)p.M * p.Kp;
#define MT_FEW(R) hipLaunchKernelGGL((i8_few_kernel<T, R>), grid, block, lds, st, p, KW)
  if (p.Kp <= 512)
    MT_FEW(1);
  else if (p.Kp <= 1024)
    MT_FEW(2);
  else if (p.Kp <= 2048)
    MT_FEW(4);
  else
    MT_FEW(8);
#undef MT_FEW
  return hipGetLastError();
}

// The tile by the time it is expected to take (us): a fixed part, per 64 k the longer of one tile's
// latency and its units' share of the tiles' throughput, and the results at 5.2 TB/s with a factor for how
// little their stores overlap with other tiles.  Fitted to rows 96 to 8192, K 512 to 4096, columns 512 to
// 50000 (bf16; the largest misprediction of the best tile costs 10%).
struct TileCost {
  int rows, cols;
  double fixed, latency, share, out;
};
constexpr TileCost kTiles[] = {{64, 64, 6.4, 0.170, 0.113, 1.5},
                               {64, 128, 7.1, 0.190, 0.180, 1.5},
                               {128, 128, 8.6, 0.275, 0.273, 1.1},
                               {128, 256, 9.5, 0.367, 0.510, 1.0},
                               {256, 256, 12.6, 0.580, 0.957, 1.35}};

int i8_tile(int M, int N, int Kp, int es, int num_cu) {
  int best = 0;
  double best_us = 1e30;
  for (int i = 0; i < 5; ++i) {
    const TileCost &t = kTiles[i];
    const double tiles = std::ceil((double)M / t.rows) * std::ceil((double)N / t.cols);
    const double us = t.fixed + Kp / 64 * std::max(t.latency, std::ceil(tiles / num_cu) * t.share) +
                      t.out * M * (double)N * es / 5.2e6;
    if (us < best_us) {
      best_us = us;
      best = i;
    }
  }
  return best;
}

}  // namespace

int i8_form(int M, int N, int K, int y_bytes, int num_cu) {
  const int Kp = (K + kI8KPad - 1) / kI8KPad * kI8KPad;
  // Few rows: one launch instead of two.  bf16, one and four rows x 512 x 2048: 6.4 and 6.9 us (tiles 6.8 and
  // 7.2), x 2048 x 8192: 9.5 and 10.0 (11.4 and 11.5), 512 x 50000: 8.7 and 9.2 (9.7 and 9.4); sixteen rows are
  // slower than tiles.
  return M <= kFewRows && Kp <= kFewK ? -1 : i8_tile(M, N, Kp, y_bytes, num_cu);
}

hipError_t launch_i8_product(const I8Problem &p, hipStream_t st) {
  const int form = i8_form(p.M, p.N, p.K, p.y_bf16 ? 2 : 4, p.num_cu);
  if (form < 0) return p.x_bf16 ? run_few<bf16>(p, st) : run_few<float>(p, st);
  const hipError_t e = p.x_bf16 ? run_quant<bf16>(p, st) : run_quant<float>(p, st);
  if (e != hipSuccess) return e;
  switch (form) {
    case 0: return run_tiles<1, 1, 2, 2, 4>(p, st);
    case 1: return run_tiles<1, 2, 2, 2, 4>(p, st);
    case 2: return run_tiles<2, 2, 2, 2, 3>(p, st);
    case 3: return run_tiles<2, 2, 2, 4, 3>(p, st);
    default: return run_tiles<4, 2, 2, 4, 4>(p, st);
  }
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
