// Internal declarations of the recurrent layer's operators (mt_i8.hip, mt_conv.hip, mt_scan.hip).
#pragma once

#include "mt_internal.h"

namespace mt {

constexpr int kI8KPad = 128;   // k padding of both operands
constexpr int kI8Pad = 256;    // row and column padding of both operands
constexpr int kI8MaxK = 65536; // 127 * 127 * 65536 < 2^31

// ---- products in 8 bits (mt_i8.hip) ----
struct I8Problem {
  const void *x;        // [M][ldx] fp32 or bf16
  long long ldx;
  int x_bf16;
  const int8_t *wq;     // packed columns in fragment order
  const float *ws;      // [Np] column scales, zero padded
  const float *bias;    // [Np] zero padded, or NULL
  void *y;              // [M][ldy]
  long long ldy;
  int y_bf16;
  int M, N, K, Kp;
  int8_t *xq;           // workspace: rows in fragment order
  float *xs;            // and their scales
  int num_cu;
};
// tile of a product (0..4: 64 x 64, 64 x 128, 128 x 128, 128 x 256, 256 x 256); -1: the form of few rows
int i8_form(int M, int N, int K, int y_bytes, int num_cu);
hipError_t launch_i8_product(const I8Problem &p, hipStream_t st);
// quantises W [K][N] (device memory) into wq [Np/32][Kp/32][1024] and s [Np]; *bad is set to 1 where
// W holds a NaN or an infinity
hipError_t launch_i8_pack(const float *W, int K, int N, int Kp, int Np, int8_t *wq, float *s, int *bad, hipStream_t st);

// ---- causal convolution (mt_conv.hip) ----
struct ConvArgs {
  const float *w;       // [W][D]
  const float *b;       // [D]
  int D, W, silu, bf16_io;
  int B, S;             // prompts; a step: rows M and S = 1
  const int32_t *len;   // [B] or NULL
  const int32_t *row;   // step: state rows or NULL
  int n_rows;
  const void *x;
  long long ldx;
  void *y;
  long long ldy;
  const void *state_in; // [rows][W-1][D] or NULL
  void *state_out;
  int32_t *err;
  int num_cu;
};
hipError_t launch_conv(const ConvArgs &a, hipStream_t st);
hipError_t launch_conv_step(const ConvArgs &a, hipStream_t st);

// ---- selective scan (mt_scan.hip) ----
struct ScanArgs {
  const float *A2;      // [D][Np] A * log2(e), zero padded to Np = scan_padded_states(N)
  const float *dt_bias, *skip;  // [D] each (skip: zeros if there is none)
  int D, N, Np, G, bf16_io;
  int B, S;             // prompts; a step: rows M and S = 1
  const int32_t *len;
  const int32_t *row;
  int n_rows;
  const void *x, *dt, *bm, *cm, *z;
  long long ldx, lddt, ldbc, ldz, ldy;
  void *y;
  const float *state_in;
  float *state_out;
  void *ws;
  int32_t *err;
  int num_cu;
};
// The positions of a piece [.., t1) that a lane fetches: it is number tj of J lanes, takes every J-th position
// from its first one on, tile by tile and one tile ahead, and stays at its last one at the end.
__host__ __device__ inline int scan_first_row(int t0, int tj, int t1) { return t0 + tj < t1 ? t0 + tj : t1 - 1; }
// whether the tile at ts can be computed, and the one after it fetched, without looking for the end: then every
// lane goes on past that one too, to position ts + 2 tile + tj
__host__ __device__ inline bool scan_whole_tile(int ts, int tile, int J, int t1) { return ts + 2 * tile + J <= t1; }
// whether a lane goes on after slot i of the tile at ts (whole: without looking)
__host__ __device__ inline bool scan_next_row(bool whole, int ts, int i, int J, int tj, int t1) {
  return whole || ts + (i + 1) * J + tj < t1;
}
// The kernel's fetches over a piece of len positions, on the host: the last position that lane tj fetches, or -1
// if a position of its own is not the one that it holds when that is computed.
int scan_walk_rows(int len, int tile, int J, int tj);
int scan_padded_states(int N);
int scan_pieces(int B, int S, int D, int N, int num_cu);  // pieces that the axis is cut into
size_t scan_workspace_bytes(int B, int S, int D, int N, int num_cu);
hipError_t launch_scan(const ScanArgs &a, hipStream_t st);
hipError_t launch_scan_step(const ScanArgs &a, hipStream_t st);

}  // namespace mt
