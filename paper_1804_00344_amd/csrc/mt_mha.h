// Internal declarations of the attention layer's operators (mt_mha_*.hip, mt_pages.hip).
#pragma once

#include "mt_internal.h"

namespace mt {

// device-side error bits of a layer
constexpr int kErrRow = 1, kErrLen = 2, kErrPage = 4, kErrRoom = 8;

// ---- attention (mt_mha_*.hip) ----
struct MhaArgs {
  int Hq, Hk, G, Dh, bf16_io, window;  // G query heads read one key head
  float scale;                         // of the scores, times log2(e)
  int B, S;                            // query rows b*S + i
  const int32_t *n_new;                // [B] or NULL
  const void *q;
  long long ldq;
  void *y;
  long long ldy;
  const void *k, *v;                   // paged: [n_pages, Hk, page, Dh]; else rows of stride ldk, ldv
  const int32_t *len, *table;          // paged (table != NULL)
  int n_blocks, n_pages, page_log2;
  const float *mask;                   // [B, Sk] or NULL
  long long ldk, ldv;
  int Sk;
  void *ws;
  int32_t *err;
  int num_cu;
};
// How a call is split over the chip
struct MhaPlan {
  int tiles, parts;        // of a key head's rows; of the key axis
  bool step, few, share;   // tiles of 32 rows, not of 128; of those, of four by the vector units; waves share a tile's keys
  bool sort;               // masked sentences by their work
  bool ends;               // the ends of masks looked for once and not by every workgroup
};
MhaPlan mha_plan(int Hq, int Hk, int Dh, int B, int S, long long n_keys, int window, bool f32, int num_cu);
size_t mha_workspace_bytes(int Hq, int Hk, int Dh, bool f32, int B, int S, long long n_keys, int window, int num_cu);
hipError_t launch_mha(const MhaArgs &a, hipStream_t st);

// ---- norms, rotation and store (mt_mha_append.hip) ----
struct AppendArgs {
  int Hq, Hk, Dh, bf16_io, norm, rot, rot_pairs;
  float eps, inv_Dh;
  const float *gq, *gk;      // [Dh]
  const double *turns;       // [rot/2] turns per position: frequency / (2 pi)
  int B, S;
  const int32_t *n_new, *len, *table;
  int n_blocks, n_pages, page_log2;
  const void *q, *k, *v;
  void *qo, *kp, *vp;
  long long ldq, ldk, ldv, ldqo;
  int32_t *err;
  int num_cu;
};
// positions of a workgroup, and whether results are stored past the L2s
struct AppendForm {
  int tokens;
  bool stream;
};
AppendForm append_form(int B, int S, int Hq, int Hk, int Dh, int esize, bool aligned, int num_cu);
hipError_t launch_append(const AppendArgs &a, hipStream_t st);

// ---- page tables (mt_pages.hip) ----
struct PagesArgs {
  int M_in, M;
  const int32_t *row, *add, *table_in, *len_in;
  int n_blocks, n_pages, page_log2;
  int32_t *table_out, *len_out, *free_out;  // pack: free_out counts the used pages
  int layers;
  long long head_bytes;                     // of a position: Dh elements
  int Hk;
  const void *k_in, *v_in;                  // advance: the same cache
  void *k_out, *v_out;
  int n_pages_out;
  void *ws;
  int32_t *err;
  int num_cu;
};
size_t pages_workspace_bytes(int M, int n_pages);
hipError_t launch_advance(const PagesArgs &a, hipStream_t st);
hipError_t launch_pack(const PagesArgs &a, hipStream_t st);

}  // namespace mt
