// Attention of query heads over keys and values in pages of a cache, or in rows of another length under a mask:
//   y = sum_j softmax_j(scale q.k_j) v_j over the keys that a query sees.
#include "mt_mha_dev.h"

namespace mt {

namespace {

// A wave per query and head: right for every case.
template <typename T, bool PAGED>
__global__ void __launch_bounds__(256) plain_kernel(MhaArgs a) {
  __shared__ float qs[4][256];
  const int wave = threadIdx.x >> 6;
  const long long steps = (long long)a.S * a.Hq;
  const long long u = blockIdx.x * 4ll + wave;
  if (u >= steps) return;
  const int i = (int)(u / a.Hq), hq = (int)(u % a.Hq);
  for (int b = blockIdx.y; b < a.B; b += gridDim.y) {
    const RowSpan r = row_span<PAGED>(a, b, u == 0 && (threadIdx.x & 63) == 0);
    if (i < r.n) attend_one<T, PAGED>(a, r, b, i, hq, qs[wave]);
  }
}

template <typename T, bool PAGED>
hipError_t run(const MhaArgs &a, hipStream_t st) {
  const long long steps = (long long)a.S * a.Hq;
  hipLaunchKernelGGL((plain_kernel<T, PAGED>), dim3((unsigned)((steps + 3) / 4), (unsigned)(a.B < 32768 ? a.B : 32768)),
                     dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace

size_t mha_workspace_bytes(int Hq, int Hk, int Dh, int B, int S, long long n_keys, int num_cu) { return 256; }

hipError_t launch_mha(const MhaArgs &a, hipStream_t st) {
  if (a.table) return a.bf16_io ? run<bf16, true>(a, st) : run<float, true>(a, st);
  return a.bf16_io ? run<bf16, false>(a, st) : run<float, false>(a, st);
}

}  // namespace mt
