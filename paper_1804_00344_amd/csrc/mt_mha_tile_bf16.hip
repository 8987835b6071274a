// Attention by tiles of query rows, bf16.
#include "mt_mha_tile.h"

namespace mt {

hipError_t launch_tiles_bf16(const MhaArgs &a, const TilePlan &plan, hipStream_t st) {
  return a.table ? launch_tiles_as<bf16, true>(a, plan, st) : launch_tiles_as<bf16, false>(a, plan, st);
}

}  // namespace mt
