// Attention by tiles of query rows, fp32.
#include "mt_mha_tile.h"

namespace mt {

hipError_t launch_tiles_f32(const MhaArgs &a, const TilePlan &plan, hipStream_t st) {
  return a.table ? launch_tiles_as<float, true>(a, plan, st) : launch_tiles_as<float, false>(a, plan, st);
}

}  // namespace mt
