// Attention of tiles of up to four query rows, fp32.
#include "mt_mha_row.h"

namespace mt {

hipError_t launch_rows_f32(const MhaArgs &a, const StepPlan &plan, bool share, hipStream_t st) {
  return launch_rows_typed<float>(a, plan, share, st);
}

}  // namespace mt
