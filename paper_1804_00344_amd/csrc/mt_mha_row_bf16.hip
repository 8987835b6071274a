// Attention of tiles of up to four query rows, bf16.
#include "mt_mha_row.h"

namespace mt {

hipError_t launch_rows_bf16(const MhaArgs &a, const StepPlan &plan, bool share, hipStream_t st) {
  return launch_rows_typed<bf16>(a, plan, share, st);
}

}  // namespace mt
