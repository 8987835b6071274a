// Attention of few query rows, bf16.
#include "mt_mha_step.h"

namespace mt {

hipError_t launch_steps_bf16(const MhaArgs &a, const StepPlan &plan, bool share, hipStream_t st) {
  return a.table ? launch_steps_as<bf16, true>(a, plan, share, st) : launch_steps_as<bf16, false>(a, plan, share, st);
}

}  // namespace mt
