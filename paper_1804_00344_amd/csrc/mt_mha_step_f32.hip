// Attention of few query rows, fp32.
#include "mt_mha_step.h"

namespace mt {

hipError_t launch_steps_f32(const MhaArgs &a, const StepPlan &plan, bool share, hipStream_t st) {
  return a.table ? launch_steps_as<float, true>(a, plan, share, st) : launch_steps_as<float, false>(a, plan, share, st);
}

}  // namespace mt
