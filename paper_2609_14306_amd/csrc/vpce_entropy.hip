// The backward of a loss with an entropy term (ENT in vpce_backward.h): the launches of
// vp_ce_backward with its residual tiles in that form.
#include "vpce_backward.h"

namespace vpce {

bool run_stage_entropy(int dtype, int cls, const StageArgs& a, hipStream_t s) {
  return dtype == VP_BF16 ? launch_stage<Bf16, true>(cls, a, s) : launch_stage<F32, true>(cls, a, s);
}

}  // namespace vpce
