// Resident schedule of the objectives against top lists: fp32 logits and gradient, rows of any length.
#include "aal_topk_loss_fused.h"

namespace aal {
hipError_t launch_top_fused_f32_ragged(const TopLossArgs& a, bool* used) {
  return fused_coupled<F32, GF32, false>(a, used);
}
}  // namespace aal
