// Resident schedule of the objectives against top lists: fp32 logits and gradient, rows of whole vectors.
#include "aal_topk_loss_fused.h"

namespace aal {
hipError_t launch_top_fused_f32_whole(const TopLossArgs& a, bool* used) {
  return fused_coupled<F32, GF32, true>(a, used);
}
}  // namespace aal
