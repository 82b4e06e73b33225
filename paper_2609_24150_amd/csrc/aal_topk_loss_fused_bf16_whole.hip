// Resident schedule of the objectives against top lists: bf16 logits and gradient, rows of whole vectors.
#include "aal_topk_loss_fused.h"

namespace aal {
hipError_t launch_top_fused_bf16_whole(const TopLossArgs& a, bool* used) {
  return fused_coupled<Bf16, GBf16, true>(a, used);
}
}  // namespace aal
