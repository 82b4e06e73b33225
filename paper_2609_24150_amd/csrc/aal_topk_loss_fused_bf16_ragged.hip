// Resident schedule of the objectives against top lists: bf16 logits and gradient, rows of any length.
#include "aal_topk_loss_fused.h"

namespace aal {
hipError_t launch_top_fused_bf16_ragged(const TopLossArgs& a, bool* used) {
  return fused_coupled<Bf16, GBf16, false>(a, used);
}
}  // namespace aal
