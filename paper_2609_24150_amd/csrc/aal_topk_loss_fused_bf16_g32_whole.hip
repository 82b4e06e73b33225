// Resident schedule of the objectives against top lists: bf16 logits, fp32 gradient, rows of whole vectors.
#include "aal_topk_loss_fused.h"

namespace aal {
hipError_t launch_top_fused_bf16_g32_whole(const TopLossArgs& a, bool* used) {
  return fused_coupled<Bf16, GF32, true>(a, used);
}
}  // namespace aal
