// Resident schedule of the objectives against top lists: bf16 logits, fp32 gradient, rows of any length.
#include "aal_topk_loss_fused.h"

namespace aal {
hipError_t launch_top_fused_bf16_g32_ragged(const TopLossArgs& a, bool* used) {
  return fused_coupled<Bf16, GF32, false>(a, used);
}
}  // namespace aal
