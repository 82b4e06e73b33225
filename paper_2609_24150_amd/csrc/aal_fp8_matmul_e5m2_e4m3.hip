// The product's kernels for a in e5m2 and b in e4m3.
#include "aal_fp8_matmul.h"

namespace aal {
template hipError_t launch_matmul_formats<1, 0>(const MatmulArgs&, const MatmulParams&, const MatmulPlan&);
}  // namespace aal
