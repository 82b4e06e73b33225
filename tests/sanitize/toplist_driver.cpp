// Driver and launcher stand-ins for the sanitizer build of csrc/aal_toplist_api.hip: every
// entry point with valid arguments, whose stand-ins write the whole workspace that the
// kernels would use (host buffers of exactly the advertised size), and with arguments that
// validation must reject.  Exits 0 when every check passes.
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include "aal.h"
#include "aal_toplist.h"

static int g_failures = 0, g_calls = 0;

#define CHECK(cond)                                                      \
  do {                                                                   \
    if (!(cond)) {                                                       \
      fprintf(stderr, "check failed at line %d: %s\n", __LINE__, #cond); \
      ++g_failures;                                                      \
    }                                                                    \
  } while (0)

namespace aal {

hipError_t launch_topk(const TopkArgs& a) {
  ++g_calls;
  CHECK(a.k >= 1 && a.k <= a.V && a.sc > 0.f);
  return hipSuccess;
}

hipError_t launch_top_loss(const TopLossArgs& a) {
  ++g_calls;
  memset(a.stats, 0xA5, size_t(a.R) * sizeof(TopRow));
  memset(a.row_loss, 0xA5, size_t(a.R) * sizeof(float2));
  memset(a.loss_parts, 0xA5, size_t(kTopLossParts) * 4 * sizeof(double));
  memset(a.slots, 0xA5, size_t(a.R) * 2 * sizeof(uint64_t));
  memset(a.err, 0xA5, 2 * sizeof(unsigned));
  CHECK(a.S >= 1 && a.W >= 0 && a.sc_d > 0.f && a.sc_t > 0.f);
  return hipSuccess;
}

hipError_t launch_logits(const LogitsArgs& a) {
  ++g_calls;
  CHECK(a.out != nullptr && a.z != nullptr);
  return hipSuccess;
}

}  // namespace aal

static void* const D = reinterpret_cast<void*>(uintptr_t(0x10000));  // fake device addresses
static float* const DF = reinterpret_cast<float*>(uintptr_t(0x20000));
static int32_t* const DI = reinterpret_cast<int32_t*>(uintptr_t(0x30000));
static int64_t* const DL = reinterpret_cast<int64_t*>(uintptr_t(0x40000));

static aal_status_t topk(int64_t rows, int32_t V, int32_t k, int dt = AAL_BF16, float T = 1.f) {
  return aal_topk_logits(D, aal_dtype_t(dt), rows, V, k, T, D, DI, DF, nullptr);
}

static aal_status_t loss(int lay, int64_t B, int32_t S, int32_t K, int32_t V, int32_t k, int dt = AAL_BF16, uint32_t flags = 0) {
  const size_t n = aal_topk_loss_workspace_bytes(aal_layout_t(lay), B, S, K);
  void* ws = n ? aligned_alloc(256, n) : nullptr;
  const aal_status_t s = aal_topk_loss_fwd_bwd(D, aal_dtype_t(dt), D, AAL_F32, DI, DF, aal_layout_t(lay), B, S, K, V, k, 0.5f, 2.f,
                                               aal_loss_weights_t{1.f, 0.f, 1.f, 0.f}, DF, DF, DF, DF, DF, DF, DI, D,
                                               AAL_BF16, DF, flags, ws, n, nullptr);
  free(ws);
  return s;
}

int main() {
  for (int64_t rows : {int64_t(1), int64_t(7), int64_t(1000)})
    for (int32_t k : {1, 5, 512}) CHECK(topk(rows, 1000, k) == AAL_OK);
  CHECK(topk(3, 10, 11) != AAL_OK && topk(0, 10, 1) != AAL_OK && topk(3, 0, 1) != AAL_OK && topk(3, 1000, 513) != AAL_OK);
  CHECK(topk(3, 10, 1, 17) == AAL_ERR_DTYPE);
  CHECK(topk(3, 10, 1, AAL_F32, -1.f) == AAL_ERR_ARG);
  for (int64_t B : {int64_t(1), int64_t(3), int64_t(257)})
    for (int32_t S : {1, 6, 65}) {
      CHECK(loss(AAL_LAYOUT_SEQUENCES, B, S, 6, 100, 8) == AAL_OK);
      CHECK(loss(AAL_LAYOUT_WINDOWS, B, S, 6, 100, 8, AAL_F32, AAL_FLAG_STREAMING) == AAL_OK);
    }
  CHECK(loss(9, 1, 1, 1, 10, 1) == AAL_ERR_ARG);
  CHECK(loss(AAL_LAYOUT_WINDOWS, 1, 1, 65, 10, 1) == AAL_ERR_ARG);
  CHECK(loss(AAL_LAYOUT_WINDOWS, int64_t(1) << 40, 1, 64, 10, 1) == AAL_ERR_ARG);
  CHECK(loss(AAL_LAYOUT_WINDOWS, 1, 1, 1, 10, 11) == AAL_ERR_ARG);
  CHECK(loss(AAL_LAYOUT_WINDOWS, 1, 1, 1, 10, 1, -5) == AAL_ERR_DTYPE);
  CHECK(loss(AAL_LAYOUT_WINDOWS, 1, 1, 1, 10, 1, AAL_BF16, 64) == AAL_ERR_ARG);
  aal_logits_rules_t r;
  memset(&r, 0, sizeof r);
  CHECK(aal_logits_process(D, AAL_BF16, 4, 100, &r, D, nullptr) == AAL_OK);
  CHECK(aal_logits_process(D, AAL_BF16, 4, 100, nullptr, D, nullptr) == AAL_ERR_ARG);
  CHECK(aal_logits_process(D, aal_dtype_t(3), 4, 100, &r, D, nullptr) == AAL_ERR_DTYPE);
  r.tokens = DI;
  CHECK(aal_logits_process(D, AAL_BF16, 4, 100, &r, D, nullptr) == AAL_ERR_ARG);
  r.hist_start = DL;
  r.hist_len = DI;
  r.n_tokens = 10;
  r.bias_offsets = DL;
  r.bias_ids = DI;
  r.bias_values = DF;
  r.mask = reinterpret_cast<uint32_t*>(DI);
  r.n_masks = 4;
  CHECK(aal_logits_process(D, AAL_F32, 4, 100, &r, D, nullptr) == AAL_OK);
  CHECK(aal_logits_process_bwd(D, AAL_F32, D, AAL_BF16, 4, 100, &r, D, nullptr) == AAL_OK);
  CHECK(aal_logits_process_bwd(D, AAL_F32, D, aal_dtype_t(99), 4, 100, &r, D, nullptr) == AAL_ERR_DTYPE);
  CHECK(strlen(aal_last_error()) > 0);
  r.n_masks = 3;
  CHECK(aal_logits_process(D, AAL_F32, 4, 100, &r, D, nullptr) == AAL_ERR_ARG);
  CHECK(g_calls == 9 + 18 + 3);
  if (g_failures == 0) printf("all checks passed (%d launches)\n", g_calls);
  return g_failures ? 1 : 0;
}
