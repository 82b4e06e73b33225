// Driver and launcher stand-ins for the sanitizer build of csrc/aal_head_api.hip and
// csrc/aal_beam_api.hip: entry points with valid arguments, whose stand-ins write the whole workspace that
// they advertise, and with arguments that validation must reject.  Exits 0 when every check passes.
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include "aal.h"
#include "aal_beam.h"
#include "aal_fp8.h"

static int g_failures = 0, g_calls = 0, g_states = 0;

#define CHECK(cond)                                                      \
  do {                                                                   \
    if (!(cond)) {                                                       \
      fprintf(stderr, "check failed at line %d: %s\n", __LINE__, #cond); \
      ++g_failures;                                                      \
    }                                                                    \
  } while (0)

namespace aal {

hipError_t launch_quantize(const QuantizeArgs& a) {
  ++g_calls;
  CHECK((a.q || a.qt) && (a.block_rows == 1 || a.block_rows == 128));
  return hipSuccess;
}

size_t matmul_workspace_bytes(int64_t M, int64_t N, int64_t K) { return K > 1000 ? align256(size_t(M) * N * 8) : 0; }

hipError_t launch_matmul(const MatmulArgs& a) {
  ++g_calls;
  if (const size_t n = matmul_workspace_bytes(a.M, a.N, a.K)) memset(a.ws, 0xA5, n);
  CHECK(a.a.ld >= a.K && a.b.ld >= a.K);
  return hipSuccess;
}

size_t beam_workspace_bytes(DType, int64_t B, int W, int V, int n) { return align256(size_t(B) * W * n * 8 + size_t(V)); }

hipError_t launch_beam_select(const BeamArgs& a) {
  ++g_calls;
  memset(a.ws, 0xA5, beam_workspace_bytes(a.in, a.B, a.W, a.V, a.n));
  CHECK(a.out.parents && a.out.tokens);
  return hipSuccess;
}

hipError_t launch_beam_reorder(const ReorderArgs& a) {
  ++g_calls;
  g_states += a.n_states;
  for (int i = 0; i < a.n_states; ++i) CHECK(a.in_place ? a.states[i].dst == a.states[i].src : a.states[i].dst != a.states[i].src);
  return hipSuccess;
}

}  // namespace aal

static void* const D = reinterpret_cast<void*>(uintptr_t(0x10000));  // fake device addresses
static float* const DF = reinterpret_cast<float*>(uintptr_t(0x20000));
static int32_t* const DI = reinterpret_cast<int32_t*>(uintptr_t(0x30000));

static aal_status_t product(int64_t M, int64_t N, int64_t K, int fa = 0, int sa = 0, int sb = 0) {
  aal_fp8_operand_t a{D, D, (K + 15) / 16 * 16, 1, 1, fa, sa, 1}, b{D, D, (K + 15) / 16 * 16, 1, 1, 1, sb, 128};
  const size_t n = aal_fp8_matmul_workspace_bytes(M, N, K);
  void* ws = n ? aligned_alloc(256, n) : nullptr;
  const aal_status_t s = aal_fp8_matmul(&a, &b, M, N, K, D, AAL_BF16, ws, n, nullptr);
  free(ws);
  return s;
}

static aal_status_t select(int64_t B, int32_t W, int32_t V, int32_t n, float alpha = 0.f, int dt = AAL_BF16) {
  const size_t bytes = aal_beam_select_workspace_bytes(aal_dtype_t(dt), B, W, V, n);
  void* ws = bytes ? aligned_alloc(256, bytes) : nullptr;
  aal_beam_out_t out{DF, DF, DI, DI, nullptr, nullptr};
  const aal_status_t s = aal_beam_select(D, aal_dtype_t(dt), B, W, V, n, 1.f, DF, nullptr, nullptr, alpha, -1, 0, &out, ws,
                                         bytes, nullptr);
  free(ws);
  return s;
}

int main() {
  CHECK(aal_fp8_quantize(D, AAL_BF16, 4, 100, 100, AAL_FP8_E4M3, AAL_SCALE_F32, 1, D, 112, DF, nullptr, 0, nullptr, nullptr) == AAL_OK);
  CHECK(aal_fp8_quantize(D, AAL_F32, 4, 100, 100, AAL_FP8_E5M2, AAL_SCALE_E8M0, 128, D, 112, DF, D, 16, DF, nullptr) == AAL_OK);
  CHECK(aal_fp8_quantize(D, AAL_BF16, 4, 100, 100, aal_fp8_t(7), AAL_SCALE_F32, 1, D, 112, DF, nullptr, 0, nullptr, nullptr) == AAL_ERR_DTYPE);
  CHECK(product(4, 50, 100) == AAL_OK);
  CHECK(product(4, 50, 5000, 1) == AAL_OK);
  CHECK(product(4, 50, 100, 0, 1, 1) == AAL_OK);
  CHECK(product(4, 50, 100, 0, 1, 0) == AAL_ERR_DTYPE);
  CHECK(product(4, 50, 100, -1) == AAL_ERR_DTYPE);
  CHECK(product(0, 50, 100) == AAL_ERR_ARG);
  CHECK(product(4, 50, int64_t(1) << 40) == AAL_ERR_ARG);
  CHECK(select(2, 3, 1000, 6) == AAL_OK);
  CHECK(select(1, 64, 1 << 18, 128, 0.f, AAL_F32) == AAL_OK);
  CHECK(select(2, 3, 1000, 6, 1.f) == AAL_ERR_ARG);
  CHECK(select(2, 65, 1000, 6) == AAL_ERR_ARG);
  CHECK(select(int64_t(1) << 62, 2, 1000, 6) == AAL_ERR_ARG);
  CHECK(strlen(aal_last_error()) > 0);
  // 150 states, two thirds of them in place: launched by 64
  aal_beam_state_t* states = static_cast<aal_beam_state_t*>(calloc(150, sizeof(aal_beam_state_t)));
  for (int i = 0; i < 150; ++i) states[i] = {D, i % 3 ? nullptr : static_cast<void*>(DF), 256, 64, 0, 256, 64, 0, 1, 64};
  const int before = g_calls;
  CHECK(aal_beam_reorder(states, 150, 2, 4, 4, DI, nullptr) == AAL_OK);
  CHECK(g_states == 150 && g_calls == before + 2 + 1);
  CHECK(aal_beam_reorder(states, 150, 2, 4, 3, DI, nullptr) == AAL_ERR_ARG);
  CHECK(aal_beam_reorder(states, 0, 2, 4, 3, DI, nullptr) == AAL_OK);
  free(states);
  if (g_failures == 0) printf("all checks passed (%d launches)\n", g_calls);
  return g_failures ? 1 : 0;
}
