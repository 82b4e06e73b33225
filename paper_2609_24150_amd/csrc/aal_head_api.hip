// C ABI of the 8-bit head: argument validation and dispatch.  Declarations and the contract
// of every entry point are in include/aal.h.
#include "aal_api_common.h"
#include "aal_fp8.h"

namespace {

constexpr int64_t kMostSize = int64_t(1) << 31;   // sizes are below it
constexpr int64_t kMostRows = int64_t(1) << 28;   // of an operand
constexpr int64_t kMostInner = int64_t(1) << 24;  // 256 rows' bytes are below 2^32

bool size_in_range(int64_t n) { return n >= 1 && n < kMostSize; }
bool product_sizes(int64_t M, int64_t N, int64_t K) {
  return M >= 1 && M <= kMostRows && N >= 1 && N <= kMostRows && M * N < (int64_t(1) << 37) && K >= 1 && K < kMostInner;
}
bool valid_format(int f) { return f == AAL_FP8_E4M3 || f == AAL_FP8_E5M2; }
bool valid_scale(int s) { return s == AAL_SCALE_F32 || s == AAL_SCALE_E8M0; }

aal_status_t launched(hipError_t e) {
  return e == hipSuccess ? AAL_OK : fail(AAL_ERR_HIP, "kernel launch failed: %s", hipGetErrorString(e));
}

aal_status_t check_operand(const aal_fp8_operand_t* o, const char* name, int64_t K) {
  if (!o) return fail(AAL_ERR_ARG, "%s must be non-NULL", name);
  if (!o->values || !o->scale) return fail(AAL_ERR_ARG, "%s: values and scale must be non-NULL", name);
  if (!valid_format(o->format)) return fail(AAL_ERR_DTYPE, "%s: unknown format %d", name, o->format);
  if (!valid_scale(o->scale_type)) return fail(AAL_ERR_DTYPE, "%s: unknown scale_type %d", name, o->scale_type);
  if (o->block_rows != 1 && o->block_rows != 128)
    return fail(AAL_ERR_ARG, "%s: block_rows must be 1 or 128 (got %d)", name, o->block_rows);
  if (o->ld < K || o->ld >= kMostInner) return fail(AAL_ERR_ARG, "%s: ld must be at least K and below 2^24", name);
  if (o->ld % 16 != 0 || !aligned(o->values, 16))
    return fail(AAL_ERR_ALIGN, "%s: values must be 16-byte aligned, ld a multiple of 16", name);
  if (o->scale_type == AAL_SCALE_F32 && !aligned(o->scale, 4)) return fail(AAL_ERR_ALIGN, "%s: scale must be 4-byte aligned", name);
  return AAL_OK;
}

aal::Operand operand_of(const aal_fp8_operand_t& o) {
  return {static_cast<const uint8_t*>(o.values), o.scale, o.ld, o.scale_row, o.scale_block, o.format, o.block_rows};
}

}  // namespace

extern "C" {

aal_status_t aal_fp8_quantize(const void* x, aal_dtype_t in_dtype, int64_t rows, int64_t cols, int64_t ld_x,
                              aal_fp8_t format, aal_scale_t scale_type, int32_t block_rows, void* q, int64_t ld_q,
                              void* scale, void* qt, int64_t ld_qt, void* scale_t, hipStream_t stream) {
  clear_error();
  if (!x) return fail(AAL_ERR_ARG, "x must be non-NULL");
  if (!q && !qt) return fail(AAL_ERR_ARG, "q or qt must be non-NULL");
  if ((q == nullptr) != (scale == nullptr) || (qt == nullptr) != (scale_t == nullptr))
    return fail(AAL_ERR_ARG, "q and scale, qt and scale_t go together");
  if (!size_in_range(rows) || cols < 1 || cols > (int64_t(1) << 30))
    return fail(AAL_ERR_ARG, "rows must be in [1, 2^31), cols in [1, 2^30]");
  if (ld_x < cols || ld_x >= (int64_t(1) << 40)) return fail(AAL_ERR_ARG, "ld_x must be at least cols and below 2^40");
  if (block_rows != 1 && block_rows != 128) return fail(AAL_ERR_ARG, "block_rows must be 1 or 128 (got %d)", block_rows);
  if ((q && (ld_q < cols || ld_q >= 2 * kMostSize)) || (qt && (ld_qt < rows || ld_qt >= 2 * kMostSize)))
    return fail(AAL_ERR_ARG, "ld_q must be at least cols, ld_qt at least rows, both below 2^32");
  if (!valid_dtype(raw(in_dtype))) return fail(AAL_ERR_DTYPE, "unknown in_dtype %d", raw(in_dtype));
  if (!valid_format(raw(format))) return fail(AAL_ERR_DTYPE, "unknown format %d", raw(format));
  if (!valid_scale(raw(scale_type))) return fail(AAL_ERR_DTYPE, "unknown scale_type %d", raw(scale_type));
  if (!aligned(x, raw(in_dtype) == AAL_BF16 ? 2 : 4)) return fail(AAL_ERR_ALIGN, "x must be aligned to its elements");
  if ((q && (!aligned(q, 16) || ld_q % 16 != 0)) || (qt && (!aligned(qt, 16) || ld_qt % 16 != 0)))
    return fail(AAL_ERR_ALIGN, "q and qt must be 16-byte aligned, ld_q and ld_qt multiples of 16");
  if (raw(scale_type) == AAL_SCALE_F32 && ((scale && !aligned(scale, 4)) || (scale_t && !aligned(scale_t, 4))))
    return fail(AAL_ERR_ALIGN, "scales must be 4-byte aligned");
  aal::QuantizeArgs a{};
  a.in = to_dtype(raw(in_dtype));
  a.x = x;
  a.rows = rows;
  a.cols = cols;
  a.ld = ld_x;
  a.format = static_cast<aal::Fp8>(raw(format));
  a.st = static_cast<aal::Scale>(raw(scale_type));
  a.block_rows = block_rows;
  a.q = static_cast<uint8_t*>(q);
  a.ld_q = ld_q;
  a.scale = scale;
  a.qt = static_cast<uint8_t*>(qt);
  a.ld_qt = ld_qt;
  a.scale_t = scale_t;
  a.stream = stream;
  return launched(aal::launch_quantize(a));
}

size_t aal_fp8_matmul_workspace_bytes(int64_t M, int64_t N, int64_t K) {
  return product_sizes(M, N, K) ? aal::matmul_workspace_bytes(M, N, K) : 0;
}

aal_status_t aal_fp8_matmul(const aal_fp8_operand_t* a, const aal_fp8_operand_t* b, int64_t M, int64_t N, int64_t K,
                            void* c, aal_dtype_t c_dtype, void* workspace, size_t workspace_bytes,
                            hipStream_t stream) {
  clear_error();
  if (!c) return fail(AAL_ERR_ARG, "c must be non-NULL");
  if (!product_sizes(M, N, K))
    return fail(AAL_ERR_ARG, "M and N must be in [1, 2^28], M * N below 2^37, K in [1, 2^24)");
  if (aal_status_t s = check_operand(a, "a", K); s != AAL_OK) return s;
  if (aal_status_t s = check_operand(b, "b", K); s != AAL_OK) return s;
  if (a->scale_type != b->scale_type) return fail(AAL_ERR_DTYPE, "the scales of a and b must be of one type");
  if (!valid_dtype(raw(c_dtype))) return fail(AAL_ERR_DTYPE, "unknown c_dtype %d", raw(c_dtype));
  if (!aligned(c, 16)) return fail(AAL_ERR_ALIGN, "c must be 16-byte aligned");
  if (const size_t need = aal::matmul_workspace_bytes(M, N, K)) {
    if (!workspace) return fail(AAL_ERR_WORKSPACE, "workspace must be non-NULL");
    if (!aligned(workspace, 256)) return fail(AAL_ERR_ALIGN, "workspace must be 256-byte aligned");
    if (workspace_bytes < need) return fail(AAL_ERR_WORKSPACE, "workspace has %zu bytes, %zu needed", workspace_bytes, need);
  }
  aal::MatmulArgs m{};
  m.a = operand_of(*a);
  m.b = operand_of(*b);
  m.st = static_cast<aal::Scale>(a->scale_type);
  m.M = M;
  m.N = N;
  m.K = K;
  m.c = c;
  m.out = to_dtype(raw(c_dtype));
  m.ws = workspace;
  m.stream = stream;
  return launched(aal::launch_matmul(m));
}

}  // extern "C"
