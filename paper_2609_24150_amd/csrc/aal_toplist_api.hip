// C ABI of the operators on a target's top logits and of the logits
// processing: argument validation, workspace carve-up and dispatch.
// Declarations and the contract of every entry point are in include/aal.h.
#include "aal_api_common.h"
#include "aal_toplist.h"

namespace {

constexpr int32_t kMostLossV = 1 << 19;     // the list's bitmap has a bit for each entry
constexpr int32_t kMostProcessV = 1 << 24;  // a workgroup for each piece of a row in the grid

// Neither NaN nor infinite, on the bit pattern.
bool finite(float x) {
  uint32_t u;
  memcpy(&u, &x, sizeof u);
  return ((u >> 23) & 0xffu) != 0xffu;
}

aal_status_t check_rows(int64_t rows, int32_t V, int32_t most_v) {
  if (rows < 1 || rows >= (int64_t(1) << 31)) return fail(AAL_ERR_ARG, "rows must be in [1, 2^31) (got %lld)", (long long)rows);
  if (V < 1 || V > most_v) return fail(AAL_ERR_ARG, "V must be in [1, %d] (got %d)", most_v, V);
  return AAL_OK;
}

aal_status_t check_workspace(const void* ws, size_t have, size_t need) {
  if (!ws) return fail(AAL_ERR_WORKSPACE, "workspace must be non-NULL");
  if (!aligned(ws, 256)) return fail(AAL_ERR_ALIGN, "workspace must be 256-byte aligned");
  if (have < need) return fail(AAL_ERR_WORKSPACE, "workspace has %zu bytes, %zu needed", have, need);
  return AAL_OK;
}

aal_status_t launched(hipError_t e) {
  return e == hipSuccess ? AAL_OK : fail(AAL_ERR_HIP, "kernel launch failed: %s", hipGetErrorString(e));
}

// Rows and windows of a layout; false where the sizes are none.
bool layout_sizes(int layout, int64_t B, int32_t S, int32_t K, int64_t* rows, int64_t* windows) {
  if (layout != AAL_LAYOUT_WINDOWS && layout != AAL_LAYOUT_SEQUENCES) return false;
  if (B < 1 || K < 1 || K > 64) return false;
  const int64_t s = layout == AAL_LAYOUT_WINDOWS ? K : S;
  if (s < 1 || B >= (int64_t(1) << 31) / s) return false;
  *rows = B * s;
  *windows = layout == AAL_LAYOUT_WINDOWS ? B : s < K ? 0 : B * (s - K + 1);
  return true;
}

// The pointers of a set of rules that go together.
aal_status_t check_rules(const aal_logits_rules_t* r, int64_t rows) {
  if (r->tokens) {
    if (!r->hist_start || !r->hist_len) return fail(AAL_ERR_ARG, "tokens need hist_start and hist_len");
    if (r->n_tokens < 0) return fail(AAL_ERR_ARG, "n_tokens must be >= 0");
  } else if (r->hist_start || r->hist_len || r->prompt_len || r->repetition || r->frequency || r->presence) {
    return fail(AAL_ERR_ARG, "penalties need tokens");
  }
  if (r->bias_offsets) {
    if (!r->bias_ids || !r->bias_values) return fail(AAL_ERR_ARG, "bias_offsets need bias_ids and bias_values");
    if (r->n_bias < 0 || r->n_bias >= (int64_t(1) << 31)) return fail(AAL_ERR_ARG, "n_bias must be in [0, 2^31)");
  } else if (r->bias_ids || r->bias_values) {
    return fail(AAL_ERR_ARG, "biases need bias_offsets");
  }
  if (r->mask) {
    if (r->n_masks < 1) return fail(AAL_ERR_ARG, "n_masks must be >= 1");
    if (!r->mask_row && r->n_masks != 1 && r->n_masks < rows)
      return fail(AAL_ERR_ARG, "without mask_row there must be one mask, or one for each row");
  } else if (r->mask_row) {
    return fail(AAL_ERR_ARG, "mask_row needs mask");
  }
  return AAL_OK;
}

aal::LogitsRules rules_of(const aal_logits_rules_t& r) {
  return {r.tokens,   r.n_tokens,     r.hist_start, r.hist_len,    r.prompt_len, r.repetition, r.frequency, r.presence,
          r.bias_offsets, r.bias_ids, r.bias_values, r.n_bias, r.mask, r.n_masks, r.mask_row};
}

}  // namespace

extern "C" {

aal_status_t aal_topk_logits(const void* z, aal_dtype_t in_dtype, int64_t rows, int32_t V, int32_t k,
                             float temperature, void* top_logits, int32_t* top_ids, float* rest,
                             hipStream_t stream) {
  clear_error();
  if (!z) return fail(AAL_ERR_ARG, "z must be non-NULL");
  if (!top_logits || !top_ids) return fail(AAL_ERR_ARG, "top_logits and top_ids must be non-NULL");
  if (aal_status_t s = check_rows(rows, V, 1 << 30); s != AAL_OK) return s;
  if (k < 1 || k > AAL_TOPK_MAX || k > V)
    return fail(AAL_ERR_ARG, "k must be in [1, min(V, %d)] (got %d)", AAL_TOPK_MAX, k);
  if (!valid_dtype(raw(in_dtype))) return fail(AAL_ERR_DTYPE, "unknown in_dtype %d", raw(in_dtype));
  const float sc = scale_for(temperature);
  if (!positive_finite(temperature) || sc == 0.f)
    return fail(AAL_ERR_ARG, "temperature must be finite, > 0 and >= 1e-37");
  if (!aligned(z, 16)) return fail(AAL_ERR_ALIGN, "logit pointers must be 16-byte aligned");
  aal::TopkArgs a{};
  a.in = to_dtype(raw(in_dtype));
  a.z = z;
  a.rows = rows;
  a.V = V;
  a.k = k;
  a.sc = sc;
  a.inv_t = 1.0f / temperature;
  a.top = top_logits;
  a.ids = top_ids;
  a.rest = rest;
  a.stream = stream;
  return launched(aal::launch_topk(a));
}

size_t aal_topk_loss_workspace_bytes(aal_layout_t layout, int64_t B, int32_t S, int32_t K) {
  int64_t rows = 0, windows = 0;
  return layout_sizes(raw(layout), B, S, K, &rows, &windows) ? aal::top_loss_workspace_bytes(rows) : 0;
}

aal_status_t aal_topk_loss_fwd_bwd(const void* z_draft, aal_dtype_t in_dtype, const void* top_logits,
                                   aal_dtype_t top_dtype, const int32_t* top_ids, const float* rest,
                                   aal_layout_t layout, int64_t B, int32_t S, int32_t K, int32_t V, int32_t k,
                                   float temp_draft, float temp_target, aal_loss_weights_t weights, float* loss,
                                   float* terms, float* e_tv, float* e_eal, float* accept_tv, float* accept_eal,
                                   int32_t* xstar, void* grad_draft, aal_dtype_t grad_dtype, const float* grad_scale,
                                   uint32_t flags, void* workspace, size_t workspace_bytes, hipStream_t stream) {
  clear_error();
  if (!z_draft || !top_logits || !top_ids) return fail(AAL_ERR_ARG, "z_draft, top_logits and top_ids must be non-NULL");
  if (!loss) return fail(AAL_ERR_ARG, "loss must be non-NULL");
  int64_t rows = 0, windows = 0;
  if (!layout_sizes(raw(layout), B, S, K, &rows, &windows))
    return fail(AAL_ERR_ARG, "layout, B, S or K is invalid (K in [1, 64], fewer than 2^31 rows)");
  if (aal_status_t s = check_rows(rows, V, kMostLossV); s != AAL_OK) return s;
  if (k < 1 || k > AAL_TOPK_MAX || k > V)
    return fail(AAL_ERR_ARG, "k must be in [1, min(V, %d)] (got %d)", AAL_TOPK_MAX, k);
  if (!valid_dtype(raw(in_dtype))) return fail(AAL_ERR_DTYPE, "unknown in_dtype %d", raw(in_dtype));
  if (!valid_dtype(raw(top_dtype))) return fail(AAL_ERR_DTYPE, "unknown top_dtype %d", raw(top_dtype));
  if (grad_draft && !valid_dtype(raw(grad_dtype))) return fail(AAL_ERR_DTYPE, "unknown grad_dtype %d", raw(grad_dtype));
  const float scd = scale_for(temp_draft), sct = scale_for(temp_target);
  if (!positive_finite(temp_draft) || scd == 0.f)
    return fail(AAL_ERR_ARG, "temp_draft must be finite, > 0 and >= 1e-37");
  if (!positive_finite(temp_target) || sct == 0.f)
    return fail(AAL_ERR_ARG, "temp_target must be finite, > 0 and >= 1e-37");
  if (!finite(weights.wtv) || !finite(weights.eal) || !finite(weights.kl) || !finite(weights.tv))
    return fail(AAL_ERR_ARG, "weights must be finite");
  if (flags & ~(AAL_FLAG_STREAMING | AAL_FLAG_COOPERATIVE)) return fail(AAL_ERR_ARG, "unknown flags 0x%x", flags);
  if (!aligned(z_draft, 16)) return fail(AAL_ERR_ALIGN, "logit pointers must be 16-byte aligned");
  if (grad_draft && !aligned(grad_draft, 16)) return fail(AAL_ERR_ALIGN, "grad_draft must be 16-byte aligned");
  if (aal_status_t s = check_workspace(workspace, workspace_bytes, aal::top_loss_workspace_bytes(rows));
      s != AAL_OK)
    return s;
  aal::TopLossArgs a{};
  a.in = to_dtype(raw(in_dtype));
  a.td = to_dtype(raw(top_dtype));
  a.gd = grad_draft ? to_dtype(raw(grad_dtype)) : aal::DType::kF32;
  a.zd = z_draft;
  a.top = top_logits;
  a.ids = top_ids;
  a.rest = rest;
  a.layout = raw(layout) == AAL_LAYOUT_WINDOWS ? 0 : 1;
  a.B = B;
  a.S = a.layout == 0 ? K : S;
  a.K = K;
  a.V = V;
  a.k = k;
  a.R = rows;
  a.W = windows;
  a.sc_d = scd;
  a.sc_t = sct;
  a.inv_t_d = 1.0f / temp_draft;
  a.w_wtv = weights.wtv;
  a.w_eal = weights.eal;
  a.w_kl = weights.kl;
  a.w_tv = weights.tv;
  a.loss = loss;
  a.terms = terms;
  a.e_tv = e_tv;
  a.e_eal = e_eal;
  a.accept_tv = accept_tv;
  a.accept_eal = accept_eal;
  a.xstar = xstar;
  a.grad = grad_draft;
  a.grad_scale = grad_scale;
  uint8_t* w = static_cast<uint8_t*>(workspace);
  auto carve = [&w](size_t bytes) {
    uint8_t* at = w;
    w += aal::align256(bytes);
    return at;
  };
  a.stats = reinterpret_cast<aal::TopRow*>(carve(size_t(rows) * sizeof(aal::TopRow)));
  a.row_loss = reinterpret_cast<float2*>(carve(size_t(rows) * sizeof(float2)));
  a.loss_parts = reinterpret_cast<double*>(carve(size_t(aal::kTopLossParts) * 4 * sizeof(double)));
  a.slots = reinterpret_cast<uint64_t*>(carve(size_t(rows) * 2 * sizeof(uint64_t)));
  a.err = reinterpret_cast<unsigned*>(carve(256));
  a.streaming = (flags & AAL_FLAG_STREAMING) != 0;
  a.coop = (flags & AAL_FLAG_COOPERATIVE) != 0;
  a.stream = stream;
  return launched(aal::launch_top_loss(a));
}

aal_status_t aal_logits_process(const void* z, aal_dtype_t dtype, int64_t rows, int32_t V,
                                const aal_logits_rules_t* rules, void* out, hipStream_t stream) {
  clear_error();
  if (!z || !out || !rules) return fail(AAL_ERR_ARG, "z, rules and out must be non-NULL");
  if (aal_status_t s = check_rows(rows, V, kMostProcessV); s != AAL_OK) return s;
  if (!valid_dtype(raw(dtype))) return fail(AAL_ERR_DTYPE, "unknown dtype %d", raw(dtype));
  if (!aligned(z, 16) || !aligned(out, 16)) return fail(AAL_ERR_ALIGN, "logit pointers must be 16-byte aligned");
  if (aal_status_t s = check_rules(rules, rows); s != AAL_OK) return s;
  aal::LogitsArgs a{};
  a.in = to_dtype(raw(dtype));
  a.gd = a.in;
  a.z = z;
  a.out = out;
  a.rows = rows;
  a.V = V;
  a.rules = rules_of(*rules);
  a.stream = stream;
  return launched(aal::launch_logits(a));
}

aal_status_t aal_logits_process_bwd(const void* grad_out, aal_dtype_t grad_dtype, const void* z, aal_dtype_t in_dtype,
                                    int64_t rows, int32_t V, const aal_logits_rules_t* rules, void* grad_z,
                                    hipStream_t stream) {
  clear_error();
  if (!grad_out || !z || !grad_z || !rules) return fail(AAL_ERR_ARG, "grad_out, z, rules and grad_z must be non-NULL");
  if (aal_status_t s = check_rows(rows, V, kMostProcessV); s != AAL_OK) return s;
  if (!valid_dtype(raw(in_dtype))) return fail(AAL_ERR_DTYPE, "unknown in_dtype %d", raw(in_dtype));
  if (!valid_dtype(raw(grad_dtype))) return fail(AAL_ERR_DTYPE, "unknown grad_dtype %d", raw(grad_dtype));
  if (!aligned(grad_out, 16) || !aligned(z, 16) || !aligned(grad_z, 16))
    return fail(AAL_ERR_ALIGN, "logit and gradient pointers must be 16-byte aligned");
  if (aal_status_t s = check_rules(rules, rows); s != AAL_OK) return s;
  aal::LogitsArgs a{};
  a.in = to_dtype(raw(in_dtype));
  a.gd = to_dtype(raw(grad_dtype));
  a.z = z;
  a.grad_out = grad_out;
  a.out = grad_z;
  a.rows = rows;
  a.V = V;
  a.rules = rules_of(*rules);
  a.stream = stream;
  return launched(aal::launch_logits(a));
}

}  // extern "C"
