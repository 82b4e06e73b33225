// C ABI of beam search: argument validation and dispatch.  Declarations and the contract of every entry
// point are in include/aal.h.
#include "aal_api_common.h"
#include "aal_beam.h"


namespace {

constexpr int32_t kMostV = 1 << 18;  // the merge of a request's beams holds so many parts

bool finite(float x) {
  uint32_t u;
  memcpy(&u, &x, sizeof u);
  return ((u >> 23) & 0xffu) != 0xffu;
}

aal_status_t launched(hipError_t e) {
  return e == hipSuccess ? AAL_OK : fail(AAL_ERR_HIP, "kernel launch failed: %s", hipGetErrorString(e));
}

bool select_sizes(int64_t B, int32_t W, int32_t V, int32_t n) {
  return B >= 1 && W >= 1 && W <= AAL_BEAM_MAX && B < (int64_t(1) << 31) / W && V >= 1 && V <= kMostV && n >= 1 &&
         n <= AAL_BEAM_SELECT_MAX && n <= int64_t(W) * V;
}

// |stride| times count stays far from overflow.
bool stride_in_range(int64_t s) { return s > -(int64_t(1) << 46) && s < (int64_t(1) << 46); }

}  // namespace

extern "C" {

size_t aal_beam_select_workspace_bytes(aal_dtype_t in_dtype, int64_t B, int32_t W, int32_t V, int32_t n) {
  return valid_dtype(raw(in_dtype)) && select_sizes(B, W, V, n)
             ? aal::beam_workspace_bytes(to_dtype(raw(in_dtype)), B, W, V, n)
             : 0;
}

aal_status_t aal_beam_select(const void* z, aal_dtype_t in_dtype, int64_t B, int32_t W, int32_t V, int32_t n,
                             float temperature, const float* scores, const uint8_t* finished, const int32_t* lengths,
                             float length_penalty, int32_t eos, int32_t pad, const aal_beam_out_t* out,
                             void* workspace, size_t workspace_bytes, hipStream_t stream) {
  clear_error();
  if (!z || !scores || !out) return fail(AAL_ERR_ARG, "z, scores and out must be non-NULL");
  if (!out->parents || !out->tokens) return fail(AAL_ERR_ARG, "out: parents and tokens must be non-NULL");
  if (!select_sizes(B, W, V, n))
    return fail(AAL_ERR_ARG, "sizes must be: 1 <= W <= %d, B * W < 2^31, 1 <= V <= %d, 1 <= n <= min(%d, W * V)",
                AAL_BEAM_MAX, kMostV, AAL_BEAM_SELECT_MAX);
  if (!valid_dtype(raw(in_dtype))) return fail(AAL_ERR_DTYPE, "unknown in_dtype %d", raw(in_dtype));
  if (!positive_finite(temperature) || scale_for(temperature) == 0.f)
    return fail(AAL_ERR_ARG, "temperature must be finite, > 0 and >= 1e-37");
  if (!finite(length_penalty)) return fail(AAL_ERR_ARG, "length_penalty must be finite");
  if (!lengths && length_penalty != 0.f) return fail(AAL_ERR_ARG, "a length_penalty needs lengths");
  if (!aligned(z, 16)) return fail(AAL_ERR_ALIGN, "logit pointers must be 16-byte aligned");
  const aal::DType in = to_dtype(raw(in_dtype));
  const size_t need = aal::beam_workspace_bytes(in, B, W, V, n);
  if (!workspace) return fail(AAL_ERR_WORKSPACE, "workspace must be non-NULL");
  if (!aligned(workspace, 256)) return fail(AAL_ERR_ALIGN, "workspace must be 256-byte aligned");
  if (workspace_bytes < need) return fail(AAL_ERR_WORKSPACE, "workspace has %zu bytes, %zu needed", workspace_bytes, need);
  aal::BeamArgs a{};
  a.in = in;
  a.z = z;
  a.B = B;
  a.W = W;
  a.V = V;
  a.n = n;
  a.temperature = temperature;
  a.scores = scores;
  a.finished = finished;
  a.lengths = lengths;
  a.length_penalty = length_penalty;
  a.eos = eos;
  a.pad = pad;
  a.out = {out->scores, out->rank, out->parents, out->tokens, out->finished, out->lengths};
  a.ws = workspace;
  a.stream = stream;
  return launched(aal::launch_beam_select(a));
}

aal_status_t aal_beam_reorder(const aal_beam_state_t* states, int32_t n_states, int64_t B, int32_t W, int32_t n,
                              const int32_t* parents, hipStream_t stream) {
  clear_error();
  if (n_states < 0 || (n_states > 0 && !states)) return fail(AAL_ERR_ARG, "states must be non-NULL, n_states >= 0");
  if (!parents) return fail(AAL_ERR_ARG, "parents must be non-NULL");
  if (W < 1 || n < 1 || n > AAL_BEAM_SELECT_MAX || B < 1 || B >= (int64_t(1) << 31) / n || B >= (int64_t(1) << 31) / W)
    return fail(AAL_ERR_ARG, "sizes must be: W >= 1, 1 <= n <= %d, B * n and B * W < 2^31", AAL_BEAM_SELECT_MAX);
  int in_place = 0;
  for (int32_t i = 0; i < n_states; ++i) {
    const aal_beam_state_t& s = states[i];
    if (s.segments < 0 || s.segment_bytes < 0 || s.segments >= (int64_t(1) << 39) || s.segment_bytes >= (int64_t(1) << 39) ||
        (s.segment_bytes > 0 && s.segments > (int64_t(1) << 39) / s.segment_bytes))
      return fail(AAL_ERR_ARG, "state %d: segments * segment_bytes must be in [0, 2^39]", i);
    if (!s.src && s.segments * s.segment_bytes > 0) return fail(AAL_ERR_ARG, "state %d: src must be non-NULL", i);
    // more than any memory holds: sums of such sizes would overflow, and their launches never end
    if (s.segments * s.segment_bytes > (int64_t(1) << 50) / (B * n))
      return fail(AAL_ERR_ARG, "state %d: B * n * segments * segment_bytes must be in [0, 2^50]", i);
    for (int64_t st : {s.src_request, s.src_beam, s.src_segment, s.dst_request, s.dst_beam, s.dst_segment})
      if (!stride_in_range(st)) return fail(AAL_ERR_ARG, "state %d: a stride is out of range", i);
    in_place += s.dst == nullptr;
  }
  if (in_place && (n != W || n > AAL_BEAM_MAX))
    return fail(AAL_ERR_ARG, "in place, n must be W and at most %d (got n = %d, W = %d)", AAL_BEAM_MAX, n, W);
  for (int where = 0; where < 2; ++where) {
    // states in place and others are different kernels; 64 at a time, on the stack
    aal::BeamState some[64];
    aal::ReorderArgs a{};
    a.states = some;
    a.B = B;
    a.W = W;
    a.n = n;
    a.parents = parents;
    a.in_place = where == 0;
    a.stream = stream;
    for (int32_t i = 0; i <= n_states; ++i) {
      if (a.n_states == 64 || (i == n_states && a.n_states > 0)) {
        if (aal_status_t st = launched(aal::launch_beam_reorder(a)); st != AAL_OK) return st;
        a.n_states = 0;
      }
      if (i == n_states || (states[i].dst == nullptr) != a.in_place) continue;
      const aal_beam_state_t& s = states[i];
      uint8_t* src = const_cast<uint8_t*>(static_cast<const uint8_t*>(s.src));
      aal::BeamState& to = some[a.n_states++];
      to = {src, static_cast<uint8_t*>(s.dst), s.src_request, s.src_beam, s.src_segment,
            s.dst_request, s.dst_beam, s.dst_segment, s.segments, s.segment_bytes};
      if (a.in_place) {
        to.dst = src;
        to.dst_request = s.src_request;
        to.dst_beam = s.src_beam;
        to.dst_segment = s.src_segment;
      }
    }
  }
  return AAL_OK;
}

}  // extern "C"
