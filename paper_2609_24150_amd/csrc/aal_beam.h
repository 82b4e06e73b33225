// Host-side interfaces of beam search: selection over beams and vocabulary,
// reordering of the beams' states.
#pragma once

#include "aal_internal.h"

namespace aal {

constexpr int kBeamMax = 64, kBeamSelectMax = 128;

struct BeamOut {
  float* scores;
  float* rank;
  int32_t* parents;
  int32_t* tokens;
  uint8_t* finished;
  int32_t* lengths;
};

// What a part of a row leaves: its largest logit and the sum of exp((z - that) / T).
struct BeamPart {
  double s;
  float m;
  int32_t pad;
};
static_assert(sizeof(BeamPart) == 16, "BeamPart layout");

struct BeamArgs {
  DType in;
  const void* z;
  int64_t B;
  int W, V, n;
  float temperature;
  const float* scores;
  const uint8_t* finished;  // may be null
  const int32_t* lengths;   // may be null
  float length_penalty;
  int32_t eos, pad;
  BeamOut out;
  void* ws;
  hipStream_t stream;
};

size_t beam_workspace_bytes(DType in, int64_t B, int W, int V, int n);
hipError_t launch_beam_select(const BeamArgs& a);

struct BeamState {
  const uint8_t* src;
  uint8_t* dst;
  int64_t src_request, src_beam, src_segment;
  int64_t dst_request, dst_beam, dst_segment;
  int64_t segments, segment_bytes;
};

struct ReorderArgs {
  const BeamState* states;  // host memory
  int n_states;
  int64_t B;
  int W, n;
  const int32_t* parents;
  bool in_place;
  hipStream_t stream;
};

hipError_t launch_beam_reorder(const ReorderArgs& a);

}  // namespace aal
