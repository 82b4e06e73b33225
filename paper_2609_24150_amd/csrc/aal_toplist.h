// Host-side interfaces of the operators on a target's top logits: extraction
// of a row's largest logits, the training objectives against such lists, and
// the processing of logits (biases, penalties, grammar masks).
#pragma once

#include "aal_internal.h"

namespace aal {

// A launch holds fewer than 2^32 threads: kernels of a workgroup or more per row take 2^22 rows
// of at most 512 threads at a time.
constexpr int64_t kLaunchRows = int64_t(1) << 22;
template <class F>
hipError_t for_row_parts(int64_t rows, F&& launch) {
  for (int64_t row0 = 0; row0 < rows; row0 += kLaunchRows)
    if (hipError_t e = launch(row0, unsigned(rows - row0 < kLaunchRows ? rows - row0 : kLaunchRows)); e != hipSuccess)
      return e;
  return hipSuccess;
}

// ------------------------------------------------------------ extraction
struct TopkArgs {
  DType in;
  const void* z;
  int64_t rows;
  int V, k;
  float sc, inv_t; // log2(e)/T, 1/T
  void* top;       // [rows, k] of the logits' type
  int32_t* ids;    // [rows, k]
  float* rest;     // [rows], may be null
  hipStream_t stream;
};

hipError_t launch_topk(const TopkArgs& a);

// ------------------------------------------- objectives against top lists
// Per-row results of the row pass and coefficients of the gradient.  72 bytes.
struct TopRow {
  float mu, ml;       // draft: largest unlisted and listed logit, the references of 2^(z*sc - m*sc)
  float qu, ql;       // and what takes a value against them to q
  float tmax, inv_zt; // target: largest logit of the list, p_i = inv_zt 2^((t - tmax)*sct)
  float a_tv, a_eal;  // acceptances
  float qlt;          // sum of q over the entries (the remainder among them) with q < p
  float kl;           // KL(p || q) in nats
  float pu;           // p_rest / sum of the unlisted values against mu, 0 where there are none
  int32_t xstar;      // greedy token of the list, -1 for an empty one
  int32_t flags;      // kTopHas: the row has a target; kTopRestBelow: q_rest < p_rest
  float cR;           // unlisted entries: g = cR 2^(z*sc - mu*sc)
  float cA, cB;       // listed entries: g = q (q < p ? cA : cB) - cP p + cX [v = x*]
  float cP, cX;
};
static_assert(sizeof(TopRow) == 72, "TopRow layout");
constexpr int kTopHas = 1, kTopRestBelow = 2;

struct TopLossArgs {
  DType in, td, gd;        // draft logits, listed logits, gradient
  const void* zd;
  const void* top;
  const int32_t* ids;
  const float* rest;       // may be null
  int layout;              // 0 windows, 1 sequences
  int64_t B;
  int S, K, V, k;
  int64_t R, W;            // rows, windows
  float sc_d, sc_t, inv_t_d;
  float w_wtv, w_eal, w_kl, w_tv;
  float* loss;
  float* terms;            // the rest may be null
  float* e_tv;
  float* e_eal;
  float* accept_tv;
  float* accept_eal;
  int32_t* xstar;
  void* grad;
  const float* grad_scale;
  TopRow* stats;           // workspace [R]
  float2* row_loss;        // workspace [R]: KL, windows that contain the row * (1 - a_tv)
  double* loss_parts;      // workspace [kTopLossParts][4]
  uint64_t* slots;         // workspace [R][2]: tagged acceptances of the resident schedule
  unsigned* err;           // workspace [2]: poll time-out flag of the resident schedule, a counter
  bool streaming, coop;
  hipStream_t stream;
};
constexpr int kTopLossParts = 64;

inline size_t top_loss_workspace_bytes(int64_t rows) {
  return align256(size_t(rows) * sizeof(TopRow)) +
         align256(size_t(rows) * sizeof(float2)) + align256(size_t(kTopLossParts) * 4 * sizeof(double)) +
         align256(size_t(rows) * 2 * sizeof(uint64_t)) + 256;
}

hipError_t launch_top_loss(const TopLossArgs& a);

// The resident schedule, by element types and by whether V is a multiple of the 16-byte
// vector; *used = false (and nothing enqueued) where no kernel holds the row.
hipError_t launch_top_fused_bf16_whole(const TopLossArgs& a, bool* used);
hipError_t launch_top_fused_bf16_ragged(const TopLossArgs& a, bool* used);
hipError_t launch_top_fused_bf16_g32_whole(const TopLossArgs& a, bool* used);
hipError_t launch_top_fused_bf16_g32_ragged(const TopLossArgs& a, bool* used);
hipError_t launch_top_fused_f32_whole(const TopLossArgs& a, bool* used);
hipError_t launch_top_fused_f32_ragged(const TopLossArgs& a, bool* used);

// ------------------------------------------------------ logits processing
struct LogitsRules {
  const int32_t* tokens;
  int64_t n_tokens;
  const int64_t* hist_start;
  const int32_t* hist_len;
  const int32_t* prompt_len;   // may be null: nothing but generated tokens
  const float* repetition;     // may be null: 1
  const float* frequency;      // may be null: 0
  const float* presence;       // may be null: 0
  const int64_t* bias_offsets;
  const int32_t* bias_ids;
  const float* bias_values;
  int64_t n_bias;
  const uint32_t* mask;
  int64_t n_masks;
  const int32_t* mask_row;     // may be null: row r takes mask r (or the only one)
};

struct LogitsArgs {
  DType in;                // logits
  DType gd;                // backward: gradients
  const void* z;
  const void* grad_out;    // null: forward
  void* out;               // processed logits, or the gradient w.r.t. z
  int64_t rows;
  int V;
  LogitsRules rules;
  hipStream_t stream;
};

hipError_t launch_logits(const LogitsArgs& a);

}  // namespace aal
