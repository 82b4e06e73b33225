// What a server does to logits before it samples from them or verifies drafts
// with them (aal_logits_process), and the gradient through it
// (aal_logits_process_bwd):
//
//   x  = z + bias
//   x  = x > 0 ? x / repetition : x * repetition      tokens of the row's history
//   x -= frequency * c + presence * [c > 0]           c: times among the generated tokens
//   out = -inf where the row's grammar mask has no bit, else x (rounded once)
//
//   dz = 0 where blocked, g / repetition or g * repetition at a history's token
//   (by the sign of z + bias), else g
//
// One workgroup per row and slice of the vocabulary.  Its counters lie in LDS:
// 16 bits an entry (the high one: in the prompt) for rows that generated up to
// 32,767 tokens, 32 bits and half the slice at a time for longer ones or rows
// with biases.  It counts the history's tokens that fall into the slice, then
// streams the slice; a vector without counts, biases and blocked entries is
// copied as it is.
#include "aal_device.h"
#include "aal_rowops.h"
#include "aal_toplist.h"

namespace aal {
namespace {

constexpr int kLpWords = 8192;       // counter words of a slice: 16,384 entries of 16 bits
constexpr uint32_t kPrompt16 = 0x8000u, kPrompt32 = 0x80000000u;
constexpr int kNarrowMost = 32767;   // generated tokens that 15 bits count

struct LogitsParams {
  const void* src;   // forward: z; backward: the gradient that comes in
  const void* z;
  int z_bf16;
  void* out;
  int64_t rows;
  int V;
  int slice;         // vectors of a workgroup
  LogitsRules r;
};

__device__ __forceinline__ int64_t clamp64(int64_t x, int64_t lo, int64_t hi) {
  return x < lo ? lo : x > hi ? hi : x;
}

// The E mask bits of the vector whose first element is entry i of the row;
// entries outside [0, V) read as blocked or not, whatever they are.
template <int E>
__device__ __forceinline__ uint32_t mask_bits(const uint32_t* m, int i, int words) {
  const int w0 = i >> 5;  // -1 for a vector that starts before its row
  const uint32_t lo = m[max(w0, 0)], hi = m[min(max(w0 + 1, 0), words - 1)];
  const uint32_t a = w0 < 0 ? 0u : lo;
  return uint32_t(((uint64_t(hi) << 32) | a) >> (i & 31)) & ((1u << E) - 1u);
}

template <class TI, bool VEC, bool BWD, int BLK>
__global__ __launch_bounds__(BLK) void k_logits(LogitsParams p) {
  using Rv = RowVecs<TI, VEC>;
  using TG = std::conditional_t<TI::kVec == 8, GBf16, GF32>;
  constexpr int E = Rv::E;
  __shared__ __attribute__((aligned(16))) uint32_t sh_cnt[kLpWords];
  __shared__ __attribute__((aligned(16))) uint32_t sh_pos[kLpWords];

  const int64_t row = blockIdx.x;
  const Rv rv(row, p.rows, p.V);
  const int64_t e0 = row * int64_t(p.V);
  const int gs0 = int(blockIdx.y) * p.slice, gs1 = min(rv.ng, gs0 + p.slice);

  // the row's rules; whatever the arrays hold, reads stay inside them
  int64_t h0 = 0;
  int nh = 0, np = 0;
  float rep = 1.f, freq = 0.f, pres = 0.f;
  if (p.r.tokens != nullptr) {
    h0 = clamp64(p.r.hist_start[row], 0, p.r.n_tokens);
    nh = int(clamp64(p.r.hist_len[row], 0, p.r.n_tokens - h0));
    np = p.r.prompt_len != nullptr ? min(max(p.r.prompt_len[row], 0), nh) : 0;
    if (p.r.repetition != nullptr) rep = p.r.repetition[row];
    if (p.r.frequency != nullptr) freq = p.r.frequency[row];
    if (p.r.presence != nullptr) pres = p.r.presence[row];
  }
  int64_t b0 = 0;
  int nb = 0;
  if (p.r.bias_offsets != nullptr) {
    b0 = clamp64(p.r.bias_offsets[row], 0, p.r.n_bias);
    nb = int(clamp64(p.r.bias_offsets[row + 1], b0, p.r.n_bias) - b0);
  }
  const uint32_t* mask = nullptr;
  const int words = (p.V + 31) / 32;
  if (p.r.mask != nullptr) {
    const int64_t m = p.r.mask_row != nullptr ? int64_t(p.r.mask_row[row]) : p.r.n_masks == 1 ? 0 : row;
    if (m >= 0 && m < p.r.n_masks) mask = p.r.mask + m * words;
  }
  const bool wide = nb > 0 || nh - np > kNarrowMost;
  const bool rules = nh > 0 || nb > 0;
  const int step = wide ? kLpWords / E : 2 * kLpWords / E;  // vectors that the counters cover

  for (int gp0 = gs0; gp0 < gs1; gp0 += step) {
    const int gp1 = min(gs1, gp0 + step);
    if (rules) {
      const int n = (gp1 - gp0) * E;  // entries of this part
      const int used = wide ? n : (n + 1) / 2;
      __syncthreads();
      for (int i = threadIdx.x; i < used; i += BLK) {
        sh_cnt[i] = 0;
        if (nb > 0) sh_pos[i] = 0;
      }
      __syncthreads();
      const int first = gp0 * E - rv.head;  // the entry of counter 0
      for (int i = threadIdx.x; i < nh; i += BLK) {
        const int t = p.r.tokens[h0 + i];
        const int at = t - first;
        if (t < 0 || t >= p.V || at < 0 || at >= n) continue;
        if (wide) {
          if (i < np) atomicOr(&sh_cnt[at], kPrompt32);
          else atomicAdd(&sh_cnt[at], 1u);
        } else {
          const int sh = (at & 1) * 16;
          if (i < np) atomicOr(&sh_cnt[at >> 1], kPrompt16 << sh);
          else atomicAdd(&sh_cnt[at >> 1], 1u << sh);
        }
      }
      for (int i = threadIdx.x; i < nb; i += BLK) {
        const int t = p.r.bias_ids[b0 + i];
        const int at = t - first;
        // of equal ids the last one counts
        if (t >= 0 && t < p.V && at >= 0 && at < n) atomicMax(&sh_pos[at], uint32_t(i) + 1u);
      }
      __syncthreads();
    }
    for (int gi = gp0 + int(threadIdx.x); gi < gp1; gi += BLK) {
      u32x4 w = rv.load(p.src, gi);
      const int at = (gi - gp0) * E;
      uint32_t cnt[E], pos[E], any = 0;
#pragma unroll
      for (int e = 0; e < E; ++e) cnt[e] = pos[e] = 0;
      if (rules) {
#pragma unroll
        for (int e = 0; e < E; ++e) {
          if (wide) {
            cnt[e] = sh_cnt[at + e];
            if (nb > 0) pos[e] = sh_pos[at + e];
          } else {
            const uint32_t c = sh_cnt[(at + e) >> 1] >> ((e & 1) * 16) & 0xffffu;
            cnt[e] = (c & 0x7fffu) | (c & kPrompt16 ? kPrompt32 : 0u);
          }
          any |= cnt[e] | pos[e];
        }
      }
      float x[E];
      TI::unpack(to_uint4(w), x);
      if (any) {
#pragma unroll
        for (int e = 0; e < E; ++e) {
          if ((cnt[e] | pos[e]) == 0) continue;
          const int v = rv.index(gi, e);
          float y = x[e];
          if constexpr (BWD) y = p.z_bf16 ? Bf16::load1(p.z, e0 + v) : F32::load1(p.z, e0 + v);
          if (pos[e]) y += p.r.bias_values[b0 + pos[e] - 1];
          if constexpr (BWD) {
            if (cnt[e]) x[e] = y > 0.f ? x[e] / rep : x[e] * rep;
          } else {
            if (cnt[e]) {
              y = y > 0.f ? y / rep : y * rep;
              const uint32_t c = cnt[e] & ~kPrompt32;
              y -= freq * float(c) + (c ? pres : 0.f);
            }
            x[e] = y;
          }
        }
      }
      if (mask != nullptr) {
        const uint32_t free = mask_bits<E>(mask, rv.index(gi, 0), words);
        // by whole numbers: a blocked entry may hold anything, NaN too
        constexpr uint32_t kBlocked = BWD ? 0u : 0xff800000u;
#pragma unroll
        for (int e = 0; e < E; ++e)
          x[e] = __builtin_bit_cast(float, free >> e & 1u ? __builtin_bit_cast(uint32_t, x[e]) : kBlocked);
      }
      rv.template store<TG>(p.out, gi, x);
    }
  }
}

template <class TI, bool VEC, bool BWD>
hipError_t launch_vec(const LogitsArgs& a) {
  constexpr int kBlk = 512;
  LogitsParams p{};
  p.src = BWD ? a.grad_out : a.z;
  p.z = a.z;
  p.z_bf16 = a.in == DType::kBf16;
  p.out = a.out;
  p.rows = a.rows;
  p.V = a.V;
  p.r = a.rules;
  const int ng = a.V / TI::kVec + 2;  // at most: a row may start and end inside a vector
  p.slice = 2 * kLpWords / TI::kVec;
  const unsigned slices = unsigned((ng + p.slice - 1) / p.slice);
  k_logits<TI, VEC, BWD, kBlk><<<dim3(unsigned(a.rows), slices), kBlk, 0, a.stream>>>(p);
  return hipGetLastError();
}

template <class TI, bool BWD>
hipError_t launch_typed(const LogitsArgs& a) {
  return a.V % TI::kVec == 0 ? launch_vec<TI, true, BWD>(a) : launch_vec<TI, false, BWD>(a);
}

}  // namespace

hipError_t launch_logits(const LogitsArgs& a) {
  if (a.grad_out != nullptr)
    return a.gd == DType::kBf16 ? launch_typed<Bf16, true>(a) : launch_typed<F32, true>(a);
  return a.in == DType::kBf16 ? launch_typed<Bf16, false>(a) : launch_typed<F32, false>(a);
}

}  // namespace aal
