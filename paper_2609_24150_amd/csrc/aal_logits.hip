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
// One workgroup per row and slice of the vocabulary: it loads its first vectors, counts
// the history's tokens that fall into the slice in LDS, and streams the slice. A
// vector without counts, biases and blocked entries is copied as it is.
//   forward   16 bits an entry, the high one for the prompt
//   backward  one bit an entry: only whether the history holds it
//   wide      32 bits, and 32 more for the place of a bias, a part of the slice at a
//             time: rows that generated more than 32,767 tokens or have more than 256 biases
// Up to 256 biases of a row are marked by a bit an entry and found through a hash table in
// LDS (a search of the list cost 16,760 rows of 16,609 with up to 100 biases 927 us).
// A row whose penalties change nothing has no history.
//
// Bound by memory: 3,584 rows of 128,256 bf16, each with a prompt and up to 7 windows' tokens of
// history and a grammar mask: forward 344 us, 5.3 TB/s, 95% of what a lone read and write take;
// backward, which reads a third array where the history has entries, 395 us, 83%.
#include "aal_device.h"
#include "aal_rowops.h"
#include "aal_toplist.h"

namespace aal {
namespace {

constexpr int kLpWords = 8192;       // counter words, at most: 16,384 entries of 16 bits
constexpr uint32_t kPrompt16 = 0x8000u, kPrompt32 = 0x80000000u;
constexpr int kNarrowMost = 32767;   // generated tokens that 15 bits count
constexpr int kBiasMost = 256;       // biases of a row in LDS
constexpr int kBiasSlots = 2 * kBiasMost;
__device__ __forceinline__ int bias_slot(int v) { return int((uint32_t(v) * 2654435761u) >> 16) & (kBiasSlots - 1); }

struct LogitsParams {
  const void* src;   // forward: z; backward: the gradient that comes in
  const void* z;
  int z_bf16;
  void* out;
  int64_t rows, row0;  // all of them, the first one of the launch
  int V;
  int slice;         // vectors of a workgroup
  int words;         // counter words in LDS, a multiple of 8
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

// U vectors of a thread are loaded at once.
template <class TI, bool VEC, bool BWD, bool BIAS, int BLK, int U, int MINW>
__global__ __launch_bounds__(BLK, MINW) void k_logits(LogitsParams p) {
  using Rv = RowVecs<TI, VEC>;
  using TG = std::conditional_t<TI::kVec == 8, GBf16, GF32>;
  constexpr int E = Rv::E;
  constexpr int kBiasRounds = (kBiasMost + BLK - 1) / BLK;
  extern __shared__ __attribute__((aligned(16))) uint32_t sh_cnt[];  // p.words of them
  uint32_t* const sh_biased = sh_cnt + p.words;                      // BIAS: a bit an entry
  // the part's biases by entry (a hash table), and the place of the last one there
  __shared__ int sh_bkey[BIAS ? kBiasSlots : 1];
  __shared__ uint32_t sh_bpos[BIAS ? kBiasSlots : 1];
  __shared__ float sh_bval[BIAS ? kBiasSlots : 1];

  const int64_t row = p.row0 + blockIdx.x;
  const Rv rv(row, p.rows, p.V);
  const int64_t e0 = row * int64_t(p.V);
  const int gs0 = int(blockIdx.y) * p.slice, gs1 = min(rv.ng, gs0 + p.slice);
  if (gs0 >= gs1) return;

  // the row's rules; whatever the arrays hold, reads stay inside them
  int64_t h0 = 0;
  int nh = 0, np = 0;
  float rep = 1.f, freq = 0.f, pres = 0.f;
  if (p.r.tokens != nullptr) {
    if (p.r.repetition != nullptr) rep = p.r.repetition[row];
    if (!BWD && p.r.frequency != nullptr) freq = p.r.frequency[row];
    if (!BWD && p.r.presence != nullptr) pres = p.r.presence[row];
    if (rep != 1.f || freq != 0.f || pres != 0.f) {
      h0 = clamp64(p.r.hist_start[row], 0, p.r.n_tokens);
      nh = int(clamp64(p.r.hist_len[row], 0, p.r.n_tokens - h0));
      if (!BWD && p.r.prompt_len != nullptr) np = min(max(p.r.prompt_len[row], 0), nh);
    }
  }
  int64_t b0 = 0;
  int nb = 0;
  if constexpr (BIAS) {
    b0 = clamp64(p.r.bias_offsets[row], 0, p.r.n_bias);
    nb = int(clamp64(p.r.bias_offsets[row + 1], b0, p.r.n_bias) - b0);
    if (BWD && nh == 0) nb = 0;  // a bias alone leaves the gradient as it is
  }
  const uint32_t* mask = nullptr;
  const int words = (p.V + 31) / 32;
  if (p.r.mask != nullptr) {
    const int64_t m = p.r.mask_row != nullptr ? int64_t(p.r.mask_row[row]) : p.r.n_masks == 1 ? 0 : row;
    if (m >= 0 && m < p.r.n_masks) mask = p.r.mask + m * words;
  }
  const bool many = BIAS && nb > kBiasMost;
  const bool wide = many || (!BWD && nh - np > kNarrowMost);
  const bool rules = nh > 0 || nb > 0;
  uint32_t* const sh_pos = sh_cnt + p.words / 2;
  // vectors that the counters cover
  const int step = wide ? (many ? p.words / 2 : p.words) / E : p.slice;

  for (int gp0 = gs0; gp0 < gs1; gp0 += step) {
    const int gp1 = min(gs1, gp0 + step);
    // the first vectors are on their way while the history is counted
    u32x4 w[1][U];
    rv.load({p.src}, gp0 + int(threadIdx.x), BLK, w);
    if (rules) {
      const int n = (gp1 - gp0) * E;  // entries of this part
      const int used = ((wide ? n : BWD ? (n + 31) / 32 : n / 2) + 3) / 4;
      __syncthreads();
      const uint4 zero = make_uint4(0, 0, 0, 0);
      for (int i = threadIdx.x; i < used; i += BLK) {
        reinterpret_cast<uint4*>(sh_cnt)[i] = zero;
        if (many) reinterpret_cast<uint4*>(sh_pos)[i] = zero;
      }
      if (BIAS && nb > 0 && !many) {
        for (int i = threadIdx.x; i < (n + 127) / 128; i += BLK) reinterpret_cast<uint4*>(sh_biased)[i] = zero;
        for (int i = threadIdx.x; i < kBiasSlots; i += BLK) {
          sh_bkey[i] = -1;
          sh_bpos[i] = 0;
        }
      }
      __syncthreads();
      const int first = gp0 * E - rv.head;  // the entry of counter 0
      const int lo = max(first, 0), hi = min(first + n, p.V);  // the entries of this part
      auto count = [&](uint32_t i, int t) {
        if (t < lo || t >= hi) return;
        const int at = t - first;
        if (wide) {
          if (i < uint32_t(np)) atomicOr(&sh_cnt[at], kPrompt32);
          else atomicAdd(&sh_cnt[at], 1u);
        } else if (BWD) {
          atomicOr(&sh_cnt[at >> 5], 1u << (at & 31));
        } else {
          const int sh = (at & 1) * 16;
          if (i < uint32_t(np)) atomicOr(&sh_cnt[at >> 1], kPrompt16 << sh);
          else atomicAdd(&sh_cnt[at >> 1], 1u << sh);
        }
      };
      // four tokens of a thread at once: a wait for memory per 4 BLK tokens (unsigned: the index
      // of the next ones passes 2^31 in a history of nearly that length)
      const uint32_t tokens = uint32_t(nh);
      uint32_t i = threadIdx.x;
      for (; i + 3 * BLK < tokens; i += 4 * BLK) {
        int t[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) t[q] = p.r.tokens[h0 + i + q * BLK];
#pragma unroll
        for (int q = 0; q < 4; ++q) count(i + q * BLK, t[q]);
      }
      for (; i < tokens; i += BLK) count(i, p.r.tokens[h0 + i]);
      if constexpr (BIAS) {
        // of equal ids the last one counts
        if (many) {
          for (int j = threadIdx.x; j < nb; j += BLK) {
            const int t = p.r.bias_ids[b0 + j];
            if (t >= lo && t < hi) atomicMax(&sh_pos[t - first], uint32_t(j) + 1u);
          }
        } else {
          int slot[kBiasRounds];
          float value[kBiasRounds];
#pragma unroll
          for (int q = 0; q < kBiasRounds; ++q) {
            const int j = int(threadIdx.x) + q * BLK;
            slot[q] = -1;
            if (j >= nb) continue;
            const int t = p.r.bias_ids[b0 + j];
            value[q] = p.r.bias_values[b0 + j];
            if (t < lo || t >= hi) continue;
            int h = bias_slot(t);
            for (int n = 0; n < kBiasSlots; ++n) {  // never more than half full
              const int was = atomicCAS(&sh_bkey[h], -1, t);
              if (was == -1 || was == t) break;
              h = (h + 1) & (kBiasSlots - 1);
            }
            slot[q] = h;
            atomicMax(&sh_bpos[h], uint32_t(j) + 1u);
            atomicOr(&sh_biased[(t - first) >> 5], 1u << ((t - first) & 31));
          }
          if (nb > 0) __syncthreads();
#pragma unroll
          for (int q = 0; q < kBiasRounds; ++q)
            if (slot[q] >= 0 && sh_bpos[slot[q]] == uint32_t(threadIdx.x) + uint32_t(q * BLK) + 1u) sh_bval[slot[q]] = value[q];
        }
      }
      __syncthreads();
    }
    // the counters of a vector (bit 31: in the prompt), and a bit for each biased entry
    auto counters = [&](int gi, uint32_t (&c)[E], uint32_t& biased) {
      const int at = (gi - gp0) * E;
      uint32_t any = 0;
      biased = 0;
      if (wide) {
#pragma unroll
        for (int e = 0; e < E; ++e) {
          c[e] = sh_cnt[at + e];
          any |= c[e];
          if (many && sh_pos[at + e] != 0u) biased |= 1u << e;
        }
        if (BIAS && nb > 0 && !many) biased = sh_biased[at >> 5] >> (at & 31) & ((1u << E) - 1u);
        return any;
      }
      if constexpr (BWD) {
        any = sh_cnt[at >> 5] >> (at & 31) & ((1u << E) - 1u);
#pragma unroll
        for (int e = 0; e < E; ++e) c[e] = any >> e & 1u;
      } else {
        uint32_t two[E / 2];
        __builtin_memcpy(two, __builtin_assume_aligned(sh_cnt + at / 2, E * 2), E * 2);
#pragma unroll
        for (int q = 0; q < E / 2; ++q) any |= two[q];
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const uint32_t h = e & 1 ? two[e / 2] >> 16 : two[e / 2] & 0xffffu;
          c[e] = (h & 0x7fffu) | ((h & kPrompt16) << 16);
        }
      }
      if (BIAS && nb > 0) biased = sh_biased[at >> 5] >> (at & 31) & ((1u << E) - 1u);
      return any;
    };
    auto bias_of = [&](int gi, int e) {
      if (many) return p.r.bias_values[b0 + sh_pos[(gi - gp0) * E + e] - 1];
      const int v = rv.index(gi, e);
      int h = bias_slot(v);
      for (int n = 0; n < kBiasSlots && sh_bkey[h] != v; ++n) h = (h + 1) & (kBiasSlots - 1);
      return sh_bval[h];
    };
    for (int base = gp0 + int(threadIdx.x); base < gp1; base += BLK * U) {
      if (base >= gp0 + BLK * U) rv.load({p.src}, base, BLK, w);
      // backward: the logits of the vectors with seen entries, all on their way at once
      u32x4 zv[BWD ? U : 1];
      const bool same = BWD && p.z_bf16 == (E == 8);
      if constexpr (BWD)
        if (rules && same) {
#pragma unroll
          for (int u = 0; u < U; ++u) {
            const int gi = base + u * BLK;
            uint32_t c[E], biased;
            zv[u] = Rv::none();
            if (gi < gp1 && counters(gi, c, biased)) zv[u] = rv.load(p.z, gi);
          }
        }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int gi = base + u * BLK;
        if (gi >= gp1) break;
        float x[E];
        TI::unpack(to_uint4(w[0][u]), x);
        if (rules) {
          uint32_t c[E], biased;
          const uint32_t any = counters(gi, c, biased);
          if constexpr (BWD) {
            if (any) {
              float y[E];
              if (same) {
                TI::unpack(to_uint4(zv[u]), y);
              } else {
#pragma unroll
                for (int e = 0; e < E; ++e) {
                  const int64_t at = e0 + (c[e] ? rv.index(gi, e) : 0);
                  y[e] = p.z_bf16 ? Bf16::load1(p.z, at) : F32::load1(p.z, at);
                }
              }
#pragma unroll
              for (int e = 0; e < E; ++e) {
                if (c[e] == 0u) continue;
                if (BIAS && (biased >> e & 1u)) y[e] += bias_of(gi, e);
                x[e] = y[e] > 0.f ? x[e] / rep : x[e] * rep;
              }
            }
          } else if (any | biased) {
#pragma unroll
            for (int e = 0; e < E; ++e) {
              float y = x[e];
              if (BIAS && (biased >> e & 1u)) y += bias_of(gi, e);
              if (c[e]) {
                y = y > 0.f ? y / rep : y * rep;
                const uint32_t n = c[e] & ~kPrompt32;
                y -= freq * float(n) + (n ? pres : 0.f);
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
}

// Entries of a workgroup's slice: as many as the counters hold at once (backward, where
// they hold a whole row, a quarter of 131,072), fewer where that makes fewer than
// 1,024 workgroups, four a CU, but at least 4,096 or the history is read too often.
template <bool BWD>
int slice_entries(int64_t rows, int V) {
  int n = BWD ? 32768 : 2 * kLpWords;
  while (n > 4096 && rows * ((V + n - 1) / n) < 1024) n /= 2;
  return n;
}

template <class TI, bool VEC, bool BWD, bool BIAS>
hipError_t launch_vec(const LogitsArgs& a) {
  LogitsParams p{};
  p.src = BWD ? a.grad_out : a.z;
  p.z = a.z;
  p.z_bf16 = a.in == DType::kBf16;
  p.out = a.out;
  p.rows = a.rows;
  p.V = a.V;
  p.r = a.rules;
  const int ng = a.V / TI::kVec + (VEC ? 0 : 2);  // at most: a row may start and end inside a vector
  // slices of one size, to a KB
  const int most = slice_entries<BWD>(a.rows, a.V) / TI::kVec, slices = (ng + most - 1) / most;
  p.slice = ((ng + slices - 1) / slices + 63) / 64 * 64;
  // LDS by the slice, so that as many workgroups of short rows fit a CU as of long ones: of the forward's
  // counters in both directions (the backward's bits need less, but its registers, not
  // LDS, say how many workgroups fit)
  const int entries = p.slice * TI::kVec;
  p.words = (entries / 2 < kLpWords ? entries / 2 : kLpWords);
  const size_t lds = size_t(p.words + (BIAS ? entries / 32 : 0)) * 4;
  auto run = [&](auto kern, int blk) {
    return for_row_parts(a.rows, [&](int64_t row0, unsigned n) {
      p.row0 = row0;
      kern<<<dim3(n, unsigned(slices)), blk, lds, a.stream>>>(p);
      return hipGetLastError();
    });
  };
  constexpr int kMinWaves = !VEC && BIAS ? 4 : BWD ? 5 : BIAS || !VEC ? 6 : 8;
  if (ng <= 512) return run(k_logits<TI, VEC, BWD, BIAS, 128, 4, kMinWaves>, 128);
  if (ng <= 1024) return run(k_logits<TI, VEC, BWD, BIAS, 256, 4, kMinWaves>, 256);
  return run(k_logits<TI, VEC, BWD, BIAS, 512, 4, kMinWaves>, 512);
}

template <class TI, bool BWD>
hipError_t launch_typed(const LogitsArgs& a) {
  const bool bias = a.rules.bias_offsets != nullptr;
  if (a.V % TI::kVec == 0) return bias ? launch_vec<TI, true, BWD, true>(a) : launch_vec<TI, true, BWD, false>(a);
  return bias ? launch_vec<TI, false, BWD, true>(a) : launch_vec<TI, false, BWD, false>(a);
}

}  // namespace

hipError_t launch_logits(const LogitsArgs& a) {
  if (a.grad_out != nullptr)
    return a.gd == DType::kBf16 ? launch_typed<Bf16, true>(a) : launch_typed<F32, true>(a);
  return a.in == DType::kBf16 ? launch_typed<Bf16, false>(a) : launch_typed<F32, false>(a);
}

}  // namespace aal
