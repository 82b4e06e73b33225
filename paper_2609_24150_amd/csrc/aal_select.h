// Pieces of selection by size that the extraction of top logits and beam search share.
#pragma once

#include "aal_device.h"

namespace aal {
namespace {

// A whole number that orders as the logits do, -0 as +0: 16 bits for bf16
// (in the upper half), 32 for fp32.
template <class TI>
constexpr int key_bits() { return TI::kVec == 8 ? 16 : 32; }
template <class TI>
__device__ __forceinline__ uint32_t order_key(float x) {
  const uint32_t b = __builtin_bit_cast(uint32_t, x) == 0x80000000u ? 0u : __builtin_bit_cast(uint32_t, x);
  return (b ^ (uint32_t(int32_t(b) >> 31) | 0x80000000u)) & (key_bits<TI>() == 16 ? 0xffff0000u : 0xffffffffu);
}
template <class TI>
__device__ __forceinline__ float key_logit(uint32_t key) {
  return __builtin_bit_cast(float, key ^ ((key >> 31) ? 0x80000000u : key_bits<TI>() == 16 ? 0xffff0000u : 0xffffffffu));
}

// A threshold that at least k of the block's values (N per thread) reach, and
// few more: every wave bisects for one that its share of k reaches, without a
// barrier, and the lowest of them serves for all.  -inf where some wave has
// fewer finite values than its share.  Shares may differ, if they make k together.
template <class TI, int WAVES, int N>
__device__ __forceinline__ float threshold_of_shares(const float (&x)[N], int share, float top, float* sh) {
  constexpr int kShift = 32 - key_bits<TI>();
  const uint32_t least = order_key<TI>(kNegInf) >> kShift;
  uint32_t lo = least, hi = (order_key<TI>(top) >> kShift) + 1u;  // lo is reached by the share or all, hi by none
  const int most = share + share / 8 + 1;
  // the first probe two octaves below the top, where the share mostly is above: less to bisect
  const uint32_t octaves = 2u << (23 - kShift);
  uint32_t probe = hi > least + octaves ? hi - octaves : lo + (hi - lo) / 2;
  while (hi > lo + 1u) {
    const float t = key_logit<TI>(probe << kShift);
    int c = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) c += __popcll(__builtin_amdgcn_ballot_w64(x[i] >= t));
    if (c >= share) {
      lo = probe;
      if (c <= most) break;
    } else {
      hi = probe;
    }
    probe = lo + (hi - lo) / 2;
  }
  float t = share == 0 ? top : key_logit<TI>(lo << kShift);
  if constexpr (WAVES > 1) {
    if ((threadIdx.x & (kWave - 1)) == 0) sh[threadIdx.x / kWave] = t;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < WAVES; ++i) t = fminf(t, sh[i]);
    __syncthreads();
  }
  return t;
}
template <class TI, int WAVES, int N>
__device__ __forceinline__ float threshold(const float (&x)[N], int k, float top, float* sh) {
  return threshold_of_shares<TI, WAVES>(x, (k + WAVES - 1) / WAVES, top, sh);
}

}  // namespace
}  // namespace aal
