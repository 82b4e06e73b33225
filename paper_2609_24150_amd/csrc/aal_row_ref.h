// The reference of a row's sums of exponentials, for the operators on top lists.
#pragma once

#include "aal_device.h"

namespace aal {
namespace {

// Entries count 2^(z sc - msc), sc = log2(e) / T, the logit `m` 1.  msc is m sc rounded, by up
// to 2^-25 of it, which cancels between entries but is an exponent: beyond 2^27 (8) sums
// could overflow or vanish.  A reference that large ("steep": a masked row, a temperature
// near zero) takes the difference before the product, which is exact where the result
// is no 0.  A sum that is not yet against the row's reference is against at least
// -2^27, from where a larger one loses nothing.
constexpr float kSteep = 0x1p27f;
struct RowRef {
  float m, sc, msc;
  bool steep;
};
__device__ __forceinline__ RowRef row_ref(float m, float sc) {
  const float msc = m == kNegInf ? 0.f : m * sc;
  return {m, sc, msc, fabsf(msc) > kSteep};
}
__device__ __forceinline__ float log2_of(const RowRef& r, float z) {
  return r.steep ? (z - r.m) * r.sc : __builtin_fmaf(z, r.sc, -r.msc);
}
// The reference of a thread's own sum whose largest logit is m.
__device__ __forceinline__ float own_ref(float m, float sc) { return fmaxf(m * sc, -kSteep); }

}  // namespace
}  // namespace aal
