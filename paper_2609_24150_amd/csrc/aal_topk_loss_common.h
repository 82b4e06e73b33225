// What the two schedules of the objectives against top lists share: the list of a
// row, its windows and its coefficients (the mathematics is stated in
// aal_topk_loss.hip).
#pragma once

#include "aal_device.h"
#include "aal_resident_common.h"
#include "aal_rowops.h"
#include "aal_toplist.h"

#include <limits.h>

namespace aal {
namespace {

constexpr int kTopMax = 512;
constexpr float kLn2 = 0.693147180559945309417f;
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kDeepScale = 0x1p-64f;

struct TopLossParams {
  const void* zd;
  const void* top;
  const int32_t* ids;
  const float* rest;
  int64_t R;
  int V, k;
  float scd, sct;
  int top_bf16;
  TopRow* stats;       // multi-kernel schedule
  uint64_t* slots;     // [R][2]: the rows' acceptances, tagged
  float2* row_loss;    // [R]: KL, windows that contain the row * (1 - a_tv)
  unsigned* err;       // poll time-out
  unsigned* counter;   // of k_top_loss's workgroups: zeroed by the first kernel
  float* accept_tv;    // may be null
  float* accept_eal;
  int32_t* xstar;
  // windows and weights
  int layout;
  int S, K;
  int64_t W;
  float w_wtv, w_eal, w_kl, w_tv;
  // the weights over what they are averaged over, and over the draft's temperature
  double f_wtv, f_eal, f_kl, f_tv;
  const float* grad_scale;
};

__device__ __forceinline__ float load_top(const TopLossParams& p, int64_t i) {
  return p.top_bf16 ? Bf16::load1(p.top, i) : F32::load1(p.top, i);
}

// The reference of a draft row's sums: 2^(z sc - msc).
struct RowRef {
  float m, sc, msc;
  bool deep;
};
__device__ __forceinline__ RowRef row_ref(float m, float sc) {
  const bool deep = m * sc < -1e30f && m != kNegInf;
  const float s = deep ? kDeepScale : sc;
  return {m, s, m == kNegInf ? 0.f : m * s, deep};
}
// log2 of q's numerator at a listed entry (exact where a deep row's is huge)
__device__ __forceinline__ float listed_log2(const RowRef& r, float z, float sc) {
  return r.deep ? (z - r.m) * sc : __builtin_fmaf(z, r.sc, -r.msc);
}

// The bitmap of a row's listed ids, one bit per element counted from the row's
// first vector on, so that a vector's bits lie in one byte (or half a byte).
__host__ __device__ constexpr int bitmap_words(int V) { return (V + 7) / 32 + 1; }
template <int E>
__device__ __forceinline__ uint32_t listed_bits(const uint32_t* map, int gi) {
  if constexpr (E == 8) return reinterpret_cast<const uint8_t*>(map)[gi];
  return (reinterpret_cast<const uint8_t*>(map)[gi >> 1] >> (4 * (gi & 1))) & 15u;
}

// What one wave makes of a row's list, its entries' t and z in LDS (t = -inf marks
// one that is no part of it), in three steps: the target alone, the listed draft
// logits against the row's reference, and the sums with the draft's unlisted mass.
struct ListTarget {
  float tmax, inv_zt, lzt;  // p_i = inv_zt 2^((t - tmax) sct); lzt = log2 of that sum's inverse
  float pr, lpr;               // p_r and its log2, which is exact where p_r is denormal
  int star;
  bool has;
};
__device__ ListTarget list_target(const TopLossParams& p, int64_t row, const float* sh_t, const int* sh_id) {
  const int lane = threadIdx.x & (kWave - 1);
  float best = kNegInf;
  int star = INT_MAX;
  for (int i = lane; i < p.k; i += kWave) {
    const float t = sh_t[i];
    if (t == kNegInf) continue;
    const int id = sh_id[i];
    if (t > best || (t == best && id < star)) {
      best = t;
      star = id;
    }
  }
  ListTarget o;
  o.tmax = wave_max(best);
  o.star = wave_min_i(best == o.tmax ? star : INT_MAX);
  const bool any = o.tmax != kNegInf;
  const float rest = p.rest != nullptr ? p.rest[row] : kNegInf;
  o.has = any || rest != kNegInf;
  float st = 0.f;
  for (int i = lane; i < p.k; i += kWave)
    if (sh_t[i] != kNegInf) st += ex2((sh_t[i] - o.tmax) * p.sct);
  st = wave_sum(st);
  // the remainder against the list's largest, in log2: the larger of the two is the reference
  float D = 0.f, f = 1.f, g = 0.f;  // list terms times f, the remainder's g
  if (!any) {
    f = 0.f;
    g = rest != kNegInf ? 1.f : 0.f;
  } else if (rest != kNegInf) {
    D = float(double(rest) * 1.4426950408889634 - double(o.tmax) * double(p.sct));
    f = ex2(-fmaxf(D, 0.f));
    g = ex2(fminf(D, 0.f));
  }
  const float zt = __builtin_fmaf(st, f, g);
  o.inv_zt = o.has ? f / zt : 0.f;
  o.lzt = o.has ? -__log2f(zt) - fmaxf(D, 0.f) : 0.f;
  o.pr = o.has ? g / zt : 0.f;
  o.lpr = o.has ? fminf(D, 0.f) - __log2f(zt) : 0.f;
  return o;
}
__device__ __forceinline__ float list_draft(const TopLossParams& p, const float* sh_t, const float* sh_z, RowRef ref) {
  float sz = 0.f;
  for (int i = threadIdx.x & (kWave - 1); i < p.k; i += kWave)
    if (sh_t[i] != kNegInf) sz += ex2(listed_log2(ref, sh_z[i], p.scd));
  return wave_sum(sz);
}
__device__ TopRow list_row(const TopLossParams& p, const ListTarget& o, const float* sh_t, const float* sh_z,
                           const int* sh_id, RowRef ref, float sz, float su) {
  const float zd = sz + su, inv_s = zd > 0.f ? 1.f / zd : 0.f;
  // log2 of the sums' ratio (a draft row without a finite entry has q = 0 everywhere)
  const float dl = (zd > 0.f ? __log2f(zd) : 0.f) + o.lzt;
  const float qr = p.rest != nullptr ? su * inv_s : 0.f;
  float v[4] = {0.f, 0.f, 0.f, 0.f};  // sums of min(p, q), q where q < p, p log2(p / q), q at x*
  for (int i = threadIdx.x & (kWave - 1); i < p.k; i += kWave) {
    const float t = sh_t[i];
    if (t == kNegInf) continue;
    const float lt = (t - o.tmax) * p.sct, lz = listed_log2(ref, sh_z[i], p.scd);
    const float pv = ex2(lt) * o.inv_zt, qv = ex2(lz) * inv_s;
    v[0] += fminf(pv, qv);
    v[1] += qv < pv ? qv : 0.f;
    v[2] += pv > 0.f ? pv * ((lt - lz) + dl) : 0.f;
    v[3] += sh_id[i] == o.star ? qv : 0.f;
  }
  wave_sum_n(v);
  TopRow r{};
  r.msc = ref.msc;
  r.inv_s = inv_s;
  r.tmax = o.tmax;
  r.inv_zt = o.inv_zt;
  r.a_tv = v[0] + fminf(o.pr, qr);
  r.a_eal = v[3];
  const bool below = qr < o.pr;
  r.qlt = v[1] + (below ? qr : 0.f);
  r.kl = (v[2] + (o.pr > 0.f ? o.pr * (o.lpr - __log2f(qr)) : 0.f)) * kLn2;
  r.share = qr > 0.f ? o.pr / qr : 0.f;
  r.xstar = o.star == INT_MAX ? -1 : o.star;
  r.flags = (o.has ? kTopHas : 0) | (below ? kTopRestBelow : 0) | (ref.deep ? kTopDeep : 0);
  return r;
}

// p and the gradient at a listed entry.
__device__ __forceinline__ float listed_p(const TopRow& s, float t, float sct) {
  return ex2((t - s.tmax) * sct) * s.inv_zt;
}
__device__ __forceinline__ float listed_grad(const TopRow& s, float q, float pv, int id) {
  float g = q * (q < pv ? s.cA : s.cB) - s.cP * pv;
  if (id == s.xstar) g += s.cX;
  return g;
}

// The windows that contain row r: starts t0..t1 (none if t1 < t0), the first
// row of its sequence, and its place s there.
struct RowWindows {
  int64_t base, own;  // own: the window that starts at r, where `starts`
  int s, t0, t1;
  bool starts;
};
__device__ __forceinline__ RowWindows row_windows(int64_t r, int layout, int S, int K) {
  RowWindows w;
  if (layout == 0) {
    w.own = r / K;
    w.base = w.own * K;
    w.s = int(r - w.base);
    w.t0 = w.t1 = 0;
    w.starts = w.s == 0;
  } else {
    const int64_t b = r / S;
    w.base = b * S;
    w.s = int(r - w.base);
    w.t0 = max(0, w.s - K + 1);
    w.t1 = min(w.s, S - K);
    w.own = b * int64_t(max(0, S - K + 1)) + w.s;
    w.starts = w.s <= S - K;
  }
  return w;
}
__device__ __forceinline__ double windows_of(const RowWindows& w) { return w.t1 >= w.t0 ? double(w.t1 - w.t0 + 1) : 0.0; }

// dE/da at place j of a window whose rows' acceptances are a[0..K-1].
template <class F>
__device__ __forceinline__ double window_d(F a, int K, int j) {
  double P = 1.0, S = 1.0;
  for (int i = 0; i < j; ++i) P *= double(a(i));
  for (int i = K - 1; i > j; --i) S = 1.0 + double(a(i)) * S;
  return P * S;
}

// The coefficients of a row from dE/da summed over its windows.
__device__ __forceinline__ void row_coefs(TopRow& o, const TopLossParams& p, double d_tv, double d_eal, double count) {
  const double f = p.grad_scale ? double(*p.grad_scale) : 1.0;
  const double c_tv = -f * (p.f_wtv * d_tv + p.f_tv * count);
  const double c_eal = -f * p.f_eal * d_eal * double(o.a_eal);
  const double c_kl = (o.flags & kTopHas) ? f * p.f_kl : 0.0;
  const double q_lt = double(o.qlt);
  o.cR = float((c_tv * (((o.flags & kTopRestBelow) ? 1.0 : 0.0) - q_lt) - c_eal + c_kl * (1.0 - double(o.share))) *
               double(o.inv_s));
  o.cA = float(c_tv * (1.0 - q_lt) - c_eal + c_kl);
  o.cB = float(-c_tv * q_lt - c_eal + c_kl);
  o.cP = float(c_kl);
  o.cX = float(c_eal);
}

// What a row leaves for the caller and for the sums of the loss.
__device__ __forceinline__ void write_row(const TopLossParams& p, int64_t r, const TopRow& o, double count) {
  p.row_loss[r] = make_float2(o.kl, float(count * (1.0 - double(o.a_tv))));
  if (p.accept_tv) p.accept_tv[r] = o.a_tv;
  if (p.accept_eal) p.accept_eal[r] = o.a_eal;
  if (p.xstar) p.xstar[r] = o.xstar;
}

inline TopLossParams params_of(const TopLossArgs& a) {
  TopLossParams p{};
  p.zd = a.zd;
  p.top = a.top;
  p.ids = a.ids;
  p.rest = a.rest;
  p.R = a.R;
  p.V = a.V;
  p.k = a.k;
  p.scd = a.sc_d;
  p.sct = a.sc_t;
  p.top_bf16 = a.td == DType::kBf16;
  p.stats = a.stats;
  p.slots = a.slots;
  p.row_loss = a.row_loss;
  p.err = a.err;
  p.counter = a.err + 1;
  p.accept_tv = a.accept_tv;
  p.accept_eal = a.accept_eal;
  p.xstar = a.xstar;
  p.layout = a.layout;
  p.S = a.S;
  p.K = a.K;
  p.W = a.W;
  p.w_wtv = a.w_wtv;
  p.w_eal = a.w_eal;
  p.w_kl = a.w_kl;
  p.w_tv = a.w_tv;
  const double inv_w = a.W > 0 ? double(a.inv_t_d) / double(a.W) : 0.0;
  p.f_wtv = double(a.w_wtv) * inv_w;
  p.f_eal = double(a.w_eal) * inv_w;
  p.f_kl = double(a.w_kl) * double(a.inv_t_d) / double(a.R);
  p.f_tv = double(a.w_tv) * inv_w / a.K;
  p.grad_scale = a.grad_scale;
  return p;
}

}  // namespace
}  // namespace aal
