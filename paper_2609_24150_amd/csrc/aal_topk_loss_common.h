// What the two schedules of the objectives against top lists share: the list of a
// row, its windows and its coefficients (the mathematics is stated in
// aal_topk_loss.hip).
#pragma once

#include "aal_device.h"
#include "aal_resident_common.h"
#include "aal_row_ref.h"
#include "aal_rowops.h"
#include "aal_toplist.h"

#include <limits.h>

namespace aal {
namespace {

constexpr int kTopMax = 512;
constexpr float kLn2 = 0.693147180559945309417f;

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

// The bitmap of a row's listed ids, one bit per element counted from the row's
// first vector on, so that a vector's bits lie in one byte (or half a byte).
__host__ __device__ constexpr int bitmap_words(int V) { return (V + 7) / 32 + 1; }
template <int E>
__device__ __forceinline__ uint32_t listed_bits(const uint32_t* map, int gi) {
  if constexpr (E == 8) return reinterpret_cast<const uint8_t*>(map)[gi];
  return (reinterpret_cast<const uint8_t*>(map)[gi >> 1] >> (4 * (gi & 1))) & 15u;
}

// What one wave makes of a row's list, its entries' t and z in LDS (t = -inf marks
// one that is no part of it), in three steps: the target alone, the draft's listed
// logits alone, and both with the draft's unlisted mass.  List and remainder have a reference and a
// sum each, on the target's side and on the draft's, so that neither vanishes however far it lies
// below the other; they are joined through the log2 of one reference over the other.
struct Join {
  float f, g, up, dn;  // what takes values of the list and of the remainder to the larger reference, and -log2 of f, log2 of g
};
__device__ __forceinline__ Join join(float D) {
  const float up = fmaxf(D, 0.f), dn = fminf(D, 0.f);
  return {ex2(-up), ex2(dn), up, dn};
}
struct ListTarget {
  float tmax, inv_zt;  // p_i = inv_zt 2^((t - tmax) sct)
  float pr;
  float iz, up, dn;    // log2 p_i = (t - tmax) sct + log2 iz - up, log2 p_r = log2 iz + dn
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
  // the remainder, one entry, against the list's largest
  Join j = join(any && rest != kNegInf ? float(double(rest) * 1.4426950408889634 - double(o.tmax) * double(p.sct)) : 0.f);
  if (!any) j.f = 0.f;
  if (rest == kNegInf) j.g = 0.f;
  const float zt = __builtin_fmaf(st, j.f, j.g);
  o.iz = o.has ? 1.f / zt : 0.f;
  o.inv_zt = j.f * o.iz;
  o.pr = j.g * o.iz;
  o.up = j.up;
  o.dn = j.dn;
  return o;
}
struct ListDraft {
  RowRef ref;
  float s;
};
__device__ __forceinline__ ListDraft list_draft(const TopLossParams& p, const float* sh_t, const float* sh_z) {
  const int lane = threadIdx.x & (kWave - 1);
  float m = kNegInf, s = 0.f;
  for (int i = lane; i < p.k; i += kWave)
    if (sh_t[i] != kNegInf) m = fmaxf(m, sh_z[i]);
  const RowRef ref = row_ref(wave_max(m), p.scd);
  for (int i = lane; i < p.k; i += kWave)
    if (sh_t[i] != kNegInf) s += ex2(log2_of(ref, sh_z[i]));
  return {ref, wave_sum(s)};
}
// u, su: the unlisted entries' reference and their sum against it.
__device__ TopRow list_row(const TopLossParams& p, const ListTarget& o, const float* sh_t, const float* sh_z,
                           const int* sh_id, const ListDraft& l, const RowRef& u, float su) {
  float D = u.steep || l.ref.steep ? (u.m - l.ref.m) * p.scd : u.msc - l.ref.msc;
  if (u.m == kNegInf) D = l.ref.m == kNegInf ? 0.f : kNegInf;
  else if (l.ref.m == kNegInf) D = -kNegInf;
  const Join j = join(D);
  const float zd = l.s * j.f + su * j.g, iz = zd > 0.f ? 1.f / zd : 0.f;  // 0: a draft row without a finite entry
  const float ql = j.f * iz, qu = j.g * iz, qr = p.rest != nullptr ? su * qu : 0.f;
  // log2 p - log2 q of a listed entry is (lt - lz) + dl, of the remainder lr: one logarithm each, of sums
  const float zz = zd * o.iz;
  const float dl = (zz > 0.f ? __log2f(zz) : 0.f) + (j.up - o.up);
  const float lr = su > 0.f ? __log2f(zz / su) + (o.dn - j.dn) : -kNegInf;
  float v[4] = {0.f, 0.f, 0.f, 0.f};  // sums of min(p, q), q where q < p, p log2(p / q), q at x*
  for (int i = threadIdx.x & (kWave - 1); i < p.k; i += kWave) {
    const float t = sh_t[i];
    if (t == kNegInf) continue;
    const float lt = (t - o.tmax) * p.sct, lz = log2_of(l.ref, sh_z[i]);
    const float pv = ex2(lt) * o.inv_zt, qv = ex2(lz) * ql;
    v[0] += fminf(pv, qv);
    v[1] += qv < pv ? qv : 0.f;
    v[2] += pv > 0.f ? pv * ((lt - lz) + dl) : 0.f;
    v[3] += sh_id[i] == o.star ? qv : 0.f;
  }
  wave_sum_n(v);
  TopRow r{};
  r.mu = u.m;
  r.ml = l.ref.m;
  r.qu = qu;
  r.ql = ql;
  r.tmax = o.tmax;
  r.inv_zt = o.inv_zt;
  r.a_tv = v[0] + fminf(o.pr, qr);
  r.a_eal = v[3];
  const bool below = qr < o.pr;
  r.qlt = v[1] + (below ? qr : 0.f);
  r.kl = (v[2] + (o.pr > 0.f ? o.pr * lr : 0.f)) * kLn2;
  r.pu = su > 0.f ? o.pr / su : 0.f;
  r.xstar = o.star == INT_MAX ? -1 : o.star;
  r.flags = (o.has ? kTopHas : 0) | (below ? kTopRestBelow : 0);
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
  // (p_r q_v / q_r of the KL term as p_r over the unlisted sum: q_r may be 0 in fp32)
  o.cR = float((c_tv * (((o.flags & kTopRestBelow) ? 1.0 : 0.0) - q_lt) - c_eal + c_kl) * double(o.qu) -
               c_kl * double(o.pu));
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
