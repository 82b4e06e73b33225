// The training objectives against a target's top logits (aal_topk_loss_fwd_bwd).
//
// The target of a row is a list of k logits and a remainder, the log-sum-exp of
// all other entries, which counts as one more entry that the draft's mass
// outside the list is compared with:
//   p_i = exp(t_i / T_t) / Z, p_r = exp(rest) / Z;   q_i = q(id_i), q_r = sum of q outside the list
//   a_tv = sum_i min(p_i, q_i) + min(p_r, q_r),  KL = sum_i p_i ln(p_i / q_i) + p_r ln(p_r / q_r)
// All unlisted entries share one indicator m_r = [q_r < p_r] and one ratio
// p_r / q_r, so that with c_* the row's dloss/da (KL: dloss/dKL) over T_d
//   dloss/dz_v = q_v (c_tv (m_r - Q) - c_eal + c_kl (1 - p_r / q_r))         unlisted: q_v times a constant
//   dloss/dz_i = q_i (c_tv (m_i - Q) - c_eal + c_kl) - c_kl p_i + c_eal [i = x*]   listed
// with Q = sum of q over the entries with q < p (the remainder among them).
//
// Multi-kernel schedule, every shape:
//   k_top_rows  one workgroup per row: the draft's max / sum-exp over the
//               unlisted entries (a bitmap of the list in LDS keeps the listed
//               ones out, so that q_r is a sum and not a difference), then the
//               first wave does the list.
//   k_top_scan  one thread per row: dE/da over the windows that contain it and
//               the row's coefficients; the row that starts a window writes its E.
//   k_top_loss  the four terms and the weighted loss, fixed summation order.
//   k_top_grad  one constant times 2^x for every entry, then the listed ones.
#include "aal_device.h"
#include "aal_rowops.h"
#include "aal_toplist.h"

#include <limits.h>

namespace aal {
namespace {

constexpr int kTopMax = 512;
constexpr float kLn2 = 0.693147180559945309417f;
constexpr float kLog2e = 1.44269504088896340736f;

struct TopLossParams {
  const void* zd;
  const void* top;
  const int32_t* ids;
  const float* rest;
  int64_t R;
  int V, k;
  float scd, sct;
  int top_bf16;
  TopRow* stats;
};

__device__ __forceinline__ float load_top(const TopLossParams& p, int64_t i) {
  return p.top_bf16 ? Bf16::load1(p.top, i) : F32::load1(p.top, i);
}

// The bitmap of a row's listed ids, one bit per element counted from the row's
// first vector on, so that a vector's bits lie in one byte (or half a byte).
__device__ __forceinline__ int bitmap_words(int V) { return (V + 7) / 32 + 1; }
template <int E>
__device__ __forceinline__ uint32_t listed_bits(const uint32_t* map, int gi) {
  if constexpr (E == 8) return reinterpret_cast<const uint8_t*>(map)[gi];
  return (reinterpret_cast<const uint8_t*>(map)[gi >> 1] >> (4 * (gi & 1))) & 15u;
}

// What the first wave makes of a row's list: t and z of its entries in LDS
// (t = -inf marks one that is no part of the list), the draft's state over
// the unlisted entries in `un`.
__device__ TopRow list_row(const TopLossParams& p, int64_t row, const float* sh_t, const float* sh_z, LseState un) {
  const int lane = threadIdx.x & (kWave - 1);
  const bool has_rest = p.rest != nullptr;
  float tmax = kNegInf, zmax = kNegInf, best = kNegInf;
  int star = INT_MAX;
  for (int i = lane; i < p.k; i += kWave) {
    const float t = sh_t[i];
    if (t == kNegInf) continue;
    tmax = fmaxf(tmax, t);
    zmax = fmaxf(zmax, sh_z[i]);
    const int id = p.ids[row * p.k + i];
    if (t > best || (t == best && id < star)) {
      best = t;
      star = id;
    }
  }
  tmax = wave_max(tmax);
  zmax = wave_max(zmax);
  star = wave_min_i(best == tmax ? star : INT_MAX);
  const float rest2 = has_rest ? p.rest[row] * kLog2e : kNegInf;
  const float tm = tmax == kNegInf ? kNegInf : tmax * p.sct;
  float mt = fmaxf(tm, rest2);
  const bool has = mt != kNegInf;
  if (!has) mt = 0.f;
  float zm = fmaxf(zmax, un.m);
  const float msc = zm == kNegInf ? 0.f : zm * p.scd;
  float st = 0.f, sz = 0.f;
  for (int i = lane; i < p.k; i += kWave) {
    const float t = sh_t[i];
    if (t == kNegInf) continue;
    st += ex2(__builtin_fmaf(t, p.sct, -mt));
    sz += ex2(__builtin_fmaf(sh_z[i], p.scd, -msc));
  }
  st = wave_sum(st);
  sz = wave_sum(sz);
  const float er = ex2(rest2 - mt);
  const float su = un.m == kNegInf ? 0.f : un.s * ex2(un.msc - msc);
  const float zt = st + er, zd = sz + su;
  const float inv_zt = has ? 1.f / zt : 0.f, inv_s = zd > 0.f ? 1.f / zd : 0.f;
  // log2 of the sums' ratio (a draft row without a finite entry has q = 0 everywhere)
  const float dl = (zd > 0.f ? __log2f(zd) : 0.f) - (has ? __log2f(zt) : 0.f);
  const float pr = er * inv_zt, qr = has_rest ? su * inv_s : 0.f;
  float a = 0.f, q_lt = 0.f, kl = 0.f, ae = 0.f;
  for (int i = lane; i < p.k; i += kWave) {
    const float t = sh_t[i];
    if (t == kNegInf) continue;
    const float lt = __builtin_fmaf(t, p.sct, -mt), lz = __builtin_fmaf(sh_z[i], p.scd, -msc);
    const float pv = ex2(lt) * inv_zt, qv = ex2(lz) * inv_s;
    a += fminf(pv, qv);
    q_lt += qv < pv ? qv : 0.f;
    kl += pv > 0.f ? pv * ((lt - lz) + dl) : 0.f;
    ae += p.ids[row * p.k + i] == star ? qv : 0.f;
  }
  a = wave_sum(a);
  q_lt = wave_sum(q_lt);
  kl = wave_sum(kl);
  ae = wave_sum(ae);
  TopRow o{};
  o.msc = msc;
  o.inv_s = inv_s;
  o.mt = mt;
  o.inv_zt = inv_zt;
  o.a_tv = a + fminf(pr, qr);
  o.a_eal = ae;
  const bool below = qr < pr;
  o.qlt = q_lt + (below ? qr : 0.f);
  if (pr > 0.f) kl += pr * (__log2f(pr) - __log2f(qr));
  o.kl = kl * kLn2;
  o.share = qr > 0.f ? pr / qr : 0.f;
  o.xstar = star == INT_MAX ? -1 : star;
  o.flags = (has ? kTopHas : 0) | (below ? kTopRestBelow : 0);
  return o;
}

template <class TI, bool VEC, int U, int BLK>
__global__ __launch_bounds__(BLK) void k_top_rows(TopLossParams p) {
  using Rv = RowVecs<TI, VEC>;
  constexpr int E = Rv::E;
  extern __shared__ uint32_t sh_map[];
  __shared__ float sh_t[kTopMax], sh_z[kTopMax];
  __shared__ LseState sh_lse[BLK / kWave];

  const int64_t row = blockIdx.x;
  const Rv rv(row, p.R, p.V);
  const int64_t e0 = row * int64_t(p.V), l0 = row * p.k;
  const int words = bitmap_words(p.V);
  for (int i = threadIdx.x; i < words; i += BLK) sh_map[i] = 0;
  __syncthreads();
  for (int i = threadIdx.x; i < p.k; i += BLK) {
    const int id = p.ids[l0 + i];
    const float t = load_top(p, l0 + i);
    const bool in = id >= 0 && id < p.V && t != kNegInf;
    sh_t[i] = in ? t : kNegInf;
    sh_z[i] = in ? TI::load1(p.zd, e0 + id) : kNegInf;
    if (in) atomicOr(&sh_map[(id + rv.head) >> 5], 1u << ((id + rv.head) & 31));
  }
  __syncthreads();
  LseState un = lse_init();
  for (int base = threadIdx.x; base < rv.ng; base += BLK * U) {
    u32x4 w[1][U];
    float x[U][E];
    rv.load({p.zd}, base, BLK, w);
    rv.unpack(w[0], x);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int gi = base + u * BLK;
      const uint32_t bits = gi < rv.ng ? listed_bits<E>(sh_map, gi) : 0u;
      if (bits)
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (bits >> e & 1u) x[u][e] = kNegInf;
    }
    lse_fold(un, x, p.scd);
  }
  un = block_lse<BLK / kWave>(un, p.scd, sh_lse);
  if (threadIdx.x < kWave) {
    const TopRow o = list_row(p, row, sh_t, sh_z, un);
    if (threadIdx.x == 0) p.stats[row] = o;
  }
}

struct TopScanParams {
  TopRow* stats;
  int layout;
  int64_t B;
  int S, K;
  int64_t R, W;
  float w_wtv, w_eal, w_kl, w_tv;
  float inv_t_d;
  const float* grad_scale;
  float2* win;
  float2* row_loss;
  float* e_tv;
  float* e_eal;
  float* accept_tv;
  float* accept_eal;
  int32_t* xstar;
};

// The windows that contain row r: starts t0..t1 (none if t1 < t0), the first
// row of its sequence, its place s there, and the index of its own window.
struct RowWindows {
  int64_t base, own;
  int s, t0, t1;
  bool starts;
};
__device__ __forceinline__ RowWindows row_windows(int64_t r, int layout, int S, int K) {
  RowWindows w;
  if (layout == 0) {
    w.base = (r / K) * K;
    w.s = int(r - w.base);
    w.t0 = w.t1 = 0;
    w.own = r / K;
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

// The coefficients of a row from dE/da summed over its windows.
__device__ void row_coefs(TopRow& o, const TopScanParams& p, double d_tv, double d_eal, double count) {
  const double f = (p.grad_scale ? double(*p.grad_scale) : 1.0) * double(p.inv_t_d);
  const double W = double(p.W);
  const double c_tv = p.W > 0 ? f * (-double(p.w_wtv) * d_tv - double(p.w_tv) * count / p.K) / W : 0.0;
  const double c_eal = p.W > 0 ? -f * double(p.w_eal) * d_eal / W * double(o.a_eal) : 0.0;
  const double c_kl = (o.flags & kTopHas) ? f * double(p.w_kl) / double(p.R) : 0.0;
  const double q_lt = double(o.qlt);
  o.cR = float((c_tv * (((o.flags & kTopRestBelow) ? 1.0 : 0.0) - q_lt) - c_eal + c_kl * (1.0 - double(o.share))) *
               double(o.inv_s));
  o.cA = float(c_tv * (1.0 - q_lt) - c_eal + c_kl);
  o.cB = float(-c_tv * q_lt - c_eal + c_kl);
  o.cP = float(c_kl);
  o.cX = float(c_eal);
}

__global__ __launch_bounds__(kRowBlock) void k_top_scan(TopScanParams p) {
  const int64_t r = int64_t(blockIdx.x) * kRowBlock + threadIdx.x;
  if (r >= p.R) return;
  const int K = p.K;
  const RowWindows rw = row_windows(r, p.layout, p.S, K);
  const TopRow* st = p.stats + rw.base;
  double d_tv = 0.0, d_eal = 0.0;
  for (int t = rw.t0; t <= rw.t1; ++t) {
    const int j = rw.s - t;
    double Pt = 1.0, Pe = 1.0, St = 1.0, Se = 1.0;
    for (int i = 0; i < j; ++i) {
      Pt *= double(st[t + i].a_tv);
      Pe *= double(st[t + i].a_eal);
    }
    for (int i = K - 1; i > j; --i) {
      St = 1.0 + double(st[t + i].a_tv) * St;
      Se = 1.0 + double(st[t + i].a_eal) * Se;
    }
    d_tv += Pt * St;
    d_eal += Pe * Se;
  }
  const double count = double(rw.t1 - rw.t0 + 1 > 0 ? rw.t1 - rw.t0 + 1 : 0);
  TopRow o = p.stats[r];
  row_coefs(o, p, d_tv, d_eal, count);
  TopRow& out = p.stats[r];
  out.cR = o.cR;
  out.cA = o.cA;
  out.cB = o.cB;
  out.cP = o.cP;
  out.cX = o.cX;
  p.row_loss[r] = make_float2(o.kl, float(count * (1.0 - double(o.a_tv))));
  if (p.accept_tv) p.accept_tv[r] = o.a_tv;
  if (p.accept_eal) p.accept_eal[r] = o.a_eal;
  if (p.xstar) p.xstar[r] = o.xstar;
  if (rw.starts) {
    double Pt = 1.0, Pe = 1.0, Et = 0.0, Ee = 0.0;
    for (int i = 0; i < K; ++i) {
      Pt *= double(st[rw.s + i].a_tv);
      Pe *= double(st[rw.s + i].a_eal);
      Et += Pt;
      Ee += Pe;
    }
    p.win[rw.own] = make_float2(float(Et), float(Ee));
    if (p.e_tv) p.e_tv[rw.own] = float(Et);
    if (p.e_eal) p.e_eal[rw.own] = float(Ee);
  }
}

constexpr int kLossBlock = 1024;

__device__ double block_sum_d(double v, double* sh) {
  v = wave_sum_d(v);
  if ((threadIdx.x & (kWave - 1)) == 0) sh[threadIdx.x / kWave] = v;
  __syncthreads();
  double t = 0.0;
  for (int i = 0; i < kLossBlock / kWave; ++i) t += sh[i];
  __syncthreads();
  return t;
}

struct TopLossSum {
  const float2* win;
  const float2* row_loss;
  int64_t R, W;
  int K;
  float w_wtv, w_eal, w_kl, w_tv;
  double* parts;
  float* loss;
  float* terms;
  const unsigned* err;  // the resident schedule's error word, or null
};

__device__ void write_loss(const TopLossSum& p, double etv, double eeal, double kl, double tvs) {
  // a term whose weight is 0 reads 0
  const double t0 = p.W > 0 && p.w_wtv != 0.f ? -etv / double(p.W) : 0.0;
  const double t1 = p.W > 0 && p.w_eal != 0.f ? -eeal / double(p.W) : 0.0;
  const double t2 = p.w_kl != 0.f ? kl / double(p.R) : 0.0;
  const double t3 = p.W > 0 && p.w_tv != 0.f ? tvs / (double(p.W) * p.K) : 0.0;
  p.loss[0] = (p.err != nullptr && *p.err != 0u) ? __builtin_nanf("")
                                                 : float(double(p.w_wtv) * t0 + double(p.w_eal) * t1 +
                                                         double(p.w_kl) * t2 + double(p.w_tv) * t3);
  if (p.terms) {
    p.terms[0] = float(t0);
    p.terms[1] = float(t1);
    p.terms[2] = float(t2);
    p.terms[3] = float(t3);
  }
}

// Block b of n sums the windows and rows of its contiguous slice; a lone block
// writes the loss itself.
__global__ __launch_bounds__(kLossBlock) void k_top_loss_parts(TopLossSum p, int n) {
  __shared__ double sh[kLossBlock / kWave];
  const int64_t b = blockIdx.x;
  const int64_t w0 = p.W * b / n, w1 = p.W * (b + 1) / n, r0 = p.R * b / n, r1 = p.R * (b + 1) / n;
  double etv = 0.0, eeal = 0.0, kl = 0.0, tvs = 0.0;
  for (int64_t i = w0 + threadIdx.x; i < w1; i += kLossBlock) {
    const float2 e = p.win[i];
    etv += double(e.x);
    eeal += double(e.y);
  }
  for (int64_t i = r0 + threadIdx.x; i < r1; i += kLossBlock) {
    const float2 e = p.row_loss[i];
    kl += double(e.x);
    tvs += double(e.y);
  }
  etv = block_sum_d(etv, sh);
  eeal = block_sum_d(eeal, sh);
  kl = block_sum_d(kl, sh);
  tvs = block_sum_d(tvs, sh);
  if (threadIdx.x != 0) return;
  if (n == 1) {
    write_loss(p, etv, eeal, kl, tvs);
  } else {
    double* o = p.parts + b * 4;
    o[0] = etv;
    o[1] = eeal;
    o[2] = kl;
    o[3] = tvs;
  }
}
__global__ void k_top_loss(TopLossSum p, int n) {
  if (threadIdx.x != 0) return;
  double s[4] = {0.0, 0.0, 0.0, 0.0};
  for (int b = 0; b < n; ++b)
    for (int i = 0; i < 4; ++i) s[i] += p.parts[b * 4 + i];
  write_loss(p, s[0], s[1], s[2], s[3]);
}

// The gradient at list entry i of a row: q_i and p_i again from the logits.
template <class TI>
__device__ __forceinline__ float listed_grad(const TopRow& s, float t, float z, int id, float scd, float sct) {
  const float q = ex2(__builtin_fmaf(z, scd, -s.msc)) * s.inv_s;
  const float pv = ex2(__builtin_fmaf(t, sct, -s.mt)) * s.inv_zt;
  float g = q * (q < pv ? s.cA : s.cB) - s.cP * pv;
  if (id == s.xstar) g += s.cX;
  return g;
}

template <class TI, class TG, bool VEC, int U>
__global__ __launch_bounds__(kRowBlock) void k_top_grad(TopLossParams p, int splits, void* __restrict__ grad) {
  using Rv = RowVecs<TI, VEC>;
  constexpr int E = Rv::E;
  const int64_t row = blockIdx.x;
  const Rv rv(row, p.R, p.V);
  const TopRow s = p.stats[row];
  const int64_t e0 = row * int64_t(p.V), l0 = row * p.k;
  for (int base = blockIdx.y * kRowBlock * U + threadIdx.x; base < rv.ng; base += splits * kRowBlock * U) {
    u32x4 w[1][U];
    rv.load({p.zd}, base, kRowBlock, w);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int gi = base + u * kRowBlock;
      if (gi >= rv.ng) break;
      float x[E], g[E];
      TI::unpack(to_uint4(w[0][u]), x);
#pragma unroll
      for (int e = 0; e < E; ++e) g[e] = s.cR * ex2(__builtin_fmaf(x[e], p.scd, -s.msc));
      rv.template store<TG>(grad, gi, g);
    }
  }
  // the listed entries of this workgroup's vectors, over what was stored there
  __syncthreads();
  for (int i = threadIdx.x; i < p.k; i += kRowBlock) {
    const int id = p.ids[l0 + i];
    if (id < 0 || id >= p.V) continue;
    if (((id + rv.head) / E / (kRowBlock * U)) % splits != int(blockIdx.y)) continue;
    const float t = load_top(p, l0 + i);
    if (t == kNegInf) continue;
    TG::store1(grad, e0 + id, listed_grad<TI>(s, t, TI::load1(p.zd, e0 + id), id, p.scd, p.sct));
  }
}

TopLossParams params_of(const TopLossArgs& a) {
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
  return p;
}

TopScanParams scan_of(const TopLossArgs& a) {
  TopScanParams p{};
  p.stats = a.stats;
  p.layout = a.layout;
  p.B = a.B;
  p.S = a.S;
  p.K = a.K;
  p.R = a.R;
  p.W = a.W;
  p.w_wtv = a.w_wtv;
  p.w_eal = a.w_eal;
  p.w_kl = a.w_kl;
  p.w_tv = a.w_tv;
  p.inv_t_d = a.inv_t_d;
  p.grad_scale = a.grad_scale;
  p.win = a.win;
  p.row_loss = a.row_loss;
  p.e_tv = a.e_tv;
  p.e_eal = a.e_eal;
  p.accept_tv = a.accept_tv;
  p.accept_eal = a.accept_eal;
  p.xstar = a.xstar;
  return p;
}

hipError_t loss_launch(const TopLossArgs& a, const unsigned* err) {
  TopLossSum p{};
  p.win = a.win;
  p.row_loss = a.row_loss;
  p.R = a.R;
  p.W = a.W;
  p.K = a.K;
  p.w_wtv = a.w_wtv;
  p.w_eal = a.w_eal;
  p.w_kl = a.w_kl;
  p.w_tv = a.w_tv;
  p.parts = a.loss_parts;
  p.loss = a.loss;
  p.terms = a.terms;
  p.err = err;
  const int n = a.R <= 32 * kLossBlock ? 1 : kTopLossParts;
  k_top_loss_parts<<<dim3(unsigned(n)), kLossBlock, 0, a.stream>>>(p, n);
  if (n > 1) k_top_loss<<<1, kWave, 0, a.stream>>>(p, n);
  return hipGetLastError();
}

template <class TI, class TG, bool VEC>
void grad_launch(const TopLossArgs& a) {
  with_grad_shape(a.V, TI::kVec, [&](auto sh) {
    constexpr int U = decltype(sh)::kU;
    const unsigned splits = row_splits(a.R, a.V, TI::kVec, U);
    k_top_grad<TI, TG, VEC, U><<<dim3(unsigned(a.R), splits), kRowBlock, 0, a.stream>>>(params_of(a), int(splits),
                                                                                      a.grad);
  });
}

template <class TI, bool VEC>
hipError_t launch_vec(const TopLossArgs& a) {
  const size_t map = size_t((a.V + 7) / 32 + 1) * 4;
  hipError_t e = hipSuccess;
  with_row_shape<4>(a.R, a.V, TI::kVec, [&](auto sh) {
    using Sh = decltype(sh);
    k_top_rows<TI, VEC, Sh::kU, Sh::kBlock><<<dim3(unsigned(a.R)), Sh::kBlock, map, a.stream>>>(params_of(a));
    e = hipGetLastError();
  });
  if (e != hipSuccess) return e;
  k_top_scan<<<dim3(unsigned((a.R + kRowBlock - 1) / kRowBlock)), kRowBlock, 0, a.stream>>>(scan_of(a));
  if ((e = loss_launch(a, nullptr)) != hipSuccess) return e;
  if (a.grad) a.gd == DType::kBf16 ? grad_launch<TI, GBf16, VEC>(a) : grad_launch<TI, GF32, VEC>(a);
  return hipGetLastError();
}

template <class TI>
hipError_t launch_typed(const TopLossArgs& a) {
  return a.V % TI::kVec == 0 ? launch_vec<TI, true>(a) : launch_vec<TI, false>(a);
}

}  // namespace

hipError_t launch_top_loss(const TopLossArgs& a) {
  return a.in == DType::kBf16 ? launch_typed<Bf16>(a) : launch_typed<F32>(a);
}

}  // namespace aal
