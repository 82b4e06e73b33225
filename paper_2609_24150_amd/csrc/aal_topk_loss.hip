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
// Resident schedule (k_top_fused): a workgroup keeps a row in registers from
// its one read to the one write of its gradient, and takes row after row, loading the
// next one's vectors as it stores this one's.  Where a coefficient depends on the row's
// windows (WTV or EAL terms), it publishes the row's acceptances and waits for
// those of the at most K - 1 rows on either side: all workgroups of the grid
// run at once and take rows in order, and publishing waits for nothing, so the waits
// end; they are bounded all the same.
// Multi-kernel schedule, every shape (rows too long for a workgroup's registers):
//   k_top_rows  one workgroup per row: the draft's max / sum-exp over the
//               unlisted entries, then the first wave does the list.
//   k_top_scan  one thread per row: dE/da over the windows that contain it and
//               the row's coefficients.
//   k_top_grad  one constant times 2^x for every entry, then the listed ones.
// Both end with k_top_loss: every window's E, the four terms and the weighted
// loss, in a fixed order of summation.
//
// The listed entries are kept out of the unlisted sum by a bitmap of the
// vocabulary in LDS, so that q_r is a sum and not a difference.  A row whose largest logit
// is below -1e30 / sc ("deep": filled with the type's lowest value) has entries that are
// equal or further apart than any exponential holds: 2^-64 takes the place of sc
// there, so that the products stay finite.
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
  float inv_t_d;
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
  float tmax, D, inv_zt, lzt, pr;  // p_i = inv_zt 2^((t - tmax) sct); lzt = log2 of that sum's inverse
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
  r.kl = (v[2] + (o.pr > 0.f ? o.pr * (__log2f(o.pr) - __log2f(qr)) : 0.f)) * kLn2;
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
__device__ void row_coefs(TopRow& o, const TopLossParams& p, double d_tv, double d_eal, double count) {
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

// What a row leaves for the caller and for the sums of the loss.
__device__ __forceinline__ void write_row(const TopLossParams& p, int64_t r, const TopRow& o, double count) {
  p.row_loss[r] = make_float2(o.kl, float(count * (1.0 - double(o.a_tv))));
  if (p.accept_tv) p.accept_tv[r] = o.a_tv;
  if (p.accept_eal) p.accept_eal[r] = o.a_eal;
  if (p.xstar) p.xstar[r] = o.xstar;
}

// ------------------------------------------------------- resident schedule
// The bitmap reaches to the end of the last vectors that a workgroup holds.
constexpr int stage_words(int held) { return (bitmap_words(held) + 3) & ~3; }  // before the staging buffer
inline size_t fused_lds_bytes(int held, int staged, int k) {
  return size_t(stage_words(held)) * 4 + size_t(staged) * 16 + size_t(k) * 20;
}

// WK waves hold the row, NV vectors a thread; the last wave does the list, the
// windows and the coefficients beside their passes, so that neither's registers
// add to the other's.  Three barriers a row:
//   holders                                                list
//   gradient of the row before, this row's loads           finishes the row before last; this list, bitmap, p
//   1
//   each vector as it arrives: largest, sum of the unlisted
//   2
//                                                          q, acceptances, neighbours, coefficients
//   3
// So the loads of a row run under the gradient pass of the one before and under
// its own sums, and only the step between 2 and 3 (about 3 us) has none.
// The listed entries' gradient is stored over the others' after the next row's barrier 2,
// when every holder has waited for its stores.
template <class TI, class TG, bool VEC, int WK, int NV, int NS, bool COUPLED>
__global__ __launch_bounds__((WK + 1) * kWave) void k_top_fused(TopLossParams p, int grid, void* __restrict__ grad) {
  using Rv = RowVecs<TI, VEC>;
  constexpr int E = Rv::E;
  constexpr int BLK = WK * kWave;  // threads that hold the row
  constexpr int kWords = stage_words(NV * BLK * E);
  constexpr int GS = sizeof(typename TG::storage);
  extern __shared__ uint32_t sh_dyn[];
  __shared__ float sh_m[WK], sh_s[WK], sh_cR;
  __shared__ float sh_a[2][128];  // acceptances of the row's neighbours (COUPLED)
  uint32_t* const map = sh_dyn;
  u32x4* const stage = reinterpret_cast<u32x4*>(map + kWords);  // NS vectors of a holder
  const int tid = threadIdx.x, lane = tid & (kWave - 1);
  const int wv = __builtin_amdgcn_readfirstlane(tid / kWave);

  if (wv == WK) {
    // ------------------------------------------------------- the list
    float* const lt = reinterpret_cast<float*>(stage + NS * BLK);  // target logits
    float* const lz = lt + p.k;                                // the draft's
    int* const li = reinterpret_cast<int*>(lz + p.k);          // ids
    int* const done_id = li + p.k;                             // of the row before: ids
    float* const done_g = reinterpret_cast<float*>(done_id + p.k);  // and gradient
    if (blockIdx.x == 0 && lane == 0) *p.counter = 0u;
    for (int i = lane; i < kWords; i += kWave) map[i] = 0;
    int64_t before = -1;
    auto finish = [&] {
      if (before < 0 || grad == nullptr) return;
      const int64_t e0 = before * int64_t(p.V);
      for (int i = lane; i < p.k; i += kWave)
        if (done_id[i] >= 0) TG::store1(grad, e0 + done_id[i], done_g[i]);
    };
    for (int64_t row = blockIdx.x; row < p.R; row += grid) {
      const int head = Rv(row, p.R, p.V).head;
      const int64_t l0 = row * p.k, e0 = row * int64_t(p.V);
      for (int i = lane; i < p.k; i += kWave) {
        int id = p.ids[l0 + i];
        const float t = load_top(p, l0 + i);
        if (id >= p.V || t == kNegInf) id = -1;
        float z = kNegInf;
        if (id >= 0) {
          z = TI::load1(p.zd, e0 + id);
          atomicOr(&map[(id + head) >> 5], 1u << ((id + head) & 31));
        }
        li[i] = id;
        lt[i] = id >= 0 ? t : kNegInf;
        lz[i] = z;
      }
      wait_lds_all();
      lds_barrier();  // 1
      const ListTarget lt_row = list_target(p, row, lt, li);
      const RowWindows rw = row_windows(row, p.layout, p.S, p.K);
      lds_barrier();  // 2
      const float wm = lane < WK ? sh_m[lane] : kNegInf;
      const RowRef ref = row_ref(wave_max(wm), p.scd);
      if (ref.deep) lds_barrier();
      const float su = wave_sum(lane < WK ? sh_s[lane] * (ref.deep ? 1.f : ex2(fmaxf(wm * p.scd, -1e30f) - ref.msc)) : 0.f);
      TopRow o = list_row(p, lt_row, lt, lz, li, ref, list_draft(p, lt, lz, ref), su);
      if (lane == 0) {
        publish(p.slots + 2 * row, o.a_tv, 1u);
        publish(p.slots + 2 * row + 1, o.a_eal, 1u);
      }
      double d_tv = 0.0, d_eal = 0.0;
      if constexpr (COUPLED) {
        // the rows that share a window with this one: places lo..hi of its sequence
        const int lo = p.layout == 0 ? 0 : max(0, rw.s - p.K + 1);
        const int hi = p.layout == 0 ? p.K - 1 : min(p.S - 1, rw.s + p.K - 1);
        for (int i = lo + lane; i <= hi; i += kWave) {
          float a[2] = {o.a_tv, o.a_eal};
          if (i != rw.s && rw.t1 >= rw.t0) collect<2>(p.slots + 2 * (rw.base + i), 1u, p.err, a);
          sh_a[0][i - lo] = a[0];
          sh_a[1][i - lo] = a[1];
        }
        wait_lds_all();
        // one window a lane
        if (rw.t0 + lane <= rw.t1) {
          const int w0 = rw.t0 + lane - lo, j = rw.s - (rw.t0 + lane);
          if (p.w_wtv != 0.f) d_tv = window_d([&](int i) { return sh_a[0][w0 + i]; }, p.K, j);
          if (p.w_eal != 0.f) d_eal = window_d([&](int i) { return sh_a[1][w0 + i]; }, p.K, j);
        }
        if (p.w_wtv != 0.f) d_tv = wave_sum_d(d_tv);
        if (p.w_eal != 0.f) d_eal = wave_sum_d(d_eal);
      }
      const double count = windows_of(rw);
      row_coefs(o, p, d_tv, d_eal, count);
      if (lane == 0) sh_cR = o.cR;
      lds_barrier();  // 3
      finish();
      if (lane == 0) write_row(p, row, o, count);
      // the list's gradient; the bitmap is emptied
      for (int i = lane; i < p.k; i += kWave) {
        const int id = li[i];
        done_id[i] = id;
        if (id < 0) continue;
        const float q = ex2(listed_log2(ref, lz[i], p.scd)) * o.inv_s;
        done_g[i] = listed_grad(o, q, listed_p(o, lt[i], p.sct), id);
        map[(id + head) >> 5] = 0;
      }
      wait_lds_all();
      before = row;
    }
    lds_barrier();  // the holders' last stores
    finish();
    return;
  }

  // -------------------------------------------------------- the row
  // Every load is issued unconditionally, so that a vector's registers have one
  // definition a row (with conditions the compiler kept old and new vectors side by side
  // and spilled 63 registers).  Rows of whole vectors go through buffer resources, which
  // read zeros and store nothing past their end (0 bytes where there is no next
  // row); lanes past a ragged row's last vector read that one.
  const uint32_t row_bytes = uint32_t(p.V) * sizeof(typename TI::storage), grow_bytes = uint32_t(p.V) * GS;
  u32x4 w[NV];
  // the first NS vectors of a row go through LDS, straight from memory: their loads
  // are issued as soon as the row before is summed, and run while its coefficients are made
  auto stage_row = [&](const rsrc_t& rs) {
#pragma unroll
    for (int v = 0; v < NS; ++v)
      bld16_lds(rs, stage + v * BLK + wv * kWave, uint32_t(tid) * 16u, uint32_t(v) * (BLK * 16u));
  };
  static_assert(VEC || NS == 0, "ragged rows are not staged");
  auto load_row_vec = [&](const rsrc_t& rs, const Rv& rv, int last, int v) {
    if constexpr (VEC)
      w[v] = bld16(rs, uint32_t(tid) * 16u, uint32_t(v) * (BLK * 16u));
    else
      w[v] = rv.raw(p.zd, min(v * BLK + tid, last));
  };
  auto row_rsrc = [&](int64_t r, bool there) {
    return make_rsrc(static_cast<const uint8_t*>(p.zd) + r * int64_t(row_bytes), there ? row_bytes : 0u);
  };
  // a wave-uniform number that the compiler takes as new, so that it makes the
  // conditions that follow from it where they are used, not once for every vector
  auto fresh = [](int x) {
    asm volatile("" : "+s"(x));
    return x;
  };
  {
    const Rv rv(int64_t(blockIdx.x), p.R, p.V);
    const rsrc_t rs = row_rsrc(blockIdx.x, true);
    stage_row(rs);
#pragma unroll
    for (int v = NS; v < NV; ++v) {
      load_row_vec(rs, rv, rv.ng - 1, v);
      __builtin_amdgcn_sched_barrier(0);  // in the order in which they are waited for
    }
  }
  for (int64_t row = blockIdx.x; row < p.R; row += grid) {
    const Rv rv(row, p.R, p.V);
    const int last_v = fresh((rv.ng - 1) / BLK), last_t = fresh((rv.ng - 1) % BLK);
    lds_barrier();  // 1
    float m = kNegInf, s = 0.f;  // s against max(m sc, -1e30)
    auto fold = [&](const u32x4& wx, int v) {
      float x[E];
      unpackv<TI>(wx, x);
      float cm = m;
#pragma unroll
      for (int e = 0; e < E; ++e) cm = fmaxf(cm, x[e]);
      const float at = fmaxf(cm * p.scd, -1e30f);
      const float keep = ex2(fmaxf(m * p.scd, -1e30f) - at);
      m = cm;
#pragma unroll
      for (int e = 0; e < E; ++e) x[e] = ex2(__builtin_fmaf(x[e], p.scd, -at));
      const uint32_t bits = listed_bits<E>(map, v * BLK + tid);
      if (bits)
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (bits >> e & 1u) x[e] = 0.f;
      s = __builtin_fmaf(s, keep, tree_sum(x));
    };
    if constexpr (!VEC)
      if (tid == 0 && !rv.whole(0)) w[0] = rv.edge(p.zd, 0, w[0]);
    if constexpr (NS > 0) {
      // the staged vectors are older than the NV - NS loads of the others
      wait_vmem_le<NV - NS>();
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      if (v < NS) w[v] = stage[v * BLK + tid];
      if (v < last_v) {
        pin(w[v]);
        fold(w[v], v);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    // the row's last vectors, on their own: -inf past its end
    u32x4 wl = w[0];
#pragma unroll
    for (int v = 1; v < NV; ++v)
      if (v == last_v) wl = w[v];
    if (tid > last_t) wl = Rv::none();
    if constexpr (!VEC)
      if (tid == last_t && rv.ng > 1 && !rv.whole(rv.ng - 1)) wl = rv.edge(p.zd, rv.ng - 1, wl);
    pin(wl);
    fold(wl, last_v);
    wait_vmem_all();  // the stores of the row before are done
    const int64_t next = row + grid;
    const bool more = next < p.R;
    const rsrc_t rsn = row_rsrc(more ? next : row, more);
    stage_row(rsn);
    {
      const float M = wave_max(m);
      s = wave_sum(s * ex2(fmaxf(m * p.scd, -1e30f) - fmaxf(M * p.scd, -1e30f)));
      if (lane == 0) {
        sh_m[wv] = M;
        sh_s[wv] = s;
      }
      m = M;
    }
    lds_barrier();  // 2
    m = wave_max(lane < WK ? sh_m[lane] : kNegInf);
    const RowRef ref = row_ref(m, p.scd);
    if (ref.deep) {  // nothing was above -1e30: the sum again, at its scale
      s = 0.f;
      auto again = [&](const u32x4& wx, int v) {
        float x[E];
        unpackv<TI>(wx, x);
        const uint32_t bits = listed_bits<E>(map, v * BLK + tid);
#pragma unroll
        for (int e = 0; e < E; ++e) s += bits >> e & 1u ? 0.f : ex2(__builtin_fmaf(x[e], ref.sc, -ref.msc));
      };
#pragma unroll
      for (int v = 0; v < NV; ++v)
        if (v < last_v) again(w[v], v);
      again(wl, last_v);
      s = wave_sum(s);
      if (lane == 0) sh_s[wv] = s;
      lds_barrier();  // 2, for the list too
    }
    lds_barrier();  // 3
    const Rv rn(more ? next : row, p.R, p.V);
    const int last_n = more ? rn.ng - 1 : 0;
    const float cR = sh_cR;
    const int last_v3 = fresh(grad != nullptr ? last_v : -1);
    const rsrc_t gr = make_rsrc(static_cast<uint8_t*>(grad) + row * int64_t(grow_bytes), grow_bytes);
    auto store = [&](const u32x4& wx, int v) {
      const int gi = v * BLK + tid;
      float x[E];
      unpackv<TI>(wx, x);
#pragma unroll
      for (int e = 0; e < E; ++e) x[e] = cR * ex2(__builtin_fmaf(x[e], ref.sc, -ref.msc));
      if constexpr (VEC) {
        store_g<TG, E>(gr, uint32_t(gi) * (E * GS), x);  // dropped past the row
      } else if (rv.whole(gi)) {
        store_vec<TG, E>(grad, (rv.g0 + gi) * E, x);
      } else if (gi < rv.ng) {
#pragma unroll 1
        for (int e = 0; e < E; ++e) {
          const int i = rv.index(gi, e);
          float ge = x[0];
#pragma unroll
          for (int q = 1; q < E; ++q) ge = e == q ? x[q] : ge;
          if (i >= 0 && i < p.V) TG::store1(grad, (rv.g0 + gi) * E + e, ge);
        }
      }
    };
    if (last_v3 >= 0) store(wl, last_v);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      if (v < last_v3) {
        pin(w[v]);  // the packed vector was kept, not unpacked copies of it
        store(w[v], v);
      }
      if (v >= NS) load_row_vec(rsn, rn, last_n, v);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  wait_vmem_all();
  lds_barrier();  // the last stores
}

// -------------------------------------------------- multi-kernel schedule
template <class TI, bool VEC, int U, int BLK>
__global__ __launch_bounds__(BLK) void k_top_rows(TopLossParams p) {
  using Rv = RowVecs<TI, VEC>;
  constexpr int E = Rv::E;
  extern __shared__ uint32_t sh_map[];
  __shared__ float sh_t[kTopMax], sh_z[kTopMax];
  __shared__ int sh_id[kTopMax];
  __shared__ float sh_m[BLK / kWave], sh_s[BLK / kWave];

  const int64_t row = blockIdx.x;
  const Rv rv(row, p.R, p.V);
  const int64_t e0 = row * int64_t(p.V), l0 = row * p.k;
  const int words = bitmap_words(p.V);
  if (blockIdx.x == 0 && threadIdx.x == 0) *p.counter = 0u;
  for (int i = threadIdx.x; i < words; i += BLK) sh_map[i] = 0;
  __syncthreads();
  for (int i = threadIdx.x; i < p.k; i += BLK) {
    const int id = p.ids[l0 + i];
    const float t = load_top(p, l0 + i);
    const bool in = id >= 0 && id < p.V && t != kNegInf;
    sh_id[i] = id;
    sh_t[i] = in ? t : kNegInf;
    sh_z[i] = in ? TI::load1(p.zd, e0 + id) : kNegInf;
    if (in) atomicOr(&sh_map[(id + rv.head) >> 5], 1u << ((id + rv.head) & 31));
  }
  __syncthreads();
  // the largest logit of all entries, the sum over the unlisted ones against
  // max(largest sc, -1e30) so far
  float m = kNegInf, s = 0.f;
  for (int base = threadIdx.x; base < rv.ng; base += BLK * U) {
    u32x4 w[1][U];
    float x[U][E];
    rv.load({p.zd}, base, BLK, w);
    rv.unpack(w[0], x);
    float cm = m;
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int e = 0; e < E; ++e) cm = fmaxf(cm, x[u][e]);
    const float at = fmaxf(cm * p.scd, -1e30f);
    s *= ex2(fmaxf(m * p.scd, -1e30f) - at);
    m = cm;
    float c[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int gi = base + u * BLK;
      const uint32_t bits = gi < rv.ng ? listed_bits<E>(sh_map, gi) : 0u;
#pragma unroll
      for (int e = 0; e < E; ++e) x[u][e] = ex2(__builtin_fmaf(x[u][e], p.scd, -at));
      if (bits)
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (bits >> e & 1u) x[u][e] = 0.f;
      c[u] = tree_sum(x[u]);
    }
    s += tree_sum(c);
  }
  const int lane = threadIdx.x & (kWave - 1), wv = threadIdx.x / kWave;
  const float wm = wave_max(m);
  if (lane == 0) sh_m[wv] = wm;
  __syncthreads();
  float bm = sh_m[0];
  for (int i = 1; i < BLK / kWave; ++i) bm = fmaxf(bm, sh_m[i]);
  const RowRef ref = row_ref(bm, p.scd);
  if (ref.deep) {
    s = 0.f;
    for (int gi = threadIdx.x; gi < rv.ng; gi += BLK) {
      float x[E];
      TI::unpack(to_uint4(rv.load(p.zd, gi)), x);
      const uint32_t bits = listed_bits<E>(sh_map, gi);
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (!(bits >> e & 1u)) s += ex2(__builtin_fmaf(x[e], ref.sc, -ref.msc));
    }
  } else {
    s *= ex2(fmaxf(m * p.scd, -1e30f) - ref.msc);
  }
  s = wave_sum(s);
  if (lane == 0) sh_s[wv] = s;
  __syncthreads();
  if (threadIdx.x < kWave) {
    s = wave_sum(lane < BLK / kWave ? sh_s[lane] : 0.f);
    const TopRow o = list_row(p, list_target(p, row, sh_t, sh_id), sh_t, sh_z, sh_id, ref,
                              list_draft(p, sh_t, sh_z, ref), s);
    if (lane == 0) {
      p.stats[row] = o;
      publish(p.slots + 2 * row, o.a_tv, 1u);
      publish(p.slots + 2 * row + 1, o.a_eal, 1u);
    }
  }
}

__global__ __launch_bounds__(kRowBlock) void k_top_scan(TopLossParams p) {
  const int64_t r = int64_t(blockIdx.x) * kRowBlock + threadIdx.x;
  if (r >= p.R) return;
  const RowWindows rw = row_windows(r, p.layout, p.S, p.K);
  const TopRow* st = p.stats + rw.base;
  double d_tv = 0.0, d_eal = 0.0;
  for (int t = rw.t0; t <= rw.t1; ++t) {
    if (p.w_wtv != 0.f) d_tv += window_d([&](int i) { return st[t + i].a_tv; }, p.K, rw.s - t);
    if (p.w_eal != 0.f) d_eal += window_d([&](int i) { return st[t + i].a_eal; }, p.K, rw.s - t);
  }
  TopRow o = p.stats[r];
  row_coefs(o, p, d_tv, d_eal, windows_of(rw));
  TopRow& out = p.stats[r];
  out.cR = o.cR;
  out.cA = o.cA;
  out.cB = o.cB;
  out.cP = o.cP;
  out.cX = o.cX;
  write_row(p, r, o, windows_of(rw));
}

template <class TI, class TG, bool VEC, int U>
__global__ __launch_bounds__(kRowBlock) void k_top_grad(TopLossParams p, int splits, void* __restrict__ grad) {
  using Rv = RowVecs<TI, VEC>;
  constexpr int E = Rv::E;
  const int64_t row = blockIdx.x;
  const Rv rv(row, p.R, p.V);
  const TopRow s = p.stats[row];
  const float sc = s.flags & kTopDeep ? kDeepScale : p.scd;
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
      for (int e = 0; e < E; ++e) g[e] = s.cR * ex2(__builtin_fmaf(x[e], sc, -s.msc));
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
    const float q = ex2(__builtin_fmaf(TI::load1(p.zd, e0 + id), sc, -s.msc)) * s.inv_s;
    TG::store1(grad, e0 + id, listed_grad(s, q, listed_p(s, t, p.sct), id));
  }
}

// ------------------------------------------------------------------- loss
constexpr int kLossBlock = 256;

__device__ double block_sum_d(double v, double* sh) {
  v = wave_sum_d(v);
  if ((threadIdx.x & (kWave - 1)) == 0) sh[threadIdx.x / kWave] = v;
  __syncthreads();
  double t = 0.0;
  for (int i = 0; i < kLossBlock / kWave; ++i) t += sh[i];
  __syncthreads();
  return t;
}

// Every window's E and the loss: workgroup b sums the rows of its slice (a window
// counts where it starts); the last one to end adds the slices' sums in order.
__global__ __launch_bounds__(kLossBlock) void k_top_loss(TopLossParams p, int n, double* parts, float* loss,
                                                         float* terms, float* e_tv, float* e_eal,
                                                         const unsigned* err) {
  __shared__ double sh[kLossBlock / kWave];
  __shared__ int sh_last;
  const int64_t r0 = p.R * blockIdx.x / n, r1 = p.R * (int64_t(blockIdx.x) + 1) / n;
  double v[4] = {0.0, 0.0, 0.0, 0.0};  // sums of E_tv, E_eal, KL, TV
  const bool tv = p.w_wtv != 0.f || e_tv != nullptr, eal = p.w_eal != 0.f || e_eal != nullptr;
  for (int64_t r = r0 + threadIdx.x; r < r1; r += kLossBlock) {
    const RowWindows rw = row_windows(r, p.layout, p.S, p.K);
    if (rw.starts && (tv || eal)) {
      double Pt = 1.0, Pe = 1.0, Et = 0.0, Ee = 0.0;
      for (int i = 0; i < p.K; ++i) {
        Pt *= double(value_of(p.slots[2 * (r + i)]));
        Pe *= double(value_of(p.slots[2 * (r + i) + 1]));
        Et += Pt;
        Ee += Pe;
      }
      // the sums are of the E that the caller gets
      if (e_tv) e_tv[rw.own] = float(Et);
      if (e_eal) e_eal[rw.own] = float(Ee);
      v[0] += double(float(Et));
      v[1] += double(float(Ee));
    }
    const float2 l = p.row_loss[r];
    v[2] += double(l.x);
    v[3] += double(l.y);
  }
  for (int i = 0; i < 4; ++i) v[i] = block_sum_d(v[i], sh);
  if (n > 1) {
    if (threadIdx.x == 0) {
      for (int i = 0; i < 4; ++i)
        __hip_atomic_store(parts + 4 * blockIdx.x + i, v[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      sh_last = __hip_atomic_fetch_add(p.counter, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == unsigned(n - 1);
    }
    __syncthreads();
    if (!sh_last) return;
    for (int i = 0; i < 4; ++i) {
      double s = 0.0;
      for (int b = threadIdx.x; b < n; b += kLossBlock)
        s += __hip_atomic_load(parts + 4 * b + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      v[i] = block_sum_d(s, sh);
    }
  }
  if (threadIdx.x != 0) return;
  // a term whose weight is 0 reads 0
  const double t0 = p.W > 0 && p.w_wtv != 0.f ? -v[0] / double(p.W) : 0.0;
  const double t1 = p.W > 0 && p.w_eal != 0.f ? -v[1] / double(p.W) : 0.0;
  const double t2 = p.w_kl != 0.f ? v[2] / double(p.R) : 0.0;
  const double t3 = p.W > 0 && p.w_tv != 0.f ? v[3] / (double(p.W) * p.K) : 0.0;
  // a set error word (a poll of the resident schedule timed out): NaN
  loss[0] = (err != nullptr && *err != 0u) ? __builtin_nanf("")
                                           : float(double(p.w_wtv) * t0 + double(p.w_eal) * t1 +
                                                   double(p.w_kl) * t2 + double(p.w_tv) * t3);
  if (terms) {
    terms[0] = float(t0);
    terms[1] = float(t1);
    terms[2] = float(t2);
    terms[3] = float(t3);
  }
}

// Empties the acceptances' words and sets the error word.
__global__ void k_top_clear(uint64_t* p, int64_t n, unsigned* err, unsigned value) {
  const int64_t stride = int64_t(gridDim.x) * blockDim.x;
  const int64_t t = int64_t(blockIdx.x) * blockDim.x + threadIdx.x;
  for (int64_t i = t; i < n; i += stride) p[i] = 0;
  if (t == 0) *err = value;
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
  p.inv_t_d = a.inv_t_d;
  p.grad_scale = a.grad_scale;
  return p;
}

hipError_t loss_launch(const TopLossArgs& a, bool waited) {
  const int64_t want = (a.R + kLossBlock - 1) / kLossBlock;
  const int n = int(want < kTopLossParts ? want : kTopLossParts);
  k_top_loss<<<dim3(unsigned(n)), kLossBlock, 0, a.stream>>>(params_of(a), n, a.loss_parts, a.loss, a.terms, a.e_tv,
                                                            a.e_eal, waited ? a.err : nullptr);
  return hipGetLastError();
}

template <class TI, class TG, bool VEC, int WK, int NV, int NS, bool COUPLED>
hipError_t fused_launch(const TopLossArgs& a, bool* used) {
  constexpr int BLK = (WK + 1) * kWave;
  auto kern = k_top_fused<TI, TG, VEC, WK, NV, NS, COUPLED>;
  const DevInfo di = device_info();
  if (di.cus == 0 || (COUPLED && a.coop && !di.coop)) return hipSuccess;
  const size_t lds = fused_lds_bytes(NV * WK * kWave * TI::kVec, NS * WK * kWave, a.k);
  int per_cu = 0;
  hipError_t e = hipOccupancyMaxActiveBlocksPerMultiprocessor(&per_cu, kern, BLK, lds);
  if (e != hipSuccess) return e;
  int64_t grid = int64_t(per_cu) * di.cus;
  if (grid > a.R) grid = a.R;
  // a row's neighbours have to be in other workgroups' hands at the same time
  if (grid < 1 || (COUPLED && grid < a.R && grid < a.K)) return hipSuccess;
  TopLossParams p = params_of(a);
  int g = int(grid);
  void* grad = a.grad;
  if constexpr (COUPLED) {
    const int64_t words = 2 * a.R;
    k_top_clear<<<dim3(unsigned(words < 256 * 256 ? (words + 255) / 256 : 256)), 256, 0, a.stream>>>(
        a.slots, words, a.err, unsigned(initial_error_word()));
    if ((e = hipGetLastError()) != hipSuccess) return e;
    if (a.coop) {
      void* args[] = {&p, &g, &grad};
      e = hipLaunchCooperativeKernel(reinterpret_cast<const void*>(kern), dim3(unsigned(g)), dim3(BLK), args,
                                     unsigned(lds), a.stream);
      *used = e == hipSuccess;
      return e;
    }
  }
  // the grid fits the device at once (see the occupancy bound above)
  kern<<<dim3(unsigned(g)), BLK, lds, a.stream>>>(p, g, grad);
  e = hipGetLastError();
  *used = e == hipSuccess;
  return e;
}

template <class TI, class TG, bool VEC, bool COUPLED>
hipError_t fused_size(const TopLossArgs& a, bool* used) {
  const int ng = a.V / TI::kVec + (VEC ? 0 : 2);  // vectors that cover a row, at most
  if (a.R * a.V < TI::kVec) return hipSuccess;  // less than a vector in all
  constexpr int NS = VEC ? 8 : 0;
  if (ng <= 1 * 64 * 18) return fused_launch<TI, TG, VEC, 1, 18, 0, COUPLED>(a, used);
  if (ng <= 3 * 64 * 18) return fused_launch<TI, TG, VEC, 3, 18, 0, COUPLED>(a, used);
  if (ng <= 7 * 64 * 18) return fused_launch<TI, TG, VEC, 7, 18, 0, COUPLED>(a, used);
  if (ng <= 15 * 64 * 18) return fused_launch<TI, TG, VEC, 15, 18, NS, COUPLED>(a, used);
  if (ng <= 15 * 64 * 20) return fused_launch<TI, TG, VEC, 15, 20, NS, COUPLED>(a, used);
  return hipSuccess;
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
  const bool coupled = a.w_wtv != 0.f || a.w_eal != 0.f;
  bool used = false;
  hipError_t e = hipSuccess;
  if (!a.streaming) {
    if (a.gd == DType::kBf16)
      e = coupled ? fused_size<TI, GBf16, VEC, true>(a, &used) : fused_size<TI, GBf16, VEC, false>(a, &used);
    else
      e = coupled ? fused_size<TI, GF32, VEC, true>(a, &used) : fused_size<TI, GF32, VEC, false>(a, &used);
    if (e != hipSuccess) return e;
    if (used) return loss_launch(a, coupled);
  }
  with_row_shape<4>(a.R, a.V, TI::kVec, [&](auto sh) {
    using Sh = decltype(sh);
    k_top_rows<TI, VEC, Sh::kU, Sh::kBlock>
        <<<dim3(unsigned(a.R)), Sh::kBlock, size_t(bitmap_words(a.V)) * 4, a.stream>>>(params_of(a));
    e = hipGetLastError();
  });
  if (e != hipSuccess) return e;
  k_top_scan<<<dim3(unsigned((a.R + kRowBlock - 1) / kRowBlock)), kRowBlock, 0, a.stream>>>(params_of(a));
  if ((e = loss_launch(a, false)) != hipSuccess) return e;
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
