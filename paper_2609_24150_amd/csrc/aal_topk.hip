// A row's k largest logits with their ids, and the log-sum-exp of the others
// (aal_topk_logits): what a training set stores of a target's logits.
//
//   order: v before w iff z_v > z_w, or z_v = z_w and v < w
//   rest  = ln sum_{v not among the k} exp(z_v / T)
//
// One workgroup per row, which reads it once.  k_topk_rows cuts the row into lines of up
// to four vectors and keeps of each the largest logit and the sum of 2^(z sc - that) in
// a register of a thread.  k lines hold a logit at least as large as the k-th
// largest of the lines' maxima, so a threshold t that k maxima reach is passed
// by all of the k largest and by few others; it is found by bisection over whole
// numbers that order as logits, one ballot count per line and step, in every
// wave for its share of k.  The lines that reach t are read again (k = 64 of
// 128,256: 2% of the row), their entries from t on sorted.  The remainder is
// the sum of the lines below t and of the entries not taken: never a difference of sums, so it
// keeps its digits where the list has nearly all mass.  Its reference is the first entry not
// taken or, where no candidate is left over, t, unless the others lie so far below
// t that exponentials against it vanish: those are summed again, against the largest of them.
// k_topk_short, for rows of up to 16 logits per thread, bisects over the logits.
// Where ties or clusters put more entries at t than the candidates' list holds
// (rows of few distinct values, rows with fewer than k finite ones), the
// workgroup takes select_slowly, a radix select over the row that is right for everything.
//
// Bound by memory where rows are long: 14,336 rows of 128,256 bf16, k = 64: 590
// us, 6.2 TB/s, 89% of what a lone read of them takes (k = 8 94%, k = 256 75%: sorting).
// Few rows are bound by the arithmetic of the CU that each has to itself: 7 of 151,936, 18 us.
#include "aal_device.h"
#include "aal_row_ref.h"
#include "aal_rowops.h"
#include "aal_select.h"
#include "aal_toplist.h"

namespace aal {
namespace {

constexpr float kLn2 = 0.693147180559945309417f;

// A candidate as one whole number of 63 bits: larger for a larger logit, then
// for a lower index; the lowest bit tells -0, which has the key of +0.  Read as a
// double it is positive, finite and normal (for every logit that is no NaN), so that it
// compares at the rate of doubles, four times that of 64-bit whole numbers.
__device__ __forceinline__ uint64_t entry_of(uint32_t key, int v, bool neg_zero) {
  return (uint64_t(key) << 31) | ((0x3fffffffu - uint32_t(v)) << 1) | (neg_zero ? 1u : 0u);
}
__device__ __forceinline__ uint32_t entry_key(uint64_t e) { return uint32_t(e >> 31); }
__device__ __forceinline__ int entry_index(uint64_t e) { return int(0x3fffffffu - (uint32_t(e) << 1 >> 2)); }

// CAP: the most candidates, and groups read again, that fit.
template <int CAP_>
struct TopkShared {
  static constexpr int CAP = CAP_;
  alignas(16) uint64_t cand[CAP];    // entry_of() of the candidates
  alignas(16) uint64_t sorted[CAP];  // the same by rank
  uint16_t queue[CAP];               // groups read again
  alignas(16) uint32_t hist[256];
  float f[16];
  int i[1][16];
  uint32_t n, digit, need;
};

struct TopkParams {
  const void* z;
  int64_t rows, row0;  // all of them, the first one of the launch
  int V, k;
  float sc, inv_t;
  void* top;
  int32_t* ids;
  float* rest;
};

// A sum against reference a, none of whose entries is above it, against b >= a.
__device__ __forceinline__ float rescaled(float s, const RowRef& a, const RowRef& b) {
  if (a.m == kNegInf) return 0.f;
  return s * ex2(a.steep || b.steep ? (a.m - b.m) * a.sc : a.msc - b.msc);
}

template <int WAVES>
__device__ __forceinline__ float block_max(float v, float* sh) {
  v = wave_max(v);
  if constexpr (WAVES == 1) return v;
  if ((threadIdx.x & (kWave - 1)) == 0) sh[threadIdx.x / kWave] = v;
  __syncthreads();
  float m = sh[0];
#pragma unroll
  for (int i = 1; i < WAVES; ++i) m = fmaxf(m, sh[i]);
  __syncthreads();
  return m;
}

// The bucket of a candidate among 256 over [t, m], larger logits first: monotone in the logit.
template <class TI>
__device__ __forceinline__ int bucket_of(uint64_t e, float t, float scale) {
  return 255 - min(255, int((key_logit<TI>(entry_key(e)) - t) * scale));
}

// Sorts the n candidates, all in [t, m], writes the first k, and returns the sum over
// the others (this thread's share) against the first of them, whose scale is `at` (t's where
// there is none).  Up to 64 are ranked by counting; more go through 256 buckets and are
// ranked in theirs (lists of 256 of 14,336 rows of 4,000: 207 us with counting alone).
template <class TI, int BLK, class Sh>
__device__ __forceinline__ float write_ranked(const TopkParams& p, int64_t row, int n, float t, float m, RowRef& at,
                                              Sh& sh) {
  const uint64_t* sorted = sh.sorted;
  if (n <= kWave) {
    if (int(threadIdx.x) < (n & 1)) sh.cand[n] = 0;  // below every candidate
    __syncthreads();
    if (int(threadIdx.x) < n) {
      const uint64_t mine = sh.cand[threadIdx.x];
      const double at = __builtin_bit_cast(double, mine);
      int rank = 0;
#pragma unroll 4
      for (int j = 0; j < n; j += 2) {
        const double2 two = *reinterpret_cast<const double2*>(&sh.cand[j]);
        rank += (two.x > at) + (two.y > at);
      }
      sh.sorted[rank] = mine;
    }
  } else {
    const float range = m - t;
    const float scale = range > 0.f && range < 1e38f ? 255.f / range : 0.f;  // 0: one bucket
    const float from = scale > 0.f ? t : 0.f;
    for (int i = threadIdx.x; i < 256; i += BLK) sh.hist[i] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += BLK)
      atomicAdd(&sh.hist[scale > 0.f ? bucket_of<TI>(sh.cand[i], from, scale) : 0], 1u);
    __syncthreads();
    if (threadIdx.x < kWave) {  // where each bucket starts
      uint4& mine = reinterpret_cast<uint4*>(sh.hist)[threadIdx.x];
      const uint4 c = mine;
      int end = int(c.x + c.y + c.z + c.w);
      const int own = end;
      for (int off = 1; off < kWave; off <<= 1) {
        const int o = __shfl_up(end, off, kWave);
        if (int(threadIdx.x) >= off) end += o;
      }
      const uint32_t s0 = uint32_t(end - own);
      mine = make_uint4(s0, s0 + c.x, s0 + c.x + c.y, s0 + c.x + c.y + c.z);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += BLK) {
      const uint64_t e = sh.cand[i];
      sh.sorted[atomicAdd(&sh.hist[scale > 0.f ? bucket_of<TI>(e, from, scale) : 0], 1u)] = e;
    }
    __syncthreads();
    // a bucket's entries now end where the next one's start
    for (int i = threadIdx.x; i < n; i += BLK) {
      const uint64_t e = sh.sorted[i];
      const int b = scale > 0.f ? bucket_of<TI>(e, from, scale) : 0;
      const int first = b > 0 ? int(sh.hist[b - 1]) : 0, end = int(sh.hist[b]);
      int rank = first;
      for (int j = first; j < end; ++j) rank += sh.sorted[j] > e;
      sh.cand[rank] = e;
    }
    sorted = sh.cand;
  }
  __syncthreads();
  const int64_t o0 = row * int64_t(p.k);
  at = row_ref(n > p.k ? key_logit<TI>(entry_key(sorted[p.k])) : t, p.sc);
  float s = 0.f;
  for (int j = threadIdx.x; j < n; j += BLK) {
    const uint64_t key = sorted[j];
    if (j < p.k) {
      p.ids[o0 + j] = entry_index(key);
      const uint32_t b = key & 1u ? 0x80000000u : __builtin_bit_cast(uint32_t, key_logit<TI>(entry_key(key)));
      static_cast<typename TI::bits*>(p.top)[o0 + j] = typename TI::bits(key_bits<TI>() == 16 ? b >> 16 : b);
    } else {
      s += ex2(log2_of(at, key_logit<TI>(entry_key(key))));
    }
  }
  return s;
}

// Adds the entries of x (indices v0 on) that `take` has a bit for.
template <class TI, class Sh, int E>
__device__ __forceinline__ void add_candidates(Sh& sh, const float (&x)[E], int v0, uint32_t take) {
  if (take == 0u) return;
  uint32_t slot = atomicAdd(&sh.n, uint32_t(__popc(take)));
#pragma unroll
  for (int e = 0; e < E; ++e)
    if (take >> e & 1u) {
      if (slot < uint32_t(Sh::CAP))
        sh.cand[slot] = entry_of(order_key<TI>(x[e]), v0 + e, __builtin_bit_cast(uint32_t, x[e]) == 0x80000000u);
      ++slot;
    }
}

// Any row: the k-th largest key digit by digit, then a pass in index order that
// collects the larger entries and the first of its ties.  t becomes the k-th logit; returns this
// thread's share of the others' sum against it, which is the reference of choice where some of
// its ties are left over (`tied`).
template <class TI, bool VEC, int BLK, class Sh>
__device__ __forceinline__ float select_slowly(const TopkParams& p, int64_t row, Sh& sh, float& t, bool& tied) {
  using Rv = RowVecs<TI, VEC>;
  constexpr int E = Rv::E;
  constexpr int WV = BLK / kWave;
  const Rv rv(row, p.rows, p.V);
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wv = tid / kWave;
  uint32_t prefix = 0, need = uint32_t(p.k);
  for (int shift = 24; shift >= 32 - key_bits<TI>(); shift -= 8) {
    __syncthreads();
    for (int i = tid; i < 256; i += BLK) sh.hist[i] = 0;
    __syncthreads();
    for (int gi = tid; gi < rv.ng; gi += BLK) {
      float x[E];
      TI::unpack(to_uint4(rv.load(p.z, gi)), x);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int v = rv.index(gi, e);
        if (v < 0 || v >= p.V) continue;
        const uint32_t key = order_key<TI>(x[e]);
        if (shift == 24 || (key >> (shift + 8)) == (prefix >> (shift + 8)))
          atomicAdd(&sh.hist[(key >> shift) & 255u], 1u);
      }
    }
    __syncthreads();
    if (tid == 0) {
      uint32_t left = need;
      int d = 255;
      while (d > 0 && sh.hist[d] < left) left -= sh.hist[d--];
      sh.digit = uint32_t(d);
      sh.need = left;
    }
    __syncthreads();
    prefix |= sh.digit << shift;
    need = sh.need;  // of the entries whose key starts with `prefix`
  }
  t = key_logit<TI>(prefix);
  tied = sh.hist[sh.digit] > need;
  const RowRef at_t = row_ref(t, p.sc);
  if (tid == 0) sh.n = 0;
  uint32_t ties = 0;  // before this pass
  float s = 0.f;
  for (int base = 0; base < rv.ng; base += BLK) {
    const int gi = base + tid;
    uint32_t key[E];
    int mine = 0;
    float x[E];
    if (gi < rv.ng) {
      TI::unpack(to_uint4(rv.load(p.z, gi)), x);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int v = rv.index(gi, e);
        key[e] = order_key<TI>(x[e]);
        mine += v >= 0 && v < p.V && key[e] == prefix;
      }
    }
    // ties of the lanes and waves before this thread
    int before = mine;
    for (int off = 1; off < kWave; off <<= 1) {
      const int o = __shfl_up(before, off, kWave);
      if (lane >= off) before += o;
    }
    __syncthreads();
    if (lane == kWave - 1) sh.i[0][wv] = before;
    __syncthreads();
    uint32_t at = ties + uint32_t(before - mine);
    for (int i = 0; i < WV; ++i) {
      if (i < wv) at += uint32_t(sh.i[0][i]);
      ties += uint32_t(sh.i[0][i]);
    }
    if (gi >= rv.ng) continue;
    uint32_t take = 0;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int v = rv.index(gi, e);
      if (v < 0 || v >= p.V) continue;
      const bool tie = key[e] == prefix;
      if (key[e] > prefix || (tie && at < need))
        take |= 1u << e;
      else
        s += ex2(log2_of(at_t, x[e]));
      at += tie;
    }
    add_candidates<TI>(sh, x, rv.index(gi, 0), take);
  }
  __syncthreads();
  return s;
}

// The remainder, whose sum against `at` has this thread's share s.  `low`: all of it lies below t.
// Exponentials against t are flushed below 2^-126: 2^30 entries of that size make 2^-96,
// the last digits of a sum of 2^-72.  Where there is less, what is below t is summed again, over the
// row, against the largest of it.  `again`: s lacks what is below t, which a steep t is no reference for.
template <class TI, bool VEC, int BLK, class Sh>
__device__ __forceinline__ void write_rest(const TopkParams& p, int64_t row, float s, RowRef at, bool low, bool again,
                                           float t, Sh& sh) {
  constexpr int WV = BLK / kWave;
  if (p.rest == nullptr) return;
  s = block_sum<WV>(s, sh.f);
  if (again || (low && s < 0x1p-72f && t != kNegInf)) {
    using Rv = RowVecs<TI, VEC>;
    constexpr int E = Rv::E;
    const Rv rv(row, p.rows, p.V);
    if (low) {
      float m = kNegInf;
      for (int gi = threadIdx.x; gi < rv.ng; gi += BLK) {
        float x[E];
        TI::unpack(to_uint4(rv.load(p.z, gi)), x);
#pragma unroll
        for (int e = 0; e < E; ++e) m = fmaxf(m, x[e] < t ? x[e] : kNegInf);
      }
      at = row_ref(block_max<WV>(m, sh.f), p.sc);
      s = 0.f;
    }
    float more = 0.f;
    if (at.m != kNegInf)
      for (int gi = threadIdx.x; gi < rv.ng; gi += BLK) {
        float x[E];
        TI::unpack(to_uint4(rv.load(p.z, gi)), x);
#pragma unroll
        for (int e = 0; e < E; ++e) more += x[e] < t ? ex2(log2_of(at, x[e])) : 0.f;
      }
    s += block_sum<WV>(more, sh.f);
  }
  if (threadIdx.x != 0) return;
  const float ref = at.steep ? at.m * p.inv_t : at.msc * kLn2;
  p.rest[row] = s > 0.f ? __builtin_fmaf(__log2f(s), kLn2, ref) : kNegInf;
}

// Rows of up to 16 BLK logits: all of them in registers.
template <class TI, bool VEC, int BLK, int CAP>
__global__ __launch_bounds__(BLK) void k_topk_short(TopkParams p) {
  using Rv = RowVecs<TI, VEC>;
  constexpr int E = Rv::E;
  constexpr int WV = BLK / kWave;
  constexpr int U = 16 / E + (VEC ? 0 : 1);  // a row may start and end inside a vector
  __shared__ TopkShared<CAP> sh;
  const int64_t row = p.row0 + blockIdx.x;
  const Rv rv(row, p.rows, p.V);
  u32x4 w[1][U];
  rv.load({p.z}, int(threadIdx.x), BLK, w);
  float x[U][E], y[U * E];
  rv.unpack(w[0], x);
  float m = kNegInf;
  if (threadIdx.x == 0) sh.n = 0;
#pragma unroll
  for (int u = 0; u < U; ++u)
#pragma unroll
    for (int e = 0; e < E; ++e) {
      y[u * E + e] = x[u][e];
      m = fmaxf(m, x[u][e]);
    }
  m = block_max<WV>(m, sh.f);
  float t = threshold<TI, WV>(y, p.k, m, sh.f);
  RowRef rs = row_ref(t, p.sc), at;  // what is below t is summed against it
  bool tied = false, again = rs.steep;
  float s = 0.f;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int gi = int(threadIdx.x) + u * BLK;
    uint32_t take = 0;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int v = rv.index(gi, e);
      if (x[u][e] >= t)
        take |= gi < rv.ng && v >= 0 && v < p.V ? 1u << e : 0u;
      else
        s += ex2(__builtin_fmaf(x[u][e], rs.sc, -rs.msc));
    }
    add_candidates<TI>(sh, x[u], rv.index(gi, 0), take);
  }
  __syncthreads();
  int n = int(sh.n);
  if (n > CAP) {
    s = select_slowly<TI, VEC, BLK>(p, row, sh, t, tied);
    rs = row_ref(t, p.sc);
    again = false;
    n = p.k;
  }
  const float others = write_ranked<TI, BLK>(p, row, n, t, m, at, sh);
  write_rest<TI, VEC, BLK>(p, row, again ? others : rescaled(s, rs, at) + others, at, n == p.k && !tied, again, t, sh);
}

// The largest, or the sum, over the L lanes that share a line (L = 1, 2, 4).
template <int L>
__device__ __forceinline__ float line_max(float v) {
  if constexpr (L >= 2) v = fmaxf(v, dppm<0xB1>(v));
  if constexpr (L >= 4) v = fmaxf(v, dppm<0x4E>(v));
  return v;
}
template <int L>
__device__ __forceinline__ float line_sum(float v) {
  if constexpr (L >= 2) v += dppm<0xB1>(v);
  if constexpr (L >= 4) v += dppm<0x4E>(v);
  return v;
}
// Longer rows.  In every round a thread loads U vectors, each U adjacent lanes
// a line of U adjacent vectors at every step, and the lane takes the line of
// the step that it is in the U lanes.  A group of a thread is its lines of `rounds` rounds.
template <class TI, bool VEC, int U, int BLK, int NG, int CAP, bool ONE>
__global__ __launch_bounds__(BLK, 8) void k_topk_rows(TopkParams p, int rounds_) {
  using Rv = RowVecs<TI, VEC>;
  constexpr int E = Rv::E;
  constexpr int WV = BLK / kWave;
  __shared__ TopkShared<CAP> sh;
  const int64_t row = p.row0 + blockIdx.x;
  const Rv rv(row, p.rows, p.V);
  const int rounds = ONE ? 1 : rounds_;
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wv = tid / kWave, mu = tid & (U - 1);
  float gm[NG], gs[NG];  // of each group: the largest, the sum of 2^(z sc - own_ref(largest))
  float m = kNegInf;
  if (tid == 0) sh.n = 0;
#pragma unroll
  for (int g = 0; g < NG; ++g) {
    gm[g] = kNegInf;
    gs[g] = 0.f;
    for (int r = 0; r < rounds; ++r) {
      const int base = (g * rounds + r) * U * BLK;
      if (base >= rv.ng) break;
      u32x4 w[1][U];
      float x[U][E], lm = kNegInf, ls = 0.f;
      rv.load({p.z}, base + tid, BLK, w);
      rv.unpack(w[0], x);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float um = x[u][0];
#pragma unroll
        for (int e = 1; e < E; ++e) um = fmaxf(um, x[u][e]);
        um = line_max<U>(um);
        const float at = own_ref(um, p.sc);
#pragma unroll
        for (int e = 0; e < E; ++e) x[u][e] = ex2(__builtin_fmaf(x[u][e], p.sc, -at));
        const float us = line_sum<U>(tree_sum(x[u]));
        lm = mu == u ? um : lm;
        ls = mu == u ? us : ls;
      }
      if (r == 0) {
        gm[g] = lm;
        gs[g] = ls;
      } else {
        const float nm = fmaxf(gm[g], lm), at = own_ref(nm, p.sc);
        gs[g] = gs[g] * ex2(own_ref(gm[g], p.sc) - at) + ls * ex2(own_ref(lm, p.sc) - at);
        gm[g] = nm;
      }
    }
    m = fmaxf(m, gm[g]);
  }
  m = block_max<WV>(m, sh.f);
  int n = CAP + 1;
  float s = 0.f, t = threshold<TI, WV>(gm, p.k, m, sh.f);
  RowRef rs = row_ref(t, p.sc), at;  // what is below t is summed against it
  bool tied = false, again = rs.steep;
  // the groups that reach t, in an order that does not depend on timing; the sums of the others
  int mine = 0;
#pragma unroll
  for (int g = 0; g < NG; ++g) {
    if (g * rounds * U * BLK + mu * BLK + tid - mu >= rv.ng) continue;
    if (gm[g] >= t)
      ++mine;
    else
      s += gs[g] * ex2(own_ref(gm[g], p.sc) - rs.msc);
  }
  int before = mine;
  for (int off = 1; off < kWave; off <<= 1) {
    const int o = __shfl_up(before, off, kWave);
    if (lane >= off) before += o;
  }
  if (lane == kWave - 1) sh.i[0][wv] = before;
  __syncthreads();
  int to = before - mine, nq = 0;
#pragma unroll
  for (int i = 0; i < WV; ++i) {
    if (i < wv) to += sh.i[0][i];
    nq += sh.i[0][i];
  }
  if (nq <= CAP) {
#pragma unroll
    for (int g = 0; g < NG; ++g)
      if (g * rounds * U * BLK + mu * BLK + tid - mu < rv.ng && gm[g] >= t) sh.queue[to++] = uint16_t(g * BLK + tid);
    __syncthreads();
    const int per = rounds * U;  // vectors of a group
    for (int j = tid; j < nq * per; j += BLK) {
      const int q = sh.queue[j / per], sub = j % per, qt = q % BLK, qu = qt % U;
      const int gi = (((q / BLK) * rounds + sub / U) * U + qu) * BLK + qt - qu + sub % U;
      if (gi >= rv.ng) continue;
      float x[E];
      TI::unpack(to_uint4(rv.load(p.z, gi)), x);
      uint32_t take = 0;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int v = rv.index(gi, e);
        if (x[e] >= t)
          take |= VEC || (v >= 0 && v < p.V) ? 1u << e : 0u;
        else
          s += ex2(__builtin_fmaf(x[e], rs.sc, -rs.msc));
      }
      add_candidates<TI>(sh, x, rv.index(gi, 0), take);
    }
    __syncthreads();
    n = int(sh.n);
  }
  if (n > CAP) {
    s = select_slowly<TI, VEC, BLK>(p, row, sh, t, tied);
    rs = row_ref(t, p.sc);
    again = false;
    n = p.k;
  }
  const float others = write_ranked<TI, BLK>(p, row, n, t, m, at, sh);
  write_rest<TI, VEC, BLK>(p, row, again ? others : rescaled(s, rs, at) + others, at, n == p.k && !tied, again, t, sh);
}

template <class TI, bool VEC, int U, int BLK, int NG, int CAP>
void rows_launch(const TopkArgs& a, const TopkParams& p, dim3 grid, int ng) {
  const int64_t round = int64_t(NG) * U * BLK;
  if (ng <= round)
    k_topk_rows<TI, VEC, U, BLK, NG, CAP, true><<<grid, BLK, 0, a.stream>>>(p, 1);
  else if constexpr (U * BLK == 2048)
    k_topk_rows<TI, VEC, U, BLK, NG, CAP, false><<<grid, BLK, 0, a.stream>>>(p, int((ng + round - 1) / round));
}

// Short lists of short rows take one wavefront a row, without barriers and
// with room for 320 candidates, so that 27 rows fit a CU; the others as many
// threads as the row fills with eight groups of four vectors.  us per call, against 512
// threads for every row: 14,336 rows of 8,000 bf16, k = 20, 139 -> 53; 4,096 of
// 16,032, k = 50, 54 -> 36; 4,096 of 32,000, k = 64, 68 -> 57 (128 threads: 59); 14,336 of
// 1,000, k = 8, 23 with all logits in registers.  256 threads of 16 groups and 1,024
// of 4 are slower at 14,336 rows of 128,256 (k = 64: 588 and 640 against 578).
template <class TI, bool VEC>
hipError_t launch_vec(const TopkArgs& a, int64_t row0, dim3 grid) {
  const TopkParams p{a.z, a.rows, row0, a.V, a.k, a.sc, a.inv_t, a.top, a.ids, a.rest};
  const int ng = a.V / TI::kVec + (VEC ? 0 : 2);  // vectors that cover a row, at most
  // lines of U vectors have to be several times k for few of them to reach the threshold
  auto lines = [&](int U) { return ng / U >= 3 * a.k; };
  const bool few = a.k <= 128;
  if (few && a.V <= 16 * 64)
    k_topk_short<TI, VEC, 64, 320><<<grid, 64, 0, a.stream>>>(p);
  else if (few && ng <= 1024 && lines(2))
    rows_launch<TI, VEC, 2, 64, 8, 320>(a, p, grid, ng);
  else if (few && ng <= 2048 && lines(4))
    rows_launch<TI, VEC, 4, 64, 8, 320>(a, p, grid, ng);
  else if (a.V <= 16 * 128)
    k_topk_short<TI, VEC, 128, 1024><<<grid, 128, 0, a.stream>>>(p);
  else if (a.V <= 16 * 256)
    k_topk_short<TI, VEC, 256, 1024><<<grid, 256, 0, a.stream>>>(p);
  else if (a.V <= 16 * 512)
    k_topk_short<TI, VEC, 512, 1024><<<grid, 512, 0, a.stream>>>(p);
  else if (ng <= 4096 && !lines(4))
    rows_launch<TI, VEC, 1, 512, 8, 1024>(a, p, grid, ng);
  else if (ng <= 8192)
    rows_launch<TI, VEC, 4, 256, 8, 1024>(a, p, grid, ng);
  else
    rows_launch<TI, VEC, 4, 512, 8, 1024>(a, p, grid, ng);
  return hipGetLastError();
}

template <class TI>
hipError_t launch_typed(const TopkArgs& a) {
  return for_row_parts(a.rows, [&](int64_t row0, unsigned n) {
    return a.V % TI::kVec == 0 ? launch_vec<TI, true>(a, row0, dim3(n)) : launch_vec<TI, false>(a, row0, dim3(n));
  });
}

}  // namespace

hipError_t launch_topk(const TopkArgs& a) {
  return a.in == DType::kBf16 ? launch_typed<Bf16>(a) : launch_typed<F32>(a);
}

}  // namespace aal
