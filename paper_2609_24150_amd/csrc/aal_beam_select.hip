// The n best continuations of each request's beams (aal_beam_select):
//
//   total[w, v] = scores[w] + z[w, v] / T - lse_w,   rank = total / length^length_penalty
//   order: larger rank, lower beam, larger logit, lower token
//
// Within a beam the order is the logits' own, so a row's n largest logits hold its candidates.  k_beam_parts
// cuts the rows into parts, one workgroup each, which keeps its part in registers, reads it once and
// leaves the part's n largest logits in order, its largest one and the sum of exp((z - that) / T).
// k_beam_merge, one workgroup per request, joins the parts' sums, forms every candidate's rank and chooses.
//
// Two beams' candidates may differ by less than 32 bits tell apart: totals are formed in 64 bits, and so is a
// row's log-sum-exp where it counts, the exponentials of the listed logits.  Those of the others are v_exp_f32's of
// arguments with one rounding (log2(e) / T in two pieces), whose errors average out over the many of them that it
// takes to bear on the sum; it is off by 2^-20 at most, and by no more can candidates of two beams be misjudged, those of
// one not at all.  Bound by that arithmetic where there are many rows: 13 instructions a logit, 64 x 8 rows of 128,256 bf16,
// 16 chosen, 31 us or 3.5 TB/s and 12 us to merge; by latency and the merge where there are few.  Parts are cut from the row's start whatever its alignment, so that equal rows
// get equal sums, and equal beams tie exactly.
#include "aal_beam.h"
#include "aal_device.h"
#include "aal_select.h"

#include <algorithm>
#include <limits>

namespace aal {
namespace {

constexpr int kCand = 1024;  // candidates of a part that fit: all entries of fewer than n vectors do
constexpr int kQueue = 512;  // and vectors that hold some (of 256, flat rows overran it now and then: 64 us instead of 36 for 7 x 32 x 50,001)
constexpr int kLists = 2048 + kBeamMax;  // a request's parts, and its beams: 64 rows of 2^18 fp32 in parts of 8,192
constexpr int kMerge = 512;       // threads of the merge
constexpr int kWork = 4096;       // candidates of a request that may reach the bound
constexpr int kSurvivors = 1024;  // candidates of a request that reach the bound

struct BeamParams {
  const void* z;
  int64_t rows, row0;  // B * W, the first one of the launch
  int W, V, n, parts, part_len;
  float sc_hi, sc_lo;  // log2(e) / T in two pieces
  double inv_t;
  const float* scores;
  const uint8_t* finished;
  const int32_t* lengths;
  double alpha;
  int32_t eos, pad;
  BeamOut out;
  BeamPart* part;      // [rows][parts]
  uint64_t* list;      // [rows][parts][n]: entry_of(), 0 where there is none
};

// A logit and its token as one whole number: larger for a larger logit, then for a lower token; never 0.
__device__ __forceinline__ uint64_t entry_of(uint32_t key, int v) { return uint64_t(key) << 32 | (0xffffffffu - uint32_t(v)); }
__device__ __forceinline__ int entry_token(uint64_t e) { return int(0xffffffffu - uint32_t(e)); }
template <class TI>
__device__ __forceinline__ float entry_logit(uint64_t e) { return key_logit<TI>(uint32_t(e >> 32)); }

// The same within a part (its elements have 14 bits), of a type that compares fast: 30 bits, or a double of
// 46 bits behind a one.
template <class TI>
struct LocalKey {
  using type = uint32_t;
  static __device__ __forceinline__ type of(uint32_t key, int at) { return key >> 2 | (0x3fffu - uint32_t(at)); }
  static __device__ __forceinline__ uint64_t entry(type k, int s0) {
    return entry_of((k << 2) & 0xffff0000u, s0 + int(0x3fffu - (k & 0x3fffu)));
  }
};
template <>
struct LocalKey<F32> {
  using type = double;
  static __device__ __forceinline__ type of(uint32_t key, int at) {
    return __builtin_bit_cast(double, 0x3ff0000000000000u | uint64_t(key) << 14 | uint64_t(0x3fffu - uint32_t(at)));
  }
  static __device__ __forceinline__ uint64_t entry(type k, int s0) {
    const uint64_t b = __builtin_bit_cast(uint64_t, k);
    return entry_of(uint32_t(b >> 14), s0 + int(0x3fffu - (uint32_t(b) & 0x3fffu)));
  }
};

template <int WAVES>
__device__ __forceinline__ int block_count(int wave_value, int* sh) {
  __syncthreads();
  if ((threadIdx.x & (kWave - 1)) == 0) sh[threadIdx.x / kWave] = wave_value;
  __syncthreads();
  int c = 0;
#pragma unroll
  for (int i = 0; i < WAVES; ++i) c += sh[i];
  return c;
}

typedef u32x4 u32x4_e2 __attribute__((aligned(2)));  // a vector at any element

// The sum over the wave in 64 bits, without LDS: rows of 16 lanes, then across them.
template <int Ctrl, int RowMask>
__device__ __forceinline__ double dpp_d(double v) {
  const uint64_t b = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = uint32_t(__builtin_amdgcn_update_dpp(0, int(uint32_t(b)), Ctrl, RowMask, 0xF, false));
  const uint32_t hi = uint32_t(__builtin_amdgcn_update_dpp(0, int(uint32_t(b >> 32)), Ctrl, RowMask, 0xF, false));
  return __builtin_bit_cast(double, uint64_t(hi) << 32 | lo);
}
__device__ __forceinline__ double wave_sum_dpp(double v) {
  v += dpp_d<0xB1, 0xF>(v);   // quad_perm [1,0,3,2]
  v += dpp_d<0x4E, 0xF>(v);   // quad_perm [2,3,0,1]
  v += dpp_d<0x141, 0xF>(v);  // row_half_mirror
  v += dpp_d<0x140, 0xF>(v);  // row_mirror
  v += dpp_d<0x142, 0xA>(v);  // row_bcast:15
  v += dpp_d<0x143, 0xC>(v);  // row_bcast:31
  const uint64_t b = __builtin_bit_cast(uint64_t, v);
  return __builtin_bit_cast(double, uint64_t(uint32_t(__builtin_amdgcn_readlane(int(uint32_t(b >> 32)), 63))) << 32 |
                                        uint32_t(__builtin_amdgcn_readlane(int(uint32_t(b)), 63)));
}

// The largest over the wave, alike.
template <int Ctrl, int RowMask>
__device__ __forceinline__ uint32_t dpp_max(uint32_t v) {
  return max(v, uint32_t(__builtin_amdgcn_update_dpp(0, int(v), Ctrl, RowMask, 0xF, false)));
}
__device__ __forceinline__ uint32_t wave_max_key(uint32_t v) {
  v = dpp_max<0x140, 0xF>(dpp_max<0x141, 0xF>(dpp_max<0x4E, 0xF>(dpp_max<0xB1, 0xF>(v))));
  v = dpp_max<0x143, 0xC>(dpp_max<0x142, 0xA>(v));
  return uint32_t(__builtin_amdgcn_readlane(int(v), 63));
}

// A value that all lanes have, as one of the wave.
__device__ __forceinline__ float uniform(float x) {
  return __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, x)));
}

// The vector stays packed here: unpacked copies are not kept for later.
__device__ __forceinline__ void pin(u32x4& x) { asm volatile("" : "+v"(x)); }

// Vectors stay packed, 32 registers of them, and are unpacked where they are used: eight workgroups
// of 256 a CU, whose selections run under the others' loads and sums.
template <class TI, int BLK, int U>
__global__ __launch_bounds__(BLK, 7) void k_beam_parts(BeamParams p) {
  constexpr int E = TI::kVec, WV = BLK / kWave;
  constexpr int kShift = 32 - key_bits<TI>();
  using Key = LocalKey<TI>;
  __shared__ __attribute__((aligned(16))) typename Key::type cand[kCand];
  __shared__ double dsum[WV];
  __shared__ float fsh[WV];
  __shared__ int ish[WV];
  __shared__ __attribute__((aligned(16))) u32x4 queue[kQueue];
  static_assert(sizeof(queue) >= kCand * sizeof(uint64_t), "the sorted candidates take the queue's place");
  uint64_t* sorted = reinterpret_cast<uint64_t*>(queue);
  __shared__ int place[kQueue];
  __shared__ int count, vectors;
  const int64_t row = p.row0 + blockIdx.x / p.parts;
  const int part = blockIdx.x % p.parts, tid = threadIdx.x, lane = tid & (kWave - 1), wv = tid / kWave;
  if ((p.finished && p.finished[row]) || p.scores[row] == kNegInf) return;
  const int s0 = part * p.part_len, len = min(p.part_len, p.V - s0);
  const typename TI::storage* base = static_cast<const typename TI::storage*>(p.z) + row * int64_t(p.V) + s0;
  if (tid == 0) count = vectors = 0;
  u32x4 raw[U];
  float gm[U], m = kNegInf;
  auto vector = [&](int u) {
    const int at = (u * BLK + tid) * E;
    if (at + E <= len) return u32x4(__builtin_nontemporal_load(reinterpret_cast<const u32x4_e2*>(base + at)));
    typename TI::storage v[E];
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = at + e < len ? base[at + e] : TI::neg_inf();
    u32x4 w;
    __builtin_memcpy(&w, v, 16);
    return w;
  };
#pragma unroll
  for (int u = 0; u < U; ++u) raw[u] = vector(u);
#pragma unroll
  for (int u = 0; u < U; ++u) {
    float x[E];
    TI::unpack(to_uint4(raw[u]), x);
    gm[u] = x[0];
#pragma unroll
    for (int e = 1; e < E; ++e) gm[u] = fmaxf(gm[u], x[e]);
    m = fmaxf(m, gm[u]);
  }
#pragma unroll
  for (int u = 0; u < U; ++u) pin(raw[u]);
  // how many threads and how many vectors have something finite, by waves
  const float own[1] = {m};
  const int threads = __popcll(__builtin_amdgcn_ballot_w64(m != kNegInf));
  int groups = 0, all = 0;
#pragma unroll
  for (int u = 0; u < U; ++u) groups += __popcll(__builtin_amdgcn_ballot_w64(gm[u] != kNegInf));
  m = wave_max(m);
  if (lane == 0) {
    fsh[wv] = m;
    ish[wv] = groups << 16 | threads;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < WV; ++i) {
    m = fmaxf(m, fsh[i]);
    all += ish[i];
  }
  all = __builtin_amdgcn_readfirstlane(all);
  m = uniform(m);
  __syncthreads();
  const int64_t slot = row * int64_t(p.parts) + part;
  uint64_t* list = p.list + slot * p.n;
  if (m == kNegInf) {
    for (int i = tid; i < p.n; i += BLK) list[i] = 0;
    if (tid == 0) p.part[slot] = {0.0, kNegInf, 0};
    return;
  }
  // At least n logits reach t, or all finite ones do.  Threads' maxima do for short lists, an eighth of the
  // arithmetic; for more than a quarter of the threads they would let through half again as many.  A wave's share of n is
  // that of the finite maxima that it has: with equal shares a wave without any would let all of a short row through
  // (51 x 4 rows of 688: 102 us instead of 21, calls and all).
  float t = kNegInf;
  if (p.n <= BLK / 4 && (all & 0xffff) >= p.n)
    t = threshold_of_shares<TI, WV>(own, (p.n * threads + (all & 0xffff) - 1) / (all & 0xffff), m, fsh);
  else if ((all >> 16) >= p.n)
    t = threshold_of_shares<TI, WV>(gm, (p.n * groups + (all >> 16) - 1) / (all >> 16), m, fsh);
  t = uniform(t);
  // the vectors that hold some, then their entries, each by a thread of its own
  auto collect = [&](float from) {
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (gm[u] >= from && gm[u] != kNegInf) {
        const int at = atomicAdd(&vectors, 1);
        if (at < kQueue) {
          queue[at] = raw[u];
          place[at] = (u * BLK + tid) * E;
        }
      }
    __syncthreads();
    const int q = vectors;
    for (int i = tid; i < min(q, kQueue) * E; i += BLK) {
      const int e = i % E;
      const float x = TI::load1(&queue[i / E], e);
      if (x >= from && x != kNegInf) {
        const int at = atomicAdd(&count, 1);
        if (at < kCand) cand[at] = Key::of(order_key<TI>(x), place[i / E] + e);
      }
    }
    __syncthreads();
    return q > kQueue ? kCand + 1 : count;
  };
  int c = collect(t), left_ties = 0;
#pragma unroll
  for (int u = 0; u < U; ++u) pin(raw[u]);
  if (c > kCand) {
    // ties or clusters: the n-th largest logit itself, what lies above it and the first of its ties; the
    // part is read again, so that the common way keeps its registers.  Compared as whole numbers, which
    // order NaN too: no entry is listed twice, whatever the logits are.
    uint32_t lo = order_key<TI>(kNegInf) >> kShift, hi = (order_key<TI>(m) >> kShift) + 1u;
    while (hi > lo + 1u) {
      const uint32_t mid = lo + (hi - lo) / 2;
      const uint32_t f = mid << kShift;
      int reach = 0;
#pragma unroll 1
      for (int u = 0; u < U; ++u) {
        float x[E];
        TI::unpack(to_uint4(vector(u)), x);
#pragma unroll
        for (int e = 0; e < E; ++e) reach += __popcll(__builtin_amdgcn_ballot_w64(order_key<TI>(x[e]) >= f));
      }
      (block_count<WV>(reach, ish) >= p.n ? lo : hi) = mid;
    }
    const uint32_t bar = lo << kShift;
    t = uniform(key_logit<TI>(bar));
    if (tid == 0) count = 0;
    __syncthreads();
    int ties = 0;  // before this vector's turn
#pragma unroll 1
    for (int u = 0; u < U; ++u) {
      float x[E];
      TI::unpack(to_uint4(vector(u)), x);
      int mine = 0;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const uint32_t key = order_key<TI>(x[e]);
        mine += key == bar;
        if (key > bar) {  // fewer than n of them, NaN aside
          const int at = atomicAdd(&count, 1);
          if (at < p.n) cand[at] = Key::of(key, (u * BLK + tid) * E + e);
        }
      }
      int before = mine;
      for (int off = 1; off < kWave; off <<= 1) {
        const int o = __shfl_up(before, off, kWave);
        if (lane >= off) before += o;
      }
      __syncthreads();
      if (lane == kWave - 1) ish[wv] = before;
      __syncthreads();
      int at = ties + before - mine;
#pragma unroll
      for (int i = 0; i < WV; ++i) {
        if (i < wv) at += ish[i];
        ties += ish[i];
      }
      // the first n ties, from the end of the list down
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (order_key<TI>(x[e]) == bar) {
          if (at < p.n) cand[kCand - 1 - at] = Key::of(bar, (u * BLK + tid) * E + e);
          ++at;
        }
    }
    __syncthreads();
    c = min(count, p.n);
    const int taken = t != kNegInf ? min(p.n - c, ties) : 0;
    left_ties = t != kNegInf ? ties - taken : 0;
    typename Key::type tie{};
    if (tid < taken) tie = cand[kCand - 1 - tid];
    __syncthreads();
    if (tid < taken) cand[c + tid] = tie;
    c += taken;
    __syncthreads();
  }
  for (int i = tid; i < c; i += BLK) {
    const auto mine = cand[i];
    int rank = 0;
    int j = 0;
    for (; j + 8 <= c; j += 8)
#pragma unroll
      for (int k = 0; k < 8; ++k) rank += cand[j + k] > mine;
    for (; j < c; ++j) rank += cand[j] > mine;
    sorted[rank] = Key::entry(mine, s0);
  }
  // The others' sum of 2^((z - m) sc), sc in two pieces.  z sc_hi - ref takes one rounding, and so does adding
  // z sc_lo; what ref, m sc rounded, is off by is a factor of the whole sum and joins it in 64 bits.
  // References beyond 2^27 take the difference first.
  const float ref = m * p.sc_hi;
  const bool steep = __builtin_amdgcn_readfirstlane(fabsf(ref) > 0x1p27f) != 0;
  auto weight = [&](float z, bool by_difference) {
    const float d = z - m;
    return ex2(by_difference ? __builtin_fmaf(d, p.sc_hi, d * p.sc_lo)
                             : __builtin_fmaf(z, p.sc_lo, __builtin_fmaf(z, p.sc_hi, -ref)));
  };
  // without a branch in it: what is listed counts as -inf
  auto weights = [&](const u32x4& w, bool listed, bool by_difference) {
    float x[E], us = 0.f;
    TI::unpack(to_uint4(w), x);
    if (listed)
#pragma unroll
      for (int e = 0; e < E; ++e) x[e] = x[e] < t ? x[e] : kNegInf;
#pragma unroll
    for (int e = 0; e < E; ++e) us += weight(x[e], by_difference);
    return us;
  };
  float s = 0.f;
  if (steep) {
#pragma unroll 1
    for (int u = 0; u < U; ++u) s += weights(vector(u), true, true);
  } else {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      s += weights(raw[u], __builtin_amdgcn_ballot_w64(gm[u] >= t) != 0, false);
      __builtin_amdgcn_sched_barrier(0);  // not all vectors unpacked at once
    }
  }
  if (tid == 0 && left_ties) s += float(left_ties) * weight(t, steep);
  __syncthreads();
  double total = double(s);
  for (int i = tid; i < c; i += BLK)
    if (i >= p.n) total += double(weight(entry_logit<TI>(sorted[i]), steep));
  if (!steep) total *= exp2(double(ref) - double(m) * (double(p.sc_hi) + double(p.sc_lo)));
  for (int i = tid; i < p.n; i += BLK) {
    list[i] = i < c ? sorted[i] : 0;
    if (i < c) total += exp((double(entry_logit<TI>(sorted[i])) - double(m)) * p.inv_t);
  }
  total = wave_sum_dpp(total);
  if (lane == 0) dsum[wv] = total;
  __syncthreads();
  if (tid == 0) {
    total = dsum[0];
    for (int i = 1; i < WV; ++i) total += dsum[i];
    p.part[slot] = {total, m, 0};
  }
}

// What orders candidates of equal rank, the larger first: the lower beam, then the larger entry (a token has 18 bits).
__device__ __forceinline__ uint64_t tie_of(int w, uint64_t e) {
  return uint64_t(kBeamMax - 1 - w) << 50 | (e >> 32) << 18 | (uint32_t(e) & 0x3ffffu);
}
__device__ __forceinline__ int tie_beam(uint64_t t) { return kBeamMax - 1 - int(t >> 50); }
__device__ __forceinline__ uint64_t tie_entry(uint64_t t) {
  return (t >> 18) << 32 | 0xfffc0000u | (uint32_t(t) & 0x3ffffu);
}
// A rank as a whole number of the same order, -0 as +0; NaN has a place in it too, so that any inputs
// end in a choice of existing beams and tokens.
__device__ __forceinline__ uint64_t rank_key(double r) {
  const uint64_t b = __builtin_bit_cast(uint64_t, r + 0.0);
  return b ^ (uint64_t(int64_t(b) >> 63) | uint64_t(1) << 63);
}
__device__ __forceinline__ double key_rank(uint64_t k) {
  return __builtin_bit_cast(double, k ^ (k >> 63 ? uint64_t(1) << 63 : ~uint64_t(0)));
}
struct alignas(16) Candidate {
  uint64_t rank;  // rank_key()
  uint64_t tie;   // never 0
};
// without branches: both are read at once
__device__ __forceinline__ bool before(const Candidate& a, const Candidate& b) {
  return (a.rank > b.rank) | ((a.rank == b.rank) & (a.tie > b.tie));
}

// The lists of a request and, behind them, the beams that have ended as lists of one.
//
// Of lists in order, the r-th largest of their entries number i is reached by r i candidates at least: with r i >= n a
// bound below which nothing is chosen.  A wave each finds it for i = 1, 2, 4, ..., in 32 bits, which keep ranks'
// order up to ties; the largest bound leaves little more than n candidates, which are ranked by counting.
template <class TI>
__global__ __launch_bounds__(kMerge) void k_beam_merge(BeamParams p, int64_t b0) {
  constexpr int NT = kMerge, WV = NT / kWave, R = 4;
  static_assert(WV == 8, "a wave for each i up to 128");
  __shared__ double lse[kBeamMax], factor[kBeamMax], inverse[kBeamMax], score[kBeamMax];
  __shared__ int state[kBeamMax];  // 0 goes on, 1 has ended, 2 has score -inf
  __shared__ Candidate chosen[kSurvivors];
  __shared__ __attribute__((aligned(16))) uint32_t keys[kSurvivors];
  __shared__ int taken[kSurvivors];
  __shared__ uint16_t place[kSurvivors];
  __shared__ uint32_t heads[WV][kLists];
  __shared__ uint32_t work[kWork];
  __shared__ uint32_t bound;
  __shared__ int count, items;
  const int64_t b = b0 + blockIdx.x, row0 = b * p.W;
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wv = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int per = p.parts * p.n, C = p.W * per, L = p.W * p.parts;
  const uint64_t* lists = p.list + row0 * per;
  // the first lists' entries number i, before anything is known of their beams: one way to memory less to wait for
  const int number = 1 << wv;
  uint64_t early[R];
#pragma unroll
  for (int q = 0; q < R; ++q) {
    const int k = q * kWave + lane;
    early[q] = number <= p.n && k < L ? lists[k * p.n + number - 1] : 0;
  }
  if (tid == 0) {
    count = items = 0;
    bound = 1u;
  }
  // as many lanes to a beam as its parts ask for and the workgroup has
  int g = 1;
  while (g < kWave && g < p.parts && 2 * g * p.W <= NT) g <<= 1;
  for (int w0 = 0; w0 < p.W; w0 += NT / g) {
    const int w = w0 + tid / g, sub = tid % g;
    if (w >= p.W) continue;
    const float sw = p.scores[row0 + w];
    const bool done = p.finished && p.finished[row0 + w];
    const int len = p.lengths ? p.lengths[row0 + w] : 0;
    const int st = sw == kNegInf ? 2 : done ? 1 : 0;
    const BeamPart* part = p.part + (row0 + w) * p.parts;  // unspecified where the beam does not go on
    float m = kNegInf;
    for (int i = sub; i < p.parts; i += g) m = fmaxf(m, part[i].m);
    for (int off = 1; off < g; off <<= 1) m = fmaxf(m, __shfl_xor(m, off, kWave));
    double s = 0.0;
    if (st == 0 && m != kNegInf)
      for (int i = sub; i < p.parts; i += g)
        if (part[i].m != kNegInf) s += part[i].s * exp((double(part[i].m) - double(m)) * p.inv_t);
    for (int off = 1; off < g; off <<= 1) s += __shfl_xor(s, off, kWave);
    if (sub == 0) {
      lse[w] = st == 0 && m != kNegInf ? double(m) * p.inv_t + log(s) : 0.0;
      score[w] = double(sw);
      state[w] = st;
      factor[w] = p.alpha != 0.0 ? pow(double(len) + double(st == 0), p.alpha) : 1.0;
      inverse[w] = 1.0 / factor[w];
    }
  }
  __syncthreads();
  auto total_of = [&](int w, uint64_t e) {
    return state[w] == 1 ? score[w] : double(entry_logit<TI>(e)) * p.inv_t - lse[w] + score[w];
  };
  auto rank_of = [&](int w, uint64_t e) {
    const double t = total_of(w, e);
    return p.alpha != 0.0 ? t / factor[w] : t;
  };
  // the rank without its division, in 32 bits; never below the next lower key than rank_of()'s
  auto key_of = [&](int w, uint64_t e) { return order_key<F32>(float(total_of(w, e) * inverse[w])); };
  const float per_list = 1.f / float(p.parts);
  auto beam_of = [&](int k) { return int((float(k) + 0.5f) * per_list); };  // k / parts: k is under 2^12
  auto head = [&](int k, uint64_t e) {
    const int w = beam_of(k);
    return k < L && e != 0 && state[w] == 0 ? key_of(w, e) : 0u;
  };
  if (number <= p.n) {
    uint32_t key[R], ended = 0, top = 0;
    if (wv == 0 && lane < p.W && state[lane] == 1) ended = key_of(lane, 1);
#pragma unroll
    for (int q = 0; q < R; ++q) {
      const int k = q * kWave + lane;
      key[q] = head(k, early[q]);
      if (k < L) heads[wv][k] = key[q];
      top = max(top, key[q]);
    }
    for (int k = R * kWave + lane; k < L; k += kWave) {
      const uint32_t more = head(k, lists[k * p.n + number - 1]);
      heads[wv][k] = more;
      top = max(top, more);
    }
    top = wave_max_key(max(top, ended));
    const int r = (p.n + number - 1) / number, enough = r + r / 8;
    uint32_t lo = 0u, hi = top + 1u;  // lo is reached by r or is 0
    while (hi > lo + 1u) {
      const uint32_t mid = lo + (hi - lo) / 2;
      int c = __popcll(__builtin_amdgcn_ballot_w64(ended >= mid));
#pragma unroll
      for (int q = 0; q < R; ++q) c += __popcll(__builtin_amdgcn_ballot_w64(key[q] >= mid));
      for (int k = R * kWave; k < L; k += kWave)
        c += __popcll(__builtin_amdgcn_ballot_w64(k + lane < L && heads[wv][k + lane] >= mid));
      if (c >= r) {
        lo = mid;
        if (c <= enough) break;
      } else {
        hi = mid;
      }
    }
    if (lane == 0) atomicMax(&bound, lo);
  }
  __syncthreads();
  const uint32_t least = bound > 2u ? bound - 2u : 1u;  // two keys less: what multiplying may be off by
  // of a list whose entries 1, 2, 4, ..., 2^(j - 1) reach the bound, the first 2^j - 1 may
  for (int l = tid; l < L; l += NT) {
    int j = 0;
    while ((1 << j) <= p.n && heads[j][l] >= least) ++j;
    if (j == 0) continue;
    const int eights = (min(p.n, (1 << j) - 1) + 7) / 8;
    int at = atomicAdd(&items, eights);
    for (int i = 0; i < eights; ++i, ++at)
      if (at < kWork) work[at] = uint32_t(l) << 4 | uint32_t(i);
  }
  __syncthreads();
  auto consider = [&](int w, uint64_t e) {
    if (e == 0 || key_of(w, e) < least) return;
    const int at = atomicAdd(&count, 1);
    if (at < kSurvivors) chosen[at] = {rank_key(rank_of(w, e)), tie_of(w, e)};
  };
  // candidate i's beam and entry; false where there is none
  auto candidate = [&](int i, int& w, uint64_t& e) {
    if (i < C) {
      w = i / per;
      if (state[w] != 0) return false;
      e = lists[i];
      return e != 0;
    }
    w = i - C;
    e = 1;
    return w < p.W && state[w] == 1;
  };
  if (items <= kWork) {
    for (int i = tid; i < items * 8; i += NT) {
      const int l = int(work[i / 8] >> 4), k = int(work[i / 8] & 15u) * 8 + i % 8, w = beam_of(l);
      if (k < p.n && state[w] == 0) consider(w, lists[l * p.n + k]);
    }
    if (tid < p.W && state[tid] == 1) consider(tid, 1);
  } else {
    for (int i = tid; i < C + p.W; i += NT) {
      int w;
      uint64_t e;
      if (candidate(i, w, e)) consider(w, e);
    }
  }
  __syncthreads();
  const int c = count;
  const int64_t o = b * p.n;
  auto write = [&](int j, const Candidate& c) {
    const int w = tie_beam(c.tie);
    const uint64_t e = tie_entry(c.tie);
    const bool done = state[w] == 1;
    const int token = done ? p.pad : entry_token(e);
    p.out.parents[o + j] = w;
    p.out.tokens[o + j] = token;
    if (p.out.scores) p.out.scores[o + j] = float(total_of(w, e));
    if (p.out.rank) p.out.rank[o + j] = float(key_rank(c.rank));
    if (p.out.finished) p.out.finished[o + j] = done || token == p.eos;
    if (p.out.lengths) p.out.lengths[o + j] = (p.lengths ? p.lengths[row0 + w] : 0) + !done;
  };
  if (c <= kSurvivors) {
    // counted by their 32-bit keys; those that share one, by what they are: found through a chain of them, or, of many,
    // among all (the next one of a chain is known when this one has been read)
    int *first = reinterpret_cast<int*>(heads[0]), *following = reinterpret_cast<int*>(heads[1]);
    for (int i = tid; i < c; i += NT) keys[i] = order_key<F32>(float(key_rank(chosen[i].rank)));
    for (int i = c + tid; i < ((c + 15) & ~15); i += NT) keys[i] = 0u;
    for (int i = tid; i < c; i += NT) {
      taken[i] = 0;
      first[i] = -1;
    }
    __syncthreads();
    // as many threads to one as there are
    const int g = c <= NT / 8 ? 8 : c <= NT / 4 ? 4 : c <= NT / 2 ? 2 : 1;
    for (int i = tid / g; i < c; i += NT / g) {
      const uint32_t mine = keys[i];
      int at = 0;
      for (int j = tid % g * 16; j < c; j += g * 16)
#pragma unroll
        for (int k = 0; k < 16; ++k) at += keys[j + k] > mine;
      for (int off = 1; off < g; off <<= 1) at += __shfl_xor(at, off, kWave);
      if (tid % g == 0) {
        place[i] = uint16_t(at);
        atomicAdd(&taken[at], 1);
        following[i] = atomicExch(&first[at], i);
      }
    }
    __syncthreads();
    for (int i = tid; i < c; i += NT) {
      const Candidate mine = chosen[i];
      int at = place[i];
      if (at >= p.n) continue;
      const int alike = taken[at];
      if (alike > 1 && alike <= 16) {
        for (int j = first[at], k = 0; k < alike; ++k, j = following[j]) at += before(chosen[j], mine);
      } else if (alike > 1) {
        const uint32_t key = keys[i];
        for (int j = 0; j < c; j += 8) {
          uint32_t same = 0;
#pragma unroll
          for (int k = 0; k < 8; ++k) same |= keys[j + k] == key ? 1u << k : 0u;
          for (; same; same &= same - 1u) at += before(chosen[j + __builtin_ctz(same)], mine);
        }
      }
      if (at < p.n) write(at, mine);
    }
  } else {
    // too many that the bound does not tell apart (rows of equal logits): one after the other
    Candidate last{~uint64_t(0), ~uint64_t(0)};
    for (int found = 0; found < p.n; ++found) {
      Candidate best{0, 0};
      for (int i = tid; i < C + p.W; i += NT) {
        int w;
        uint64_t e;
        if (!candidate(i, w, e)) continue;
        const Candidate c{rank_key(rank_of(w, e)), tie_of(w, e)};
        if (before(last, c) && before(c, best)) best = c;
      }
      for (int off = 32; off > 0; off >>= 1) {
        const Candidate c{uint64_t(__shfl_xor((unsigned long long)best.rank, off, kWave)),
                          uint64_t(__shfl_xor((unsigned long long)best.tie, off, kWave))};
        if (before(c, best)) best = c;
      }
      __syncthreads();
      if (lane == 0) chosen[wv] = best;
      __syncthreads();
      for (int i = 0; i < WV; ++i)
        if (before(chosen[i], best)) best = chosen[i];
      last = best;
      if (tid == 0) write(found, best);
    }
  }
  for (int j = min(c, p.n) + tid; j < p.n; j += NT) {
    p.out.parents[o + j] = -1;
    p.out.tokens[o + j] = p.pad;
    if (p.out.scores) p.out.scores[o + j] = kNegInf;
    if (p.out.rank) p.out.rank[o + j] = kNegInf;
    if (p.out.finished) p.out.finished[o + j] = 1;
    if (p.out.lengths) p.out.lengths[o + j] = 0;
  }
}

// How rows are cut: vectors per thread of a part's workgroup, parts of a row.  The longest parts of which there are 64:
// more of them are read sooner, and are more lists for a request's merge, the longer way of the two.  1 x 32 rows of 50,001 fp32,
// 64 chosen: 20 us, 26 where 256 parts are wanted, 65 where 1,024 are; 7 x 32 of bf16, 128 chosen, 33.6 against 36.4; 1 x 4
// of 128,256 bf16, 8 chosen: 14 us, 17 in parts of the greatest length.
struct Cut {
  int u, parts, len;
};
Cut cut_rows(DType in, int64_t B, int W, int V) {
  const int E = in == DType::kBf16 ? 8 : 4;
  for (int u = 8;; u /= 2) {
    const int most = 256 * u * E, parts = (V + most - 1) / most;
    const int len = ((V + parts - 1) / parts + E - 1) / E * E;
    const Cut c{u, (V + len - 1) / len, len};
    if (u == 1 || B * W * c.parts >= 64 || 2 * W * c.parts + kBeamMax > kLists) return c;
  }
}

template <class TI>
hipError_t launch_typed(const BeamArgs& a) {
  const Cut c = cut_rows(a.in, a.B, a.W, a.V);
  BeamParams p{};
  p.z = a.z;
  p.rows = a.B * a.W;
  p.W = a.W;
  p.V = a.V;
  p.n = a.n;
  p.parts = c.parts;
  p.part_len = c.len;
  p.inv_t = 1.0 / double(a.temperature);
  // the lower piece is above 0, so that a logit of -inf is no NaN; from T = 2^120 on it may be less than half of the
  // least fp32 number, which stands for it then: 2^-150 of a logit, 2^-22 at most, more in an exponent
  const double sc = 1.4426950408889634073599246810019 / double(a.temperature);
  p.sc_hi = float(sc);
  if (double(p.sc_hi) >= sc) p.sc_hi = __builtin_nextafterf(p.sc_hi, 0.f);
  p.sc_lo = std::max(float(sc - double(p.sc_hi)), std::numeric_limits<float>::denorm_min());
  p.scores = a.scores;
  p.finished = a.finished;
  p.lengths = a.lengths;
  p.alpha = double(a.length_penalty);
  p.eos = a.eos;
  p.pad = a.pad;
  p.out = a.out;
  p.part = static_cast<BeamPart*>(a.ws);
  p.list = reinterpret_cast<uint64_t*>(static_cast<uint8_t*>(a.ws) + align256(size_t(p.rows) * c.parts * sizeof(BeamPart)));
  // a launch holds fewer than 2^32 threads
  const int64_t most = (int64_t(1) << 21) / c.parts;
  for (; p.row0 < p.rows; p.row0 += most) {
    const dim3 grid(unsigned((p.rows - p.row0 < most ? p.rows - p.row0 : most) * c.parts));
    if (c.u == 8)
      k_beam_parts<TI, 256, 8><<<grid, 256, 0, a.stream>>>(p);
    else if (c.u == 4)
      k_beam_parts<TI, 256, 4><<<grid, 256, 0, a.stream>>>(p);
    else if (c.u == 2)
      k_beam_parts<TI, 256, 2><<<grid, 256, 0, a.stream>>>(p);
    else
      k_beam_parts<TI, 256, 1><<<grid, 256, 0, a.stream>>>(p);
  }
  for (int64_t b0 = 0; b0 < a.B; b0 += int64_t(1) << 21)
    k_beam_merge<TI><<<dim3(unsigned(a.B - b0 < (int64_t(1) << 21) ? a.B - b0 : int64_t(1) << 21)), kMerge, 0, a.stream>>>(p, b0);
  return hipGetLastError();
}

}  // namespace

size_t beam_workspace_bytes(DType in, int64_t B, int W, int V, int n) {
  const Cut c = cut_rows(in, B, W, V);
  const size_t slots = size_t(B) * size_t(W) * size_t(c.parts);
  return align256(slots * sizeof(BeamPart)) + align256(slots * size_t(n) * sizeof(uint64_t));
}

hipError_t launch_beam_select(const BeamArgs& a) {
  return a.in == DType::kBf16 ? launch_typed<Bf16>(a) : launch_typed<F32>(a);
}

}  // namespace aal
