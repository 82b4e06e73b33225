// A row's k largest logits with their ids, and the log-sum-exp of the others
// (aal_topk_logits): what a training set stores of a target's logits.
//
//   order: v before w iff z_v > z_w, or z_v = z_w and v < w
//   rest  = ln sum_{v not among the k} exp(z_v / T)
//
// One workgroup per row.  k_topk_rows reads the row once: a thread cuts its
// vectors into eight groups and keeps of each the largest logit and the sum
// of 2^(z sc - that) in registers.  k groups hold a logit at least as large as
// the k-th largest of the groups' maxima, so a threshold t that k to 1.25 k + 16
// maxima reach (found by bisection over whole numbers that order as logits,
// one ballot count per group and step) is passed by all of the k largest and
// by few others; the groups that reach t, a few hundred vectors, are read
// again, their entries from t on are ranked by counting.  The remainder is the sum of
// the groups below t and of the entries not taken: never a difference of sums.
// k_topk_short, for rows of up to 16 logits per thread, bisects over the logits.
// Where ties put more entries at t than the candidates' list holds (rows of
// few distinct values), the workgroup takes select_slowly, a radix select
// over the row that is right for everything.
#include "aal_device.h"
#include "aal_rowops.h"
#include "aal_toplist.h"

namespace aal {
namespace {

constexpr int kTopkMax = 512;
constexpr int kCap = 1024;     // candidates, and groups read again
constexpr int kGroups = 8;     // groups of a thread
constexpr float kLn2 = 0.693147180559945309417f;

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

struct TopkShared {
  alignas(16) uint64_t cand[kCap];    // (key, ~index) of the candidates
  alignas(16) uint64_t sorted[kCap];  // the same by rank
  uint16_t queue[kCap];               // groups read again
  uint32_t hist[256];
  float f[16];
  int i[2][16];
  uint32_t n, digit, need;
};

struct TopkParams {
  const void* z;
  int64_t rows;
  int V, k;
  float sc;
  void* top;
  int32_t* ids;
  float* rest;
};

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

// The number of the block's keys (N per thread) that reach t, to every thread.
// `turn` alternates between calls.
template <int WAVES, int N>
__device__ __forceinline__ int count_from(const uint32_t (&key)[N], uint32_t t, int (*sh)[16], int turn) {
  int c = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) c += __popcll(__builtin_amdgcn_ballot_w64(key[i] >= t));
  if constexpr (WAVES == 1) return c;
  if ((threadIdx.x & (kWave - 1)) == 0) sh[turn][threadIdx.x / kWave] = c;
  __syncthreads();
  c = 0;
#pragma unroll
  for (int i = 0; i < WAVES; ++i) c += sh[turn][i];
  return c;
}

// A threshold that at least `k` of the block's keys reach, and at most k + k/4
// + 16 unless ties forbid it; `top` is the largest key.  Keys of 0 are none.
template <class TI, int WAVES, int N>
__device__ __forceinline__ uint32_t threshold(const uint32_t (&key)[N], int k, uint32_t top, int (*sh)[16]) {
  constexpr int kShift = 32 - key_bits<TI>();
  uint32_t lo = 0, hi = (top >> kShift) + 1u;  // lo is reached by k keys or all, hi by none (1 past the top)
  const int most = k + k / 4 + 16;
  int turn = 0;
  // the first probe two octaves below the top, where k keys mostly are above: less to bisect
  uint32_t probe = hi > (2u << (23 - kShift)) ? hi - (2u << (23 - kShift)) : hi / 2;
  while (hi - lo > 1u) {
    const int c = count_from<WAVES>(key, probe << kShift, sh, turn);
    turn ^= 1;
    if (c >= k) {
      lo = probe;
      if (c <= most) break;
    } else {
      hi = probe;
    }
    probe = lo + (hi - lo) / 2;
  }
  __syncthreads();
  return lo << kShift;
}

// Ranks the n >= k candidates, writes the first k and returns the sum of 2^(z sc - msc) over
// the others (this thread's share).
template <class TI, int BLK>
__device__ __forceinline__ float write_ranked(const TopkParams& p, int64_t row, int n, float msc, TopkShared& sh) {
  const int even = (n + 1) & ~1;
  if (threadIdx.x == 0 && even != n) sh.cand[n] = 0;  // below every candidate
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += BLK) {
    const uint64_t mine = sh.cand[i];
    int rank = 0;
    for (int j = 0; j < even; j += 2) {
      const ulonglong2 two = *reinterpret_cast<const ulonglong2*>(&sh.cand[j]);
      rank += (two.x > mine) + (two.y > mine);
    }
    sh.sorted[rank] = mine;
  }
  __syncthreads();
  const int64_t e0 = row * int64_t(p.V), o0 = row * int64_t(p.k);
  float s = 0.f;
  for (int j = threadIdx.x; j < n; j += BLK) {
    const uint64_t key = sh.sorted[j];
    if (j < p.k) {
      const int v = int(0xffffffffu - uint32_t(key));
      p.ids[o0 + j] = v;
      static_cast<typename TI::storage*>(p.top)[o0 + j] = static_cast<const typename TI::storage*>(p.z)[e0 + v];
    } else {
      s += ex2(__builtin_fmaf(key_logit<TI>(uint32_t(key >> 32)), p.sc, -msc));
    }
  }
  return s;
}

__device__ __forceinline__ void add_candidate(TopkShared& sh, uint32_t key, int v) {
  const uint32_t slot = atomicAdd(&sh.n, 1u);
  if (slot < uint32_t(kCap)) sh.cand[slot] = (uint64_t(key) << 32) | (0xffffffffu - uint32_t(v));
}

// Any row: the k-th largest key digit by digit, then a pass in index order that
// collects the larger entries and the first of its ties.  Returns this thread's share of the
// others' sum of 2^(z sc - msc).
template <class TI, bool VEC, int BLK>
__device__ __attribute__((noinline)) float select_slowly(const TopkParams& p, int64_t row, float msc, TopkShared& sh) {
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
  if (tid == 0) sh.n = 0;
  uint32_t ties = 0;  // before this round
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
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int v = rv.index(gi, e);
      if (v < 0 || v >= p.V) continue;
      const bool tie = key[e] == prefix;
      if (key[e] > prefix || (tie && at < need))
        add_candidate(sh, key[e], v);
      else
        s += ex2(__builtin_fmaf(x[e], p.sc, -msc));
      at += tie;
    }
  }
  __syncthreads();
  return s;
}

template <int WAVES>
__device__ __forceinline__ void write_rest(const TopkParams& p, int64_t row, float s, float msc, TopkShared& sh) {
  if (p.rest == nullptr) return;
  s = block_sum<WAVES>(s, sh.f);
  if (threadIdx.x == 0) p.rest[row] = s > 0.f ? (msc + __log2f(s)) * kLn2 : kNegInf;
}

// Rows of up to 16 BLK logits: all of them in registers.
template <class TI, bool VEC, int BLK>
__global__ __launch_bounds__(BLK) void k_topk_short(TopkParams p) {
  using Rv = RowVecs<TI, VEC>;
  constexpr int E = Rv::E;
  constexpr int WV = BLK / kWave;
  constexpr int U = 16 / E + (VEC ? 0 : 1);  // a row may start and end inside a vector
  __shared__ TopkShared sh;
  const int64_t row = blockIdx.x;
  const Rv rv(row, p.rows, p.V);
  u32x4 w[1][U];
  rv.load({p.z}, int(threadIdx.x), BLK, w);
  uint32_t key[U * E];
  float m = kNegInf;
  if (threadIdx.x == 0) sh.n = 0;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int gi = int(threadIdx.x) + u * BLK;
    float x[E];
    TI::unpack(to_uint4(w[0][u]), x);
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int v = rv.index(gi, e);
      m = fmaxf(m, x[e]);
      key[u * E + e] = gi < rv.ng && (VEC || (v >= 0 && v < p.V)) ? order_key<TI>(x[e]) : 0u;
    }
  }
  m = block_max<WV>(m, sh.f);
  const float msc = m == kNegInf ? 0.f : m * p.sc;
  const uint32_t t = threshold<TI, WV>(key, p.k, order_key<TI>(m), sh.i);
  float s = 0.f;
#pragma unroll
  for (int u = 0; u < U; ++u)
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const uint32_t c = key[u * E + e];
      if (c == 0u) continue;
      if (c >= t)
        add_candidate(sh, c, rv.index(int(threadIdx.x) + u * BLK, e));
      else
        s += ex2(__builtin_fmaf(key_logit<TI>(c), p.sc, -msc));
    }
  __syncthreads();
  int n = int(sh.n);
  if (n > kCap) {
    s = select_slowly<TI, VEC, BLK>(p, row, msc, sh);
    n = p.k;
  }
  s += write_ranked<TI, BLK>(p, row, n, msc, sh);
  write_rest<WV>(p, row, s, msc, sh);
}

// Longer rows: a group of a thread is `rounds` rounds of U vectors.
template <class TI, bool VEC, int U, int BLK>
__global__ __launch_bounds__(BLK) void k_topk_rows(TopkParams p, int rounds) {
  using Rv = RowVecs<TI, VEC>;
  constexpr int E = Rv::E;
  constexpr int WV = BLK / kWave;
  __shared__ TopkShared sh;
  const int64_t row = blockIdx.x;
  const Rv rv(row, p.rows, p.V);
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wv = tid / kWave;
  float gm[kGroups], gs[kGroups];
  uint32_t key[kGroups];
  float m = kNegInf;
  if (tid == 0) sh.n = 0;
#pragma unroll
  for (int g = 0; g < kGroups; ++g) {
    LseState st = lse_init();
    for (int r = 0; r < rounds; ++r) {
      const int base = (g * rounds + r) * U * BLK + tid;
      if (base >= rv.ng) break;
      u32x4 w[1][U];
      float x[U][E];
      rv.load({p.z}, base, BLK, w);
      rv.unpack(w[0], x);
      lse_fold(st, x, p.sc);
    }
    gm[g] = st.m;
    gs[g] = st.s;
    key[g] = g * rounds * U * BLK + tid < rv.ng ? order_key<TI>(st.m) : 0u;
    m = fmaxf(m, st.m);
  }
  m = block_max<WV>(m, sh.f);
  const float msc = m == kNegInf ? 0.f : m * p.sc;
  const uint32_t t = threshold<TI, WV>(key, p.k, order_key<TI>(m), sh.i);
  // the groups that reach t, in an order that does not depend on timing; the sums of the others
  float s = 0.f;
  int mine = 0;
#pragma unroll
  for (int g = 0; g < kGroups; ++g) {
    if (key[g] == 0u) continue;
    if (key[g] >= t)
      ++mine;
    else if (gm[g] != kNegInf)
      s += gs[g] * ex2(gm[g] * p.sc - msc);
  }
  int before = mine;
  for (int off = 1; off < kWave; off <<= 1) {
    const int o = __shfl_up(before, off, kWave);
    if (lane >= off) before += o;
  }
  if (lane == kWave - 1) sh.i[0][wv] = before;
  __syncthreads();
  int at = before - mine, nq = 0;
#pragma unroll
  for (int i = 0; i < WV; ++i) {
    if (i < wv) at += sh.i[0][i];
    nq += sh.i[0][i];
  }
  int n = kCap + 1;
  if (nq <= kCap) {
#pragma unroll
    for (int g = 0; g < kGroups; ++g)
      if (key[g] != 0u && key[g] >= t) sh.queue[at++] = uint16_t(g * BLK + tid);
    __syncthreads();
    const int per = rounds * U;  // vectors of a group
    for (int j = tid; j < nq * per; j += BLK) {
      const int q = sh.queue[j / per], sub = j % per;
      const int gi = ((q / BLK) * per + sub) * BLK + q % BLK;
      if (gi >= rv.ng) continue;
      float x[E];
      TI::unpack(to_uint4(rv.load(p.z, gi)), x);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int v = rv.index(gi, e);
        if (!VEC && (v < 0 || v >= p.V)) continue;
        const uint32_t c = order_key<TI>(x[e]);
        if (c >= t)
          add_candidate(sh, c, v);
        else
          s += ex2(__builtin_fmaf(x[e], p.sc, -msc));
      }
    }
    __syncthreads();
    n = int(sh.n);
  }
  if (n > kCap) {
    s = select_slowly<TI, VEC, BLK>(p, row, msc, sh);
    n = p.k;
  }
  s += write_ranked<TI, BLK>(p, row, n, msc, sh);
  write_rest<WV>(p, row, s, msc, sh);
}

template <class TI, bool VEC>
hipError_t launch_vec(const TopkArgs& a) {
  const TopkParams p{a.z, a.rows, a.V, a.k, a.sc, a.top, a.ids, a.rest};
  const dim3 grid{unsigned(a.rows)};
  constexpr int kBlk = 512;
  // vectors that cover a row, at most
  const int ng = a.V / TI::kVec + (VEC ? 0 : 2);
  if (a.V <= 16 * 64)
    k_topk_short<TI, VEC, 64><<<grid, 64, 0, a.stream>>>(p);
  else if (a.V <= 16 * 128)
    k_topk_short<TI, VEC, 128><<<grid, 128, 0, a.stream>>>(p);
  else if (a.V <= 16 * 256)
    k_topk_short<TI, VEC, 256><<<grid, 256, 0, a.stream>>>(p);
  else if (a.V <= 16 * kBlk)
    k_topk_short<TI, VEC, kBlk><<<grid, kBlk, 0, a.stream>>>(p);
  else if (ng <= kGroups * kBlk)
    k_topk_rows<TI, VEC, 1, kBlk><<<grid, kBlk, 0, a.stream>>>(p, 1);
  else if (ng <= kGroups * kBlk * 2)
    k_topk_rows<TI, VEC, 2, kBlk><<<grid, kBlk, 0, a.stream>>>(p, 1);
  else
    k_topk_rows<TI, VEC, 4, kBlk><<<grid, kBlk, 0, a.stream>>>(
        p, int((int64_t(ng) + kGroups * kBlk * 4 - 1) / (kGroups * kBlk * 4)));
  return hipGetLastError();
}

template <class TI>
hipError_t launch_typed(const TopkArgs& a) {
  return a.V % TI::kVec == 0 ? launch_vec<TI, true>(a) : launch_vec<TI, false>(a);
}

}  // namespace

size_t topk_workspace_bytes(int64_t, int, int) { return 256; }

hipError_t launch_topk(const TopkArgs& a) {
  return a.in == DType::kBf16 ? launch_typed<Bf16>(a) : launch_typed<F32>(a);
}

}  // namespace aal
