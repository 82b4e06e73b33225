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
// Two beams' candidates may differ by less than 32 bits tell apart, and a choice cannot be off by a
// rounding: totals are formed in 64 bits, and so is a row's log-sum-exp where it counts,
// the exponentials of the listed logits.  Those of the others are v_exp_f32's of arguments with one
// rounding (log2(e) / T in two pieces), whose errors average out over the many of them that it takes to
// bear on the sum.  Parts are cut from the row's start whatever its alignment, so that equal rows
// get equal sums, and equal beams tie exactly.
#include "aal_beam.h"
#include "aal_device.h"
#include "aal_select.h"

namespace aal {
namespace {

constexpr int kCand = 512;      // candidates of a part that fit
constexpr int kMergeMost = 64;  // candidates per thread of the merge
constexpr int kSurvivors = 1024;

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

template <class TI, int BLK, int U>
__global__ __launch_bounds__(BLK) void k_beam_parts(BeamParams p) {
  constexpr int E = TI::kVec, WV = BLK / kWave;
  constexpr int kShift = 32 - key_bits<TI>();
  __shared__ uint64_t cand[kCand], sorted[kCand];
  __shared__ double dsum[WV];
  __shared__ float fsh[WV];
  __shared__ int ish[WV];
  __shared__ int count;
  const int64_t row = p.row0 + blockIdx.x / p.parts;
  const int part = blockIdx.x % p.parts, tid = threadIdx.x, lane = tid & (kWave - 1), wv = tid / kWave;
  if ((p.finished && p.finished[row]) || p.scores[row] == kNegInf) return;
  const int s0 = part * p.part_len, len = min(p.part_len, p.V - s0);
  const typename TI::storage* base = static_cast<const typename TI::storage*>(p.z) + row * int64_t(p.V) + s0;
  float x[U][E], gm[U], m = kNegInf;
  if (tid == 0) count = 0;
  u32x4 raw[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int at = (u * BLK + tid) * E;
    if (at + E <= len) raw[u] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_e2*>(base + at));
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int at = (u * BLK + tid) * E;
    if (at + E <= len) {
      TI::unpack(to_uint4(raw[u]), x[u]);
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e) x[u][e] = at + e < len ? TI::load1(base, at + e) : kNegInf;
    }
    gm[u] = x[u][0];
#pragma unroll
    for (int e = 1; e < E; ++e) gm[u] = fmaxf(gm[u], x[u][e]);
    m = fmaxf(m, gm[u]);
  }
  m = wave_max(m);
  if (lane == 0) fsh[wv] = m;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < WV; ++i) m = fmaxf(m, fsh[i]);
  __syncthreads();
  const int64_t slot = row * int64_t(p.parts) + part;
  uint64_t* list = p.list + slot * p.n;
  if (m == kNegInf) {
    for (int i = tid; i < p.n; i += BLK) list[i] = 0;
    if (tid == 0) p.part[slot] = {0.0, kNegInf, 0};
    return;
  }
  // at least n logits reach t, or all finite ones do
  float t = threshold<TI, WV>(gm, p.n, m, fsh);
  auto collect = [&](float from, bool strict) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (!(gm[u] >= from)) continue;
#pragma unroll
      for (int e = 0; e < E; ++e)
        if ((strict ? x[u][e] > from : x[u][e] >= from) && x[u][e] != kNegInf) {
          const int at = atomicAdd(&count, 1);
          if (at < kCand) cand[at] = entry_of(order_key<TI>(x[u][e]), s0 + (u * BLK + tid) * E + e);
        }
    }
  };
  collect(t, false);
  __syncthreads();
  int c = count, left_ties = 0;
  if (c > kCand) {
    // ties or clusters: the n-th largest logit itself, and the first of its ties
    uint32_t lo = order_key<TI>(kNegInf) >> kShift, hi = (order_key<TI>(m) >> kShift) + 1u;
    while (hi > lo + 1u) {
      const uint32_t mid = lo + (hi - lo) / 2;
      const float f = key_logit<TI>(mid << kShift);
      int reach = 0;
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int e = 0; e < E; ++e) reach += __popcll(__builtin_amdgcn_ballot_w64(x[u][e] >= f));
      (block_count<WV>(reach, ish) >= p.n ? lo : hi) = mid;
    }
    t = key_logit<TI>(lo << kShift);
    if (tid == 0) count = 0;
    __syncthreads();
    collect(t, true);
    __syncthreads();
    c = count;
    if (t != kNegInf) {
      int ties = 0;  // before this vector's turn
#pragma unroll
      for (int u = 0; u < U; ++u) {
        int mine = 0;
#pragma unroll
        for (int e = 0; e < E; ++e) mine += x[u][e] == t;
        int before = mine;
        for (int off = 1; off < kWave; off <<= 1) {
          const int o = __shfl_up(before, off, kWave);
          if (lane >= off) before += o;
        }
        __syncthreads();
        if (lane == kWave - 1) ish[wv] = before;
        __syncthreads();
        int at = c + ties + before - mine;
#pragma unroll
        for (int i = 0; i < WV; ++i) {
          if (i < wv) at += ish[i];
          ties += ish[i];
        }
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (x[u][e] == t) {
            if (at < p.n) cand[at] = entry_of(order_key<TI>(t), s0 + (u * BLK + tid) * E + e);
            ++at;
          }
      }
      const int taken = min(p.n - c, ties);
      left_ties = ties - taken;
      c += taken;
    }
    __syncthreads();
  }
  for (int i = tid; i < c; i += BLK) {
    const uint64_t mine = cand[i];
    int rank = 0;
    for (int j = 0; j < c; ++j) rank += cand[j] > mine;
    sorted[rank] = mine;
  }
  // the others' sum, while the list is being sorted
  auto weight = [&](float z) {
    const float d = z - m;
    return ex2(__builtin_fmaf(d, p.sc_hi, d * p.sc_lo));
  };
  float s = 0.f;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    float us = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) us += x[u][e] < t ? weight(x[u][e]) : 0.f;
    s += us;
  }
  if (tid == 0 && left_ties) s += float(left_ties) * weight(t);
  __syncthreads();
  double total = double(s);
  for (int i = tid; i < max(c, p.n); i += BLK) {
    if (i < p.n) {
      list[i] = i < c ? sorted[i] : 0;
      if (i < c) total += exp((double(entry_logit<TI>(sorted[i])) - double(m)) * p.inv_t);
    } else {
      total += double(weight(entry_logit<TI>(sorted[i])));
    }
  }
  total = wave_sum_d(total);
  if (lane == 0) dsum[wv] = total;
  __syncthreads();
  if (tid == 0) {
    total = dsum[0];
    for (int i = 1; i < WV; ++i) total += dsum[i];
    p.part[slot] = {total, m, 0};
  }
}

__device__ __forceinline__ bool before(double ra, int ba, uint64_t ea, double rb, int bb, uint64_t eb) {
  return ra > rb || (ra == rb && (ba < bb || (ba == bb && ea > eb)));
}

// NT threads with up to NPT candidates each: a request's lists and, behind them, the beams that have ended.
template <class TI, int NT, int NPT>
__global__ __launch_bounds__(NT) void k_beam_merge(BeamParams p, int64_t b0) {
  constexpr int WV = NT / kWave;
  __shared__ double lse[kBeamMax], factor[kBeamMax], score[kBeamMax];
  __shared__ int state[kBeamMax];  // 0 goes on, 1 has ended, 2 has score -inf
  __shared__ double srank[kSurvivors];
  __shared__ uint64_t sentry[kSurvivors];
  __shared__ int sbeam[kSurvivors];
  __shared__ int ish[WV];
  __shared__ int count;
  const int64_t b = b0 + blockIdx.x, row0 = b * p.W;
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wv = tid / kWave;
  if (tid == 0) count = 0;
  for (int w = wv; w < p.W; w += WV) {
    const float sw = p.scores[row0 + w];
    const bool done = p.finished && p.finished[row0 + w];
    const int st = sw == kNegInf ? 2 : done ? 1 : 0;
    double l = 0.0;
    if (st == 0) {
      const BeamPart* part = p.part + (row0 + w) * p.parts;
      float m = kNegInf;
      for (int i = lane; i < p.parts; i += kWave) m = fmaxf(m, part[i].m);
      m = wave_max(m);
      double s = 0.0;
      for (int i = lane; i < p.parts; i += kWave)
        if (part[i].m != kNegInf) s += part[i].s * exp((double(part[i].m) - double(m)) * p.inv_t);
      s = wave_sum_d(s);
      if (m != kNegInf) l = double(m) * p.inv_t + log(s);
    }
    if (lane == 0) {
      const int len = p.lengths ? p.lengths[row0 + w] : 0;
      lse[w] = l;
      score[w] = double(sw);
      state[w] = st;
      factor[w] = p.alpha != 0.0 ? pow(double(len + (st == 0)), p.alpha) : 1.0;
    }
  }
  __syncthreads();
  const int per = p.parts * p.n, C = p.W * per;
  auto total_of = [&](int w, uint64_t e) {
    return state[w] == 1 ? score[w] : double(entry_logit<TI>(e)) * p.inv_t - lse[w] + score[w];
  };
  // candidate i's beam and entry; false where there is none
  auto candidate = [&](int i, int& w, uint64_t& e) {
    if (i < C) {
      w = i / per;
      if (state[w] != 0) return false;
      e = p.list[row0 * per + i];
      return e != 0;
    }
    w = i - C;
    e = 1;
    return w < p.W && state[w] == 1;
  };
  auto rank_of = [&](int w, uint64_t e) {
    const double t = total_of(w, e);
    return p.alpha != 0.0 ? t / factor[w] : t;
  };
  // ranks in 32 bits keep their order, up to ties: enough to leave most candidates out
  uint32_t key[NPT];
#pragma unroll
  for (int k = 0; k < NPT; ++k) {
    int w;
    uint64_t e;
    key[k] = candidate(k * NT + tid, w, e) ? order_key<F32>(float(rank_of(w, e))) : 0u;
  }
  auto reached = [&](uint32_t t) {
    int c = 0;
#pragma unroll
    for (int k = 0; k < NPT; ++k) c += __popcll(__builtin_amdgcn_ballot_w64(key[k] >= t));
    return block_count<WV>(c, ish);
  };
  uint32_t lo = 1u;
  const int most = p.n + p.n / 4 + 32;
  int c = reached(lo);
  if (c > most) {
    uint32_t hi = 0xffffffffu;
    while (hi > lo + 1u) {
      const uint32_t mid = lo + (hi - lo) / 2;
      const int r = reached(mid);
      if (r >= p.n) {
        lo = mid;
        c = r;
        if (r <= most) break;
      } else {
        hi = mid;
      }
    }
  }
  const int64_t o = b * p.n;
  auto write = [&](int j, int w, uint64_t e, double rank) {
    const bool done = state[w] == 1;
    const int token = done ? p.pad : entry_token(e);
    p.out.parents[o + j] = w;
    p.out.tokens[o + j] = token;
    if (p.out.scores) p.out.scores[o + j] = float(total_of(w, e));
    if (p.out.rank) p.out.rank[o + j] = float(rank);
    if (p.out.finished) p.out.finished[o + j] = done || token == p.eos;
    if (p.out.lengths) p.out.lengths[o + j] = (p.lengths ? p.lengths[row0 + w] : 0) + !done;
  };
  int found = c;
  if (c <= kSurvivors) {
#pragma unroll
    for (int k = 0; k < NPT; ++k) {
      if (key[k] < lo) continue;
      int w;
      uint64_t e;
      candidate(k * NT + tid, w, e);
      const int at = atomicAdd(&count, 1);
      srank[at] = rank_of(w, e);
      sentry[at] = e;
      sbeam[at] = w;
    }
    __syncthreads();
    for (int i = tid; i < c; i += NT) {
      const double r = srank[i];
      const uint64_t e = sentry[i];
      const int w = sbeam[i];
      int at = 0;
      for (int j = 0; j < c; ++j) at += before(srank[j], sbeam[j], sentry[j], r, w, e);
      if (at < p.n) write(at, w, e, r);
    }
  } else {
    // too many ranks that 32 bits do not tell apart: one after the other
    double lr = __builtin_huge_val();
    int lw = -1;
    uint64_t le = 0;
    for (found = 0; found < p.n; ++found) {
      double br = -__builtin_huge_val();
      int bw = kBeamMax;
      uint64_t be = 0;
#pragma unroll 1
      for (int k = 0; k < NPT; ++k) {
        int w;
        uint64_t e;
        if (!candidate(k * NT + tid, w, e)) continue;
        const double r = rank_of(w, e);
        if (before(lr, lw, le, r, w, e) && before(r, w, e, br, bw, be)) {
          br = r;
          bw = w;
          be = e;
        }
      }
      for (int off = 32; off > 0; off >>= 1) {
        const double r = __shfl_xor(br, off, kWave);
        const int w = __shfl_xor(bw, off, kWave);
        const uint64_t e = uint64_t(__shfl_xor((unsigned long long)be, off, kWave));
        if (before(r, w, e, br, bw, be)) {
          br = r;
          bw = w;
          be = e;
        }
      }
      __syncthreads();
      if (lane == 0) {
        srank[wv] = br;
        sbeam[wv] = bw;
        sentry[wv] = be;
      }
      __syncthreads();
      for (int i = 0; i < WV; ++i)
        if (before(srank[i], sbeam[i], sentry[i], br, bw, be)) {
          br = srank[i];
          bw = sbeam[i];
          be = sentry[i];
        }
      lr = br;
      lw = bw;
      le = be;
      if (tid == 0) write(found, bw, be, br);
    }
  }
  for (int j = min(found, p.n) + tid; j < p.n; j += NT) {
    p.out.parents[o + j] = -1;
    p.out.tokens[o + j] = p.pad;
    if (p.out.scores) p.out.scores[o + j] = kNegInf;
    if (p.out.rank) p.out.rank[o + j] = kNegInf;
    if (p.out.finished) p.out.finished[o + j] = 1;
    if (p.out.lengths) p.out.lengths[o + j] = 0;
  }
}

// How rows are cut: threads and vectors per thread of a part's workgroup, parts of a row.
struct Cut {
  int block, u, parts, len;
};
Cut cut_rows(DType in, int64_t B, int W, int V, int n) {
  const int E = in == DType::kBf16 ? 8 : 4;
  auto of = [&](int block, int u) {
    const int most = block * u * E, parts = (V + most - 1) / most;
    const int len = ((V + parts - 1) / parts + E - 1) / E * E;
    return Cut{block, u, (V + len - 1) / len, len};
  };
  // as long as 1,024 workgroups remain; no more candidates than the merge takes
  for (int u = 8; u >= 1; u /= 2) {
    const Cut c = of(256, u), half = u > 1 ? of(256, u / 2) : c;
    if (int64_t(W) * c.parts * n + W > kMergeMost * 256) return of(1024, 8);
    if (u == 1 || B * W * c.parts >= 1024 || int64_t(W) * half.parts * n + W > kMergeMost * 256) return c;
  }
  return of(1024, 8);
}

template <class TI>
hipError_t launch_typed(const BeamArgs& a) {
  const Cut c = cut_rows(a.in, a.B, a.W, a.V, a.n);
  BeamParams p{};
  p.z = a.z;
  p.rows = a.B * a.W;
  p.W = a.W;
  p.V = a.V;
  p.n = a.n;
  p.parts = c.parts;
  p.part_len = c.len;
  p.inv_t = 1.0 / double(a.temperature);
  // the lower piece is above 0, so that a logit of -inf is no NaN
  const double sc = 1.4426950408889634073599246810019 / double(a.temperature);
  p.sc_hi = float(sc);
  if (double(p.sc_hi) >= sc) p.sc_hi = __builtin_nextafterf(p.sc_hi, 0.f);
  p.sc_lo = float(sc - double(p.sc_hi));
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
    if (c.block == 1024)
      k_beam_parts<TI, 1024, 8><<<grid, 1024, 0, a.stream>>>(p);
    else if (c.u == 8)
      k_beam_parts<TI, 256, 8><<<grid, 256, 0, a.stream>>>(p);
    else if (c.u == 4)
      k_beam_parts<TI, 256, 4><<<grid, 256, 0, a.stream>>>(p);
    else if (c.u == 2)
      k_beam_parts<TI, 256, 2><<<grid, 256, 0, a.stream>>>(p);
    else
      k_beam_parts<TI, 256, 1><<<grid, 256, 0, a.stream>>>(p);
  }
  const int64_t cands = int64_t(a.W) * c.parts * a.n + a.W;
  for (int64_t b0 = 0; b0 < a.B; b0 += int64_t(1) << 21) {
    const dim3 grid(unsigned(a.B - b0 < (int64_t(1) << 21) ? a.B - b0 : int64_t(1) << 21));
    if (cands <= 256)
      k_beam_merge<TI, 256, 1><<<grid, 256, 0, a.stream>>>(p, b0);
    else if (cands <= 1024)
      k_beam_merge<TI, 256, 4><<<grid, 256, 0, a.stream>>>(p, b0);
    else if (cands <= 4096)
      k_beam_merge<TI, 1024, 4><<<grid, 1024, 0, a.stream>>>(p, b0);
    else if (cands <= 16384)
      k_beam_merge<TI, 1024, 16><<<grid, 1024, 0, a.stream>>>(p, b0);
    else
      k_beam_merge<TI, 1024, kMergeMost + 1><<<grid, 1024, 0, a.stream>>>(p, b0);
  }
  return hipGetLastError();
}

}  // namespace

size_t beam_workspace_bytes(DType in, int64_t B, int W, int V, int n) {
  const Cut c = cut_rows(in, B, W, V, n);
  const size_t slots = size_t(B) * size_t(W) * size_t(c.parts);
  return align256(slots * sizeof(BeamPart)) + align256(slots * size_t(n) * sizeof(uint64_t));
}

hipError_t launch_beam_select(const BeamArgs& a) {
  return a.in == DType::kBf16 ? launch_typed<Bf16>(a) : launch_typed<F32>(a);
}

}  // namespace aal
