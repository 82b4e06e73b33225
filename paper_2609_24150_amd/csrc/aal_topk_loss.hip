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
// Bound by memory and, with WTV or EAL terms, by the wait between a row's sums and its
// coefficients: 14,336 rows of 128,256 bf16, lists of 64, WTV: 1,589 us, 83% of the rate of a
// lone read and write; KL alone, which waits for nobody, 1,412 us, 93%.
// Both end with k_top_loss: every window's E, the four terms and the weighted
// loss, in a fixed order of summation.
//
// The listed entries are kept out of the unlisted sum and its reference by a bitmap of the
// vocabulary in LDS, so that q_r is a sum and not a difference, and KL and its gradient hold
// where the draft's unlisted logits lie so far below the list that q_r is 0 in fp32.
#include "aal_topk_loss_common.h"

namespace aal {
namespace {

// -------------------------------------------------- multi-kernel schedule
template <class TI, bool VEC, int U, int BLK>
__global__ __launch_bounds__(BLK) void k_top_rows(TopLossParams p, int64_t row0) {
  using Rv = RowVecs<TI, VEC>;
  constexpr int E = Rv::E;
  extern __shared__ uint32_t sh_map[];
  __shared__ float sh_t[kTopMax], sh_z[kTopMax];
  __shared__ int sh_id[kTopMax];
  __shared__ float sh_m[BLK / kWave], sh_s[BLK / kWave];

  const int64_t row = row0 + blockIdx.x;
  const Rv rv(row, p.R, p.V);
  const int64_t e0 = row * int64_t(p.V), l0 = row * p.k;
  const int words = bitmap_words(p.V);
  if (row == 0 && threadIdx.x == 0) *p.counter = 0u;
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
  // the largest unlisted logit, the sum over the unlisted ones against its own_ref so far
  float m = kNegInf, s = 0.f;
  for (int base = threadIdx.x; base < rv.ng; base += BLK * U) {
    u32x4 w[1][U];
    float x[U][E];
    rv.load({p.zd}, base, BLK, w);
    rv.unpack(w[0], x);
    float cm = m;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int gi = base + u * BLK;
      const uint32_t bits = gi < rv.ng ? listed_bits<E>(sh_map, gi) : 0u;
      if (bits)
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (bits >> e & 1u) x[u][e] = kNegInf;
#pragma unroll
      for (int e = 0; e < E; ++e) cm = fmaxf(cm, x[u][e]);
    }
    const float at = own_ref(cm, p.scd);
    s *= ex2(own_ref(m, p.scd) - at);
    m = cm;
    float c[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
      for (int e = 0; e < E; ++e) x[u][e] = ex2(__builtin_fmaf(x[u][e], p.scd, -at));
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
  if (ref.steep) {
    s = 0.f;
    for (int gi = threadIdx.x; gi < rv.ng; gi += BLK) {
      float x[E];
      TI::unpack(to_uint4(rv.load(p.zd, gi)), x);
      const uint32_t bits = listed_bits<E>(sh_map, gi);
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (!(bits >> e & 1u)) s += ex2(log2_of(ref, x[e]));
    }
  } else {
    s *= ex2(own_ref(m, p.scd) - ref.msc);
  }
  s = wave_sum(s);
  if (lane == 0) sh_s[wv] = s;
  __syncthreads();
  if (threadIdx.x < kWave) {
    s = wave_sum(lane < BLK / kWave ? sh_s[lane] : 0.f);
    const TopRow o = list_row(p, list_target(p, row, sh_t, sh_id), sh_t, sh_z, sh_id, list_draft(p, sh_t, sh_z), ref, s);
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
__global__ __launch_bounds__(kRowBlock) void k_top_grad(TopLossParams p, int64_t row0, int splits, void* __restrict__ grad) {
  using Rv = RowVecs<TI, VEC>;
  constexpr int E = Rv::E;
  const int64_t row = row0 + blockIdx.x;
  const Rv rv(row, p.R, p.V);
  const TopRow s = p.stats[row];
  const RowRef ref = row_ref(s.mu, p.scd), list = row_ref(s.ml, p.scd);
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
      for (int e = 0; e < E; ++e) g[e] = s.cR * ex2(log2_of(ref, x[e]));
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
    const float q = ex2(log2_of(list, TI::load1(p.zd, e0 + id))) * s.ql;
    TG::store1(grad, e0 + id, listed_grad(s, q, listed_p(s, t, p.sct), id));
  }
}

// ------------------------------------------------------------------- loss
constexpr int kLossBlock = 256;
static_assert(kTopLossParts <= kLossBlock, "a part a thread");

// The sums of four values over the workgroup, to every thread.
__device__ void block_sum4(double (&v)[4], double (*sh)[4]) {
  for (int off = kWave / 2; off > 0; off >>= 1)
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] += __shfl_xor(v[i], off, kWave);
  __syncthreads();
  if ((threadIdx.x & (kWave - 1)) == 0)
    for (int i = 0; i < 4; ++i) sh[threadIdx.x / kWave][i] = v[i];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[i] = 0.0;
    for (int w = 0; w < kLossBlock / kWave; ++w) v[i] += sh[w][i];
  }
}

// Every window's E and the loss: workgroup b sums the rows of its slice (a window
// counts where it starts); the last one to end adds the slices' sums in order.
__global__ __launch_bounds__(kLossBlock) void k_top_loss(TopLossParams p, int n, double* parts, float* loss,
                                                         float* terms, float* e_tv, float* e_eal,
                                                         const unsigned* err) {
  __shared__ double sh[kLossBlock / kWave][4];
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
  block_sum4(v, sh);
  if (n > 1) {
    if (threadIdx.x == 0) {
      for (int i = 0; i < 4; ++i)
        __hip_atomic_store(parts + 4 * blockIdx.x + i, v[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      sh_last = __hip_atomic_fetch_add(p.counter, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == unsigned(n - 1);
    }
    __syncthreads();
    if (!sh_last) return;
    // at most a part a thread
    for (int i = 0; i < 4; ++i)
      v[i] = int(threadIdx.x) < n ? __hip_atomic_load(parts + 4 * threadIdx.x + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0.0;
    block_sum4(v, sh);
  }
  if (threadIdx.x != 0) return;
  // a term whose weight is 0 reads 0
  const double t0 = p.W > 0 && p.w_wtv != 0.f ? -v[0] / double(p.W) : 0.0;
  const double t1 = p.W > 0 && p.w_eal != 0.f ? -v[1] / double(p.W) : 0.0;
  const double t2 = p.w_kl != 0.f ? v[2] / double(p.R) : 0.0;
  const double t3 = p.W > 0 && p.w_tv != 0.f ? v[3] / (double(p.W) * p.K) : 0.0;
  const float l = float(double(p.w_wtv) * t0 + double(p.w_eal) * t1 + double(p.w_kl) * t2 + double(p.w_tv) * t3);
  // a set error word (a poll of the resident schedule timed out): NaN, by its bits, since the build
  // takes floating-point values for anything else
  const uint32_t bits = err != nullptr && *err != 0u ? 0x7fc00000u : __builtin_bit_cast(uint32_t, l);
  loss[0] = __builtin_bit_cast(float, bits);
  if (terms) {
    terms[0] = float(t0);
    terms[1] = float(t1);
    terms[2] = float(t2);
    terms[3] = float(t3);
  }
}

hipError_t loss_launch(const TopLossArgs& a, bool waited) {
  const int64_t want = (a.R + kLossBlock - 1) / kLossBlock;
  const int n = int(want < kTopLossParts ? want : kTopLossParts);
  k_top_loss<<<dim3(unsigned(n)), kLossBlock, 0, a.stream>>>(params_of(a), n, a.loss_parts, a.loss, a.terms, a.e_tv,
                                                            a.e_eal, waited ? a.err : nullptr);
  return hipGetLastError();
}

// The resident schedule, where its kernels hold the row (fp32 logits with a bf16
// gradient take the multi-kernel one, as they do in the other objectives).
hipError_t launch_top_fused(const TopLossArgs& a, bool* used) {
  const bool whole = a.V % (a.in == DType::kBf16 ? Bf16::kVec : F32::kVec) == 0;
  if (a.in == DType::kBf16) {
    if (a.gd == DType::kBf16) return whole ? launch_top_fused_bf16_whole(a, used) : launch_top_fused_bf16_ragged(a, used);
    return whole ? launch_top_fused_bf16_g32_whole(a, used) : launch_top_fused_bf16_g32_ragged(a, used);
  }
  if (a.gd == DType::kBf16) return hipSuccess;
  return whole ? launch_top_fused_f32_whole(a, used) : launch_top_fused_f32_ragged(a, used);
}

template <class TI, class TG, bool VEC>
hipError_t grad_launch(const TopLossArgs& a) {
  hipError_t e = hipSuccess;
  with_grad_shape(a.V, TI::kVec, [&](auto sh) {
    constexpr int U = decltype(sh)::kU;
    const unsigned splits = row_splits(a.R, a.V, TI::kVec, U);
    e = for_row_parts(a.R, [&](int64_t row0, unsigned n) {
      k_top_grad<TI, TG, VEC, U><<<dim3(n, splits), kRowBlock, 0, a.stream>>>(params_of(a), row0, int(splits), a.grad);
      return hipGetLastError();
    });
  });
  return e;
}

template <class TI, bool VEC>
hipError_t launch_vec(const TopLossArgs& a) {
  hipError_t e = hipSuccess;
  with_row_shape<4>(a.R, a.V, TI::kVec, [&](auto sh) {
    using Sh = decltype(sh);
    e = for_row_parts(a.R, [&](int64_t row0, unsigned n) {
      k_top_rows<TI, VEC, Sh::kU, Sh::kBlock>
          <<<dim3(n), Sh::kBlock, size_t(bitmap_words(a.V)) * 4, a.stream>>>(params_of(a), row0);
      return hipGetLastError();
    });
  });
  if (e != hipSuccess) return e;
  k_top_scan<<<dim3(unsigned((a.R + kRowBlock - 1) / kRowBlock)), kRowBlock, 0, a.stream>>>(params_of(a));
  if ((e = loss_launch(a, false)) != hipSuccess) return e;
  if (a.grad == nullptr) return hipSuccess;
  return a.gd == DType::kBf16 ? grad_launch<TI, GBf16, VEC>(a) : grad_launch<TI, GF32, VEC>(a);
}

template <class TI>
hipError_t launch_typed(const TopLossArgs& a) {
  return a.V % TI::kVec == 0 ? launch_vec<TI, true>(a) : launch_vec<TI, false>(a);
}

}  // namespace

hipError_t launch_top_loss(const TopLossArgs& a) {
  bool used = false;
  if (!a.streaming) {
    if (hipError_t e = launch_top_fused(a, &used); e != hipSuccess) return e;
    if (used) return loss_launch(a, a.w_wtv != 0.f || a.w_eal != 0.f);
  }
  return a.in == DType::kBf16 ? launch_typed<Bf16>(a) : launch_typed<F32>(a);
}

}  // namespace aal
