// The resident schedule of the objectives against top lists: a row in the
// registers of a workgroup from its one read to the one write of its gradient.
#pragma once

#include "aal_topk_loss_common.h"

namespace aal {
namespace {

// ------------------------------------------------------- resident schedule
// The bitmap reaches to the end of the last vectors that a workgroup holds.
constexpr int stage_words(int held) { return (bitmap_words(held) + 3) & ~3; }  // before the staging buffer
inline size_t fused_lds_bytes(int held, int staged, int k) {
  return size_t(stage_words(held)) * 4 + size_t(staged) * 16 + size_t(k) * 20;
}

template <class TI, int E>
__device__ __forceinline__ u32x4 packv(const float (&x)[E]) {
  if constexpr (E == 8)
    return u32x4{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7])};
  else
    return u32x4{__builtin_bit_cast(uint32_t, x[0]), __builtin_bit_cast(uint32_t, x[1]),
                 __builtin_bit_cast(uint32_t, x[2]), __builtin_bit_cast(uint32_t, x[3])};
}

// WK waves hold the row, NV vectors a thread; the last wave does the list, the
// windows and the coefficients beside their passes, so that neither's registers
// add to the other's.  Three barriers a row:
//   holders                                                list
//   gradient of the row before, this row's loads           finishes the row before last; this list, bitmap
//   1                                                      the listed alone: p's sum, the draft's
//   each vector as it arrives: largest, sum of the unlisted
//   2
//                                                          p and q, acceptances, neighbours, coefficients
//   3
// So the loads of a row run under the gradient pass of the one before and under
// its own sums, and only the step between 2 and 3 (about 3 us) has none.
// The listed entries' gradient is stored over the others' after the next row's barrier 2,
// when every holder has waited for its stores.
// With seven holders the registers are held to what lets two workgroups run on a CU: 7,168 rows of
// 65,536 bf16, WTV, 398 us against 465 with one.  Ragged rows through the buffer resources
// and LDS too, their ends alone apart: 7,168 rows of 50,001, 334 us against 408 with an address
// and a condition for every vector, whose registers left one workgroup a CU.
// With nine vectors and a bf16 gradient, to 80 for 24 waves: one more left 20 (the same with an
// fp32 gradient, which takes 89 to 94, costs 14,336 rows of 32,000 783 us against 689).
template <class TG, int WK, int NV>
constexpr int kMinWaves = NV == 9 && sizeof(typename TG::storage) == 2 ? 6 : WK == 7 ? 4 : 1;
template <class TI, class TG, bool VEC, int WK, int NV, int NS, bool COUPLED>
__global__ __launch_bounds__((WK + 1) * kWave, (kMinWaves<TG, WK, NV>)) void k_top_fused(TopLossParams p, int grid, void* __restrict__ grad) {
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
      const ListDraft ld_row = list_draft(p, lt, lz);
      const RowWindows rw = row_windows(row, p.layout, p.S, p.K);
      lds_barrier();  // 2
      const float wm = lane < WK ? sh_m[lane] : kNegInf;
      const RowRef ref = row_ref(wave_max(wm), p.scd);
      if (ref.steep) lds_barrier();
      const float su = wave_sum(lane < WK ? sh_s[lane] * (ref.steep ? 1.f : ex2(own_ref(wm, p.scd) - ref.msc)) : 0.f);
      TopRow o = list_row(p, lt_row, lt, lz, li, ld_row, ref, su);
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
        // to lane 0, over as many lanes as there are windows
        int width = 1;
        while (width < rw.t1 - rw.t0 + 1) width *= 2;
        for (int off = width / 2; off > 0; off /= 2) {
          if (p.w_wtv != 0.f) d_tv += __shfl_xor(d_tv, off, kWave);
          if (p.w_eal != 0.f) d_eal += __shfl_xor(d_eal, off, kWave);
        }
      }
      const double count = windows_of(rw);
      row_coefs(o, p, d_tv, d_eal, count);
      if (lane == 0) sh_cR = o.cR;
      for (float* c : {&o.cA, &o.cB, &o.cP, &o.cX})
        *c = __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, *c)));
      lds_barrier();  // 3
      finish();
      if (lane == 0) write_row(p, row, o, count);
      // the list's gradient; the bitmap is emptied
      for (int i = lane; i < p.k; i += kWave) {
        const int id = li[i];
        done_id[i] = id;
        if (id < 0) continue;
        const float q = ex2(log2_of(ld_row.ref, lz[i])) * o.ql;
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
  // and spilled 63 registers).  Rows go through buffer resources of the vectors that cover
  // them, which read zeros past their end (0 bytes where there is no next row; without the
  // vector that reaches past the array, which is loaded on its own).
  constexpr uint32_t kDropped = 0x7fffff00u;  // an offset past every row
  u32x4 w[NV];
  // the first NS vectors of a row go through LDS, straight from memory: their loads
  // are issued as soon as the row before is summed, and run while its coefficients are made
  auto stage_row = [&](const rsrc_t& rs) {
#pragma unroll
    for (int v = 0; v < NS; ++v)
      bld16_lds(rs, stage + v * BLK + wv * kWave, uint32_t(tid) * 16u, uint32_t(v) * (BLK * 16u));
  };
  auto load_row_vec = [&](const rsrc_t& rs, int v) { w[v] = bld16(rs, uint32_t(tid) * 16u, uint32_t(v) * (BLK * 16u)); };
  auto row_rsrc = [&](int64_t r, bool there) {
    const Rv rv(r, p.R, p.V);
    return make_rsrc(static_cast<const uint8_t*>(p.zd) + rv.g0 * 16, there ? uint32_t(rv.nfull) * 16u : 0u);
  };
  // a wave-uniform number that the compiler takes as new, so that it makes the
  // conditions that follow from it where they are used, not once for every vector
  auto fresh = [](int x) {
    asm volatile("" : "+s"(x));
    return x;
  };
  {
    const rsrc_t rs = row_rsrc(blockIdx.x, true);
    stage_row(rs);
    // The row's first wait is for all but the NV - NS youngest loads, so none of those may go
    // before one into LDS: nothing else orders them, and the last staged vectors would be read
    // before they are there.
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int v = NS; v < NV; ++v) {
      load_row_vec(rs, v);
      __builtin_amdgcn_sched_barrier(0);  // in the order in which they are waited for
    }
  }
  for (int64_t row = blockIdx.x; row < p.R; row += grid) {
    const Rv rv(row, p.R, p.V);
    const int last_v = fresh((rv.ng - 1) / BLK), last_t = fresh((rv.ng - 1) % BLK);
    lds_barrier();  // 1
    float m = kNegInf, s = 0.f;  // of the unlisted entries; s against own_ref(m)
    auto fold = [&](const u32x4& wx, int v) {
      float x[E];
      unpackv<TI>(wx, x);
      const uint32_t bits = listed_bits<E>(map, v * BLK + tid);
      if (bits)
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (bits >> e & 1u) x[e] = kNegInf;
      float cm = m;
#pragma unroll
      for (int e = 0; e < E; ++e) cm = fmaxf(cm, x[e]);
      const float at = own_ref(cm, p.scd);
      const float keep = ex2(own_ref(m, p.scd) - at);
      m = cm;
#pragma unroll
      for (int e = 0; e < E; ++e) x[e] = ex2(__builtin_fmaf(x[e], p.scd, -at));
      s = __builtin_fmaf(s, keep, tree_sum(x));
    };
    // the staged vectors are older than the NV - NS loads of the others
    wait_vmem_le<NV - NS>();
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      if (v < NS) w[v] = stage[v * BLK + tid];
      if constexpr (!VEC)
        if (v == 0 && tid == 0 && rv.ng > 1 && !rv.whole(0)) w[0] = rv.edge(p.zd, 0, w[0]);
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
      if (tid == last_t && !rv.whole(rv.ng - 1)) {
        if (rv.ng > rv.nfull) wl = rv.raw(p.zd, rv.ng - 1);
        wl = rv.edge(p.zd, rv.ng - 1, wl);
      }
    pin(wl);
    fold(wl, last_v);
    wait_vmem_all();  // the stores of the row before are done
    const int64_t next = row + grid;
    const bool more = next < p.R;
    const rsrc_t rsn = row_rsrc(more ? next : row, more);
    stage_row(rsn);
    {
      const float M = wave_max(m);
      s = wave_sum(s * ex2(own_ref(m, p.scd) - own_ref(M, p.scd)));
      if (lane == 0) {
        sh_m[wv] = M;
        sh_s[wv] = s;
      }
      m = M;
    }
    lds_barrier();  // 2
    m = wave_max(lane < WK ? sh_m[lane] : kNegInf);
    const RowRef ref = row_ref(m, p.scd);
    const float msc = ref.steep ? 0.f : ref.msc;
    if (ref.steep) {
      // the sum again, from differences to the reference, which take the logits' place: exact in their type
      // up to half the reference, and far below every exponential beyond
      s = 0.f;
      auto again = [&](u32x4& wx, int v) {
        float x[E];
        unpackv<TI>(wx, x);
        const uint32_t bits = listed_bits<E>(map, v * BLK + tid);
#pragma unroll
        for (int e = 0; e < E; ++e) {
          x[e] -= ref.m;
          s += bits >> e & 1u ? 0.f : ex2(x[e] * p.scd);
        }
        wx = packv<TI>(x);
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
    const float cR = sh_cR;
    const int last_v3 = fresh(grad != nullptr ? last_v : -1);
    // the vectors inside the row by 16 bytes, dropped past its last one; of a ragged row's first and
    // last vector the row's elements one by one
    const rsrc_t gr = make_rsrc(static_cast<uint8_t*>(grad) + rv.g0 * (E * GS), uint32_t(rv.nfull) * (E * GS));
    auto store = [&](const u32x4& wx, int v, bool ends) {
      const int gi = v * BLK + tid;
      float x[E];
      unpackv<TI>(wx, x);
#pragma unroll
      for (int e = 0; e < E; ++e) x[e] = cR * ex2(__builtin_fmaf(x[e], p.scd, -msc));
      store_g<TG, E>(gr, VEC || !ends || rv.whole(gi) ? uint32_t(gi) * (E * GS) : kDropped, x);
      if constexpr (!VEC)
        if (ends && gi < rv.ng && !rv.whole(gi)) {
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
    if (last_v3 >= 0) store(wl, last_v, true);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      if (v < last_v3) {
        pin(w[v]);  // the packed vector was kept, not unpacked copies of it
        store(w[v], v, v == 0);
      }
      if (v >= NS) load_row_vec(rsn, v);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  wait_vmem_all();
  lds_barrier();  // the last stores
}

// Empties the acceptances' words and sets the error word.
__global__ void k_top_clear(uint64_t* p, int64_t n, unsigned* err, unsigned value) {
  const int64_t stride = int64_t(gridDim.x) * blockDim.x;
  const int64_t t = int64_t(blockIdx.x) * blockDim.x + threadIdx.x;
  for (int64_t i = t; i < n; i += stride) p[i] = 0;
  if (t == 0) *err = value;
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

// WK, NV and NS by the vectors that cover a row: the fewest vectors a thread that
// hold it in as many workgroups as 16 to 24 wavefronts of a CU make.  us per WTV call with
// lists of 64: 14,336 rows of 32,000 bf16 386 with 7 x 9 (3 workgroups a CU), 470 with 7 x 18, 510 in the
// multi-kernel schedule; of 50,000, 626 with 7 x 14, 758 with 7 x 20 (one workgroup a CU then); of
// 16,032, 213 with 3 x 12, 235 with 3 x 18, 241 with 7 x 9; of 8,000, 123 with 2 x 9, 132 with
// 1 x 18.  More vectors a thread than the row has cost loads that read nothing: rows of 50,176, the
// most that 7 x 14 holds, 7,168 of them, 310; of 50,257 with 7 x 19 344 (multi-kernel 457).  Rows of
// 1,000 are no slower in either schedule, 50 and 48.
template <class TI, class TG, bool VEC, bool COUPLED>
hipError_t fused_size(const TopLossArgs& a, bool* used) {
  const int ng = a.V / TI::kVec + (VEC ? 0 : 2);  // vectors that cover a row, at most
  if (a.R * a.V < TI::kVec) return hipSuccess;    // less than a vector in all
#define AAL_FUSED(WK, NV, NS) \
  if (ng <= WK * kWave * NV) return fused_launch<TI, TG, VEC, WK, NV, NS, COUPLED>(a, used)
  AAL_FUSED(1, 9, 4);
  AAL_FUSED(2, 9, 4);
  AAL_FUSED(3, 12, 4);
  AAL_FUSED(7, 9, 4);
  AAL_FUSED(7, 14, 6);
  AAL_FUSED(7, 19, 8);
  AAL_FUSED(15, 14, 8);
  AAL_FUSED(15, 17, 8);
  AAL_FUSED(15, 20, 8);
#undef AAL_FUSED
  return hipSuccess;
}

template <class TI, class TG, bool VEC>
hipError_t fused_coupled(const TopLossArgs& a, bool* used) {
  return a.w_wtv != 0.f || a.w_eal != 0.f ? fused_size<TI, TG, VEC, true>(a, used) : fused_size<TI, TG, VEC, false>(a, used);
}

}  // namespace
}  // namespace aal
