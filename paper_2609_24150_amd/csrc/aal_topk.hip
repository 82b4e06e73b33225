// A row's k largest logits with their ids, and the log-sum-exp of the others
// (aal_topk_logits): what a training set stores of a target's logits.
//
//   order: v before w iff z_v > z_w, or z_v = z_w and v < w
//   rest  = ln sum_{v not among the k} exp(z_v / T)
//
// k_topk_rows, one workgroup per row, every shape: a radix select over the
// order-preserving whole number of a logit (two 8-bit digits for bf16, four
// for fp32) gives the k-th largest value and how many of its ties are wanted;
// a pass in index order then collects the larger entries and the first ties
// and sums 2^(z sc - max sc) over all others, so that the remainder does not
// come from a difference of sums; the k entries are ranked by counting.
#include "aal_device.h"
#include "aal_rowops.h"
#include "aal_toplist.h"

namespace aal {
namespace {

constexpr int kTopkMax = 512;
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

template <class TI, bool VEC, int BLK>
__global__ __launch_bounds__(BLK) void k_topk_rows(const void* __restrict__ z, int64_t rows, int V, int k, float sc,
                                                   void* __restrict__ top, int32_t* __restrict__ ids,
                                                   float* __restrict__ rest) {
  using Rv = RowVecs<TI, VEC>;
  constexpr int E = Rv::E;
  constexpr int WV = BLK / kWave;
  __shared__ uint32_t sh_hist[256];
  __shared__ uint64_t sh_top[kTopkMax];
  __shared__ float sh_f[WV];
  __shared__ int sh_i[WV];
  __shared__ uint32_t sh_digit, sh_need, sh_n;

  const int64_t row = blockIdx.x;
  const Rv rv(row, rows, V);
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wv = tid / kWave;

  // the k-th largest key, digit by digit
  uint32_t prefix = 0, need = k;
  float m = kNegInf;
  for (int shift = 24; shift >= 32 - key_bits<TI>(); shift -= 8) {
    for (int i = tid; i < 256; i += BLK) sh_hist[i] = 0;
    __syncthreads();
    for (int gi = tid; gi < rv.ng; gi += BLK) {
      float x[E];
      TI::unpack(to_uint4(rv.load(z, gi)), x);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int v = rv.index(gi, e);
        if (v < 0 || v >= V) continue;
        const uint32_t key = order_key<TI>(x[e]);
        if (shift == 24) m = fmaxf(m, x[e]);
        if (shift == 24 || (key >> (shift + 8)) == (prefix >> (shift + 8)))
          atomicAdd(&sh_hist[(key >> shift) & 255u], 1u);
      }
    }
    __syncthreads();
    if (tid == 0) {
      uint32_t left = need;
      int d = 255;
      while (d > 0 && sh_hist[d] < left) left -= sh_hist[d--];
      sh_digit = uint32_t(d);
      sh_need = left;
    }
    __syncthreads();
    prefix |= sh_digit << shift;
    need = sh_need;  // of the entries whose key starts with `prefix`
  }
  // the row's largest logit
  m = wave_max(m);
  if (lane == 0) sh_f[wv] = m;
  if (tid == 0) sh_n = 0;
  __syncthreads();
  m = sh_f[0];
  for (int i = 1; i < WV; ++i) m = fmaxf(m, sh_f[i]);
  const float msc = m == kNegInf ? 0.f : m * sc;

  // in index order: the larger entries, the first `need` ties, the sum of the others
  uint32_t ties = 0;  // before this round
  float s = 0.f;
  for (int base = 0; base < rv.ng; base += BLK) {
    const int gi = base + tid;
    uint32_t key[E];
    int mine = 0;
    float x[E];
    if (gi < rv.ng) {
      TI::unpack(to_uint4(rv.load(z, gi)), x);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int v = rv.index(gi, e);
        const bool in = v >= 0 && v < V;
        key[e] = in ? order_key<TI>(x[e]) : 0u;  // below every logit's key
        mine += in && key[e] == prefix;
      }
    }
    // ties of the lanes and waves before this thread
    int before = mine;
    for (int off = 1; off < kWave; off <<= 1) {
      const int o = __shfl_up(before, off, kWave);
      if (lane >= off) before += o;
    }
    __syncthreads();
    if (lane == kWave - 1) sh_i[wv] = before;
    __syncthreads();
    uint32_t at = ties + uint32_t(before - mine);
    for (int i = 0; i < WV; ++i) {
      if (i < wv) at += uint32_t(sh_i[i]);
      ties += uint32_t(sh_i[i]);
    }
    if (gi >= rv.ng) continue;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int v = rv.index(gi, e);
      if (v < 0 || v >= V) continue;
      const bool tie = key[e] == prefix;
      if (key[e] > prefix || (tie && at < need)) {
        const uint32_t slot = atomicAdd(&sh_n, 1u);
        if (slot < uint32_t(k)) sh_top[slot] = (uint64_t(key[e]) << 32) | (0xffffffffu - uint32_t(v));
      } else {
        s += ex2(__builtin_fmaf(x[e], sc, -msc));
      }
      at += tie;
    }
  }
  __syncthreads();
  s = block_sum<WV>(s, sh_f);
  // rank by counting: the keys differ, so the ranks are 0..k-1
  const int64_t e0 = row * int64_t(V), o0 = row * int64_t(k);
  for (int i = tid; i < k; i += BLK) {
    const uint64_t mykey = sh_top[i];
    int rank = 0;
    for (int j = 0; j < k; ++j) rank += sh_top[j] > mykey;
    const int v = int(0xffffffffu - uint32_t(mykey));
    ids[o0 + rank] = v;
    static_cast<typename TI::storage*>(top)[o0 + rank] = static_cast<const typename TI::storage*>(z)[e0 + v];
  }
  if (rest != nullptr && tid == 0) rest[row] = s > 0.f ? (msc + __log2f(s)) * kLn2 : kNegInf;
}

template <class TI, bool VEC>
hipError_t launch_vec(const TopkArgs& a) {
  k_topk_rows<TI, VEC, 256><<<dim3(unsigned(a.rows)), 256, 0, a.stream>>>(a.z, a.rows, a.V, a.k, a.sc, a.top, a.ids,
                                                                        a.rest);
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
