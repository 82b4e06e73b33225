// Quantisation to 8-bit floating point with a power of two for each block of
// 128 (aal_fp8_quantize):
//
//   s = 2^e, e the least with max |x| 2^-e <= the format's largest value;  q = x / s to nearest even
//
// The division is exact, so q is rounded once.  A power of two costs a floating format no digit
// (values near a block's largest keep all of theirs) and is what the matrix instructions apply
// by themselves.
//
// Bound by memory where values have 4 bytes, by the arithmetic (14 instructions a value) where they have 2.  k_quant_rows, for blocks of 1 x 128 in the order of x, takes a block per 16 lanes, whose
// largest value is found by four lane exchanges; k_quant_tile takes tiles of 128 x 128 into registers,
// 8 x 8 values per thread, for blocks of 128 x 128 and for the transposed order: a
// thread's 8 rows are the 8 bytes that it writes of a transposed row, which goes through LDS
// to leave in whole lines.
#include "aal_fp8_device.h"

#include <algorithm>
#include <type_traits>

namespace aal {
namespace {

struct QuantParams {
  const void* x;
  int64_t rows, cols, ld;
  uint8_t* q;
  int64_t ld_q;
  void* scale;
  uint8_t* qt;
  int64_t ld_qt;
  void* scale_t;
  int64_t first;  // row of workgroups that the launch starts with
};

// Eight values of a row as they are stored.
template <class TI>
struct Eight {
  static constexpr int kWords = TI::kVec == 8 ? 4 : 8;
  uint32_t w[kWords];
  __device__ __forceinline__ void values(float (&x)[8]) const {
#pragma unroll
    for (int u = 0; u < kWords / 4; ++u) {
      float y[TI::kVec];
      TI::unpack(make_uint4(w[4 * u], w[4 * u + 1], w[4 * u + 2], w[4 * u + 3]), y);
#pragma unroll
      for (int e = 0; e < TI::kVec; ++e) x[u * TI::kVec + e] = y[e];
    }
  }
};

// Those of row r from column c on, 0 behind the row's end.
template <class TI>
__device__ __forceinline__ Eight<TI> load8(const QuantParams& p, int64_t r, int64_t c) {
  using T = typename TI::storage;
  const T* at = static_cast<const T*>(p.x) + r * p.ld + c;
  Eight<TI> x{};
  if (r >= p.rows) return x;
  if (c + 8 <= p.cols) {
#pragma unroll
    for (int u = 0; u < Eight<TI>::kWords / 4; ++u) {
      const u32x4 v = __builtin_nontemporal_load(reinterpret_cast<const u32x4_e2*>(at + u * TI::kVec));
#pragma unroll
      for (int i = 0; i < 4; ++i) x.w[4 * u + i] = v[i];
    }
  } else {
    T v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = c + e < p.cols ? at[e] : T(0);
    __builtin_memcpy(&x, v, sizeof x);
  }
  return x;
}

// Largest magnitudes, as bits of fp32, of the rows and of the columns of N x 8 values; what is not finite counts as 0.
// bf16 by pairs, magnitudes being whole numbers that order as they do; values that are not finite show in the
// result, and only then every value is looked at.
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t max_pair(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
}
template <class TI, int N>
__device__ __forceinline__ void maxima(const Eight<TI> (&x)[N], uint32_t (&rows)[N], uint32_t (&cols)[8]) {
  uint32_t all = 0;
  if constexpr (TI::kVec == 8) {
    uint32_t c[4] = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < N; ++i) {
      uint32_t a[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        a[k] = x[i].w[k] & 0x7fff7fffu;
        c[k] = max_pair(c[k], a[k]);
      }
      const uint32_t m = max_pair(max_pair(a[0], a[1]), max_pair(a[2], a[3]));
      rows[i] = max(m << 16, m & 0xffff0000u);
      all = max(all, rows[i]);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      cols[2 * k] = c[k] << 16;
      cols[2 * k + 1] = c[k] & 0xffff0000u;
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) cols[e] = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      rows[i] = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t a = x[i].w[e % Eight<TI>::kWords] & 0x7fffffffu;
        rows[i] = max(rows[i], a);
        cols[e] = max(cols[e], a);
      }
      all = max(all, rows[i]);
    }
  }
  if (all < 0x7f800000u) return;
#pragma unroll
  for (int e = 0; e < 8; ++e) cols[e] = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    float v[8];
    x[i].values(v);
    rows[i] = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      rows[i] = max(rows[i], finite_bits(v[e]));
      cols[e] = max(cols[e], finite_bits(v[e]));
    }
  }
}

// 8 bytes at `to`, of which n lie inside the row.
__device__ __forceinline__ void store8(uint8_t* to, uint32_t lo, uint32_t hi, int64_t n) {
  if (n >= 8) {
    const u32x2 w = {lo, hi};
    *reinterpret_cast<u32x2*>(to) = w;
  } else {
    const uint64_t w = uint64_t(hi) << 32 | lo;
    for (int e = 0; e < int(n); ++e) to[e] = uint8_t(w >> (8 * e));
  }
}

template <Scale S>
__device__ __forceinline__ void store_scale(void* to, int64_t i, int e) {
  if constexpr (S == Scale::kF32)
    static_cast<float*>(to)[i] = power_of_two(e);
  else
    static_cast<uint8_t*>(to)[i] = uint8_t(e + 127);
}

// The largest over the 16 lanes of a row of the wave.
__device__ __forceinline__ uint32_t row16_max(uint32_t v) {
  v = max(v, uint32_t(__builtin_amdgcn_mov_dpp(int(v), 0xB1, 0xF, 0xF, true)));
  v = max(v, uint32_t(__builtin_amdgcn_mov_dpp(int(v), 0x4E, 0xF, 0xF, true)));
  v = max(v, uint32_t(__builtin_amdgcn_mov_dpp(int(v), 0x141, 0xF, 0xF, true)));
  return max(v, uint32_t(__builtin_amdgcn_mov_dpp(int(v), 0x140, 0xF, 0xF, true)));
}

// A workgroup takes 16 rows of 512 columns, a wave four rows of them.
template <class TI, Fp8 F, Scale S>
__global__ __launch_bounds__(256) void k_quant_rows(QuantParams p, int col_groups) {
  constexpr int R = 4;
  __shared__ int se[4][16];
  const int lane = threadIdx.x & (kWave - 1), wv = threadIdx.x / kWave;
  const int64_t rg = p.first + blockIdx.x / col_groups, cg = blockIdx.x % col_groups;
  const int64_t r0 = rg * 16 + wv * R, c = cg * 512 + lane * 8;
  Eight<TI> raw[R];
  uint32_t rows[R], cols[8];
#pragma unroll
  for (int i = 0; i < R; ++i) raw[i] = load8<TI>(p, r0 + i, c);
  maxima<TI>(raw, rows, cols);
#pragma unroll
  for (int i = 0; i < R; ++i) {
    float x[8];
    raw[i].values(x);
    const int e = scale_exponent<F>(row16_max(rows[i]));
    const float inv = power_of_two(-e);
    if ((lane & 15) == 0) se[lane / 16][wv * R + i] = e;
    if (r0 + i < p.rows && c < p.cols)
      store8(p.q + (r0 + i) * p.ld_q + c, pack_fp8<F>(x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv),
             pack_fp8<F>(x[4] * inv, x[5] * inv, x[6] * inv, x[7] * inv), p.cols - c);
  }
  __syncthreads();
  if (threadIdx.x < 64) {
    const int64_t j = cg * 4 + threadIdx.x / 16, r = rg * 16 + threadIdx.x % 16;
    if (j * kFp8Block < p.cols && r < p.rows) store_scale<S>(p.scale, j * p.rows + r, se[threadIdx.x / 16][threadIdx.x % 16]);
  }
}

// A workgroup takes 128 rows of T blocks of columns: 16 T threads for the columns, 16 groups of 8 rows.  T: as many as
// make 512 bytes of a row of x (128 columns of bf16 at a time cost 3% more, 256 of fp32 15 to 25%, tiles down before across 6%).  2,048 x 128,256
// bf16 in both orders 229 us, 4.6 TB/s; 32,000 x 4,096 fp32 in blocks of 128 x 128 137 us, 5.8 TB/s.
template <class TI, Fp8 F, Scale S, bool SQUARE, int T>
__global__ __launch_bounds__(256 * T) void k_quant_tile(QuantParams p, int col_groups) {
  constexpr int WV = 4 * T, kCols = kFp8Block * T;
  __shared__ uint32_t part[WV][kCols];
  __shared__ int ce[kCols];
  alignas(16) __shared__ uint8_t turn[kCols * kFp8Block];
  // a column's 16 pieces of 8 rows stand in an order that its neighbours, which are written at a time, do not share
  auto turned = [&](int c, int r) { return &turn[c * kFp8Block + ((r / 8) ^ (c / 8 % 16)) * 8]; };
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wv = tid / kWave;
  const int64_t rb = p.first + blockIdx.x / col_groups, cg = blockIdx.x % col_groups;
  const int rl = tid / (16 * T) * 8, cl = tid % (16 * T) * 8;  // in the tile
  const int64_t r0 = rb * kFp8Block + rl, c0 = cg * kCols + cl;
  const int64_t row_blocks = (p.rows + kFp8Block - 1) / kFp8Block, col_blocks = (p.cols + kFp8Block - 1) / kFp8Block;
  const int64_t cb = cg * T + cl / kFp8Block;  // the thread's block of columns
  Eight<TI> raw[8];
  uint32_t rows[8], cols[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) raw[i] = load8<TI>(p, r0 + i, c0);
  maxima<TI>(raw, rows, cols);
  int er[8], ec[8];
  // the largest over the row groups of the wave that share a column
  auto rows_max = [&](uint32_t m) {
    if constexpr (T == 1) m = max(m, uint32_t(__shfl_xor(int(m), 16, kWave)));
    return max(m, uint32_t(__shfl_xor(int(m), 32, kWave)));
  };
  if constexpr (SQUARE) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, rows[i]);
    m = rows_max(row16_max(m));
    if (lane % 16 == 0 && lane < 16 * T) part[wv][lane / 16] = m;
    __syncthreads();
    m = 0;
#pragma unroll
    for (int w = 0; w < WV; ++w) m = max(m, part[w][cl / kFp8Block]);
    const int e = scale_exponent<F>(m);
#pragma unroll
    for (int i = 0; i < 8; ++i) er[i] = ec[i] = e;
    if (rl == 0 && cl % kFp8Block == 0 && cb < col_blocks) {
      if (p.q) store_scale<S>(p.scale, cb * row_blocks + rb, e);
      if (p.qt) store_scale<S>(p.scale_t, rb * col_blocks + cb, e);
    }
  } else {
    if (p.q) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        er[i] = scale_exponent<F>(row16_max(rows[i]));
        if (cl % kFp8Block == 0 && cb < col_blocks && r0 + i < p.rows) store_scale<S>(p.scale, cb * p.rows + r0 + i, er[i]);
      }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t m = rows_max(cols[e]);
      if (lane < 16 * T) part[wv][cl + e] = m;
    }
    __syncthreads();
    for (int i = tid; i < kCols; i += 256 * T) {
      uint32_t m = 0;
#pragma unroll
      for (int w = 0; w < WV; ++w) m = max(m, part[w][i]);
      const int e = scale_exponent<F>(m);
      ce[i] = e;
      const int64_t c = cg * kCols + i;
      if (c < p.cols) store_scale<S>(p.scale_t, rb * p.cols + c, e);
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 8; ++e) ec[e] = ce[cl + e];
  }
  float x[8][8];
#pragma unroll
  for (int i = 0; i < 8; ++i) raw[i].values(x[i]);
  if (p.q) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (r0 + i >= p.rows || c0 >= p.cols) continue;
      const float inv = power_of_two(-er[i]);
      store8(p.q + (r0 + i) * p.ld_q + c0,
             pack_fp8<F>(x[i][0] * inv, x[i][1] * inv, x[i][2] * inv, x[i][3] * inv),
             pack_fp8<F>(x[i][4] * inv, x[i][5] * inv, x[i][6] * inv, x[i][7] * inv), p.cols - c0);
    }
  }
  if (p.qt == nullptr) return;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float inv = power_of_two(-ec[e]);
    const u32x2 w = {pack_fp8<F>(x[0][e] * inv, x[1][e] * inv, x[2][e] * inv, x[3][e] * inv),
                     pack_fp8<F>(x[4][e] * inv, x[5][e] * inv, x[6][e] * inv, x[7][e] * inv)};
    *reinterpret_cast<u32x2*>(turned(cl + e, rl)) = w;
  }
  __syncthreads();
  // 16 threads write a transposed row's 128 bytes
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int c = tid / 16 + i * 16 * T, r = tid % 16 * 8;
    const int64_t gc = cg * kCols + c, gr = rb * kFp8Block + r;
    if (gc >= p.cols || gr >= p.rows) continue;
    const u32x2 w = *reinterpret_cast<const u32x2*>(turned(c, r));
    store8(p.qt + gc * p.ld_qt + gr, w.x, w.y, p.rows - gr);
  }
}

template <class TI, Fp8 F, Scale S>
hipError_t launch_typed(const QuantizeArgs& a) {
  QuantParams p{a.x, a.rows, a.cols, a.ld, a.q, a.ld_q, a.scale, a.qt, a.ld_qt, a.scale_t, 0};
  const bool tiles = a.block_rows != 1 || a.qt != nullptr;
  const int64_t down = tiles ? (a.rows + 127) / 128 : (a.rows + 15) / 16;
  constexpr int T = TI::kVec == 8 ? 2 : 1;
  const int64_t across = tiles ? (a.cols + 128 * T - 1) / (128 * T) : (a.cols + 511) / 512;
  // a launch holds fewer than 2^32 threads: up to 2^22 workgroups, or a row of them (cols <= 2^30: 2^22, or 2^23 of 256)
  const int64_t most = std::max<int64_t>(1, (int64_t(1) << 22) / across);
  for (; p.first < down; p.first += most) {
    const dim3 grid(unsigned((down - p.first < most ? down - p.first : most) * across));
    if (!tiles)
      k_quant_rows<TI, F, S><<<grid, 256, 0, a.stream>>>(p, int(across));
    else if (a.block_rows == 1)
      k_quant_tile<TI, F, S, false, T><<<grid, 256 * T, 0, a.stream>>>(p, int(across));
    else
      k_quant_tile<TI, F, S, true, T><<<grid, 256 * T, 0, a.stream>>>(p, int(across));
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_quantize(const QuantizeArgs& a) {
  auto with = [&](auto in, auto st) {
    using TI = decltype(in);
    constexpr Scale S = decltype(st)::value;
    return a.format == Fp8::kE4M3 ? launch_typed<TI, Fp8::kE4M3, S>(a) : launch_typed<TI, Fp8::kE5M2, S>(a);
  };
  using F = std::integral_constant<Scale, Scale::kF32>;
  using E = std::integral_constant<Scale, Scale::kE8M0>;
  if (a.in == DType::kBf16) return a.st == Scale::kF32 ? with(Bf16{}, F{}) : with(Bf16{}, E{});
  return a.st == Scale::kF32 ? with(F32{}, F{}) : with(F32{}, E{});
}

}  // namespace aal
