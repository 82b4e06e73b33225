// The product of two operands in 8-bit floating point with a scale for each
// block of 128 (aal_fp8_matmul):
//
//   c[m, n] = sum_j sa[m, j] sb[n, j] sum_{k in block j} a[m, k] b[n, k]
//
// One wavefront for each 32 x 32 piece of c: a block of 128 is two matrix instructions of 32 x 32 x 64, their
// result is scaled and added in fp32.  The rows of b go down the matrix tile and those of a
// across, so that a lane holds four consecutive columns of one row of c.
#include "aal_fp8_device.h"

#include <type_traits>

namespace aal {
namespace {

// Bytes [at, at + 32) of a row of K values at `row` (null: none), 0 where they lie outside.
__device__ __forceinline__ i32x8 load32(const uint8_t* row, int64_t at, int64_t K) {
  i32x8 r = {0, 0, 0, 0, 0, 0, 0, 0};
  if (row == nullptr || at >= K) return r;
  const int64_t n = K - at;
  const u32x4 lo = *reinterpret_cast<const u32x4*>(row + at);
  u32x4 hi = {0, 0, 0, 0};
  if (n > 16) hi = *reinterpret_cast<const u32x4*>(row + at + 16);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    r[i] = int(lo[i]);
    r[i + 4] = int(hi[i]);
  }
  if (n < 32) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int bytes = int(n) - 4 * i;
      if (bytes < 4) r[i] = bytes <= 0 ? 0 : int(uint32_t(r[i]) & ((1u << (8 * bytes)) - 1u));
    }
  }
  return r;
}

template <int FA, int FB, Scale S, class TC>
__global__ __launch_bounds__(64) void k_matmul(MatmulArgs p, int64_t tiles_n) {
  const int lane = threadIdx.x, l = lane & 31, h = lane >> 5;
  const int64_t m = blockIdx.x / tiles_n * 32 + l, n = blockIdx.x % tiles_n * 32;
  const uint8_t* ra = m < p.M ? p.a.v + m * p.a.ld : nullptr;
  const uint8_t* rb = n + l < p.N ? p.b.v + (n + l) * p.b.ld : nullptr;
  f32x16 sum = {};
  for (int64_t j = 0; j * kFp8Block < p.K; ++j) {
    f32x16 t = {};
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int64_t at = j * kFp8Block + u * 64 + h * 32;
      t = dot64<std::is_same_v<TC, GF32>, FB, FA>(load32(rb, at, p.K), load32(ra, at, p.K), t);
    }
    const float sa = m < p.M ? load_scale<S>(p.a.s, m / p.a.block_rows * p.a.s_row + j * p.a.s_block) : 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int64_t c = n + (i / 4) * 8 + h * 4 + i % 4;
      const float sb = c < p.N ? load_scale<S>(p.b.s, c / p.b.block_rows * p.b.s_row + j * p.b.s_block) : 0.f;
      sum[i] = __builtin_fmaf(t[i], sa * sb, sum[i]);
    }
  }
  if (m >= p.M) return;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int64_t c = n + (i / 4) * 8 + h * 4 + i % 4;
    if (c < p.N) TC::store1(p.c, m * p.N + c, sum[i]);
  }
}

template <int FA, int FB, Scale S, class TC>
hipError_t launch_typed(const MatmulArgs& a) {
  const int64_t tn = (a.N + 31) / 32, tm = (a.M + 31) / 32;
  k_matmul<FA, FB, S, TC><<<dim3(unsigned(tn * tm)), 64, 0, a.stream>>>(a, tn);
  return hipGetLastError();
}

template <Scale S, class TC>
hipError_t with_formats(const MatmulArgs& a) {
  if (a.a.format == 0) return a.b.format == 0 ? launch_typed<0, 0, S, TC>(a) : launch_typed<0, 1, S, TC>(a);
  return a.b.format == 0 ? launch_typed<1, 0, S, TC>(a) : launch_typed<1, 1, S, TC>(a);
}

}  // namespace

size_t matmul_workspace_bytes(int64_t, int64_t, int64_t) { return 0; }

hipError_t launch_matmul(const MatmulArgs& a) {
  if (a.st == Scale::kF32)
    return a.out == DType::kBf16 ? with_formats<Scale::kF32, GBf16>(a) : with_formats<Scale::kF32, GF32>(a);
  return a.out == DType::kBf16 ? with_formats<Scale::kE8M0, GBf16>(a) : with_formats<Scale::kE8M0, GF32>(a);
}

}  // namespace aal
