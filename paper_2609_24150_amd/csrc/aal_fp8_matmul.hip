// The product of 8-bit operands (aal_fp8_matmul): its launch, and the sum of the parts where the
// inner dimension is cut.  The kernels are in aal_fp8_matmul.h, the cut is aal_fp8_plan.h's.
#include "aal_fp8_matmul.h"

#include <algorithm>

namespace aal {
extern template hipError_t launch_matmul_formats<0, 0>(const MatmulArgs&, const MatmulParams&, const MatmulPlan&);
extern template hipError_t launch_matmul_formats<0, 1>(const MatmulArgs&, const MatmulParams&, const MatmulPlan&);
extern template hipError_t launch_matmul_formats<1, 0>(const MatmulArgs&, const MatmulParams&, const MatmulPlan&);
extern template hipError_t launch_matmul_formats<1, 1>(const MatmulArgs&, const MatmulParams&, const MatmulPlan&);

namespace {

__global__ __launch_bounds__(256) void k_join(const float* part, int64_t n, int splits, void* c, int out_bf16) {
  const int64_t i = (int64_t(blockIdx.x) * 256 + threadIdx.x) * 4;
  if (i >= n) return;
  float s[4] = {0.f, 0.f, 0.f, 0.f};
  if (i + 4 <= n) {
    typedef f32x4 f32x4_e4 __attribute__((aligned(4)));
#pragma unroll 4
    for (int k = 0; k < splits; ++k) {
      const f32x4 v = *reinterpret_cast<const f32x4_e4*>(part + k * n + i);
#pragma unroll
      for (int u = 0; u < 4; ++u) s[u] += v[u];
    }
  } else {
    for (int k = 0; k < splits; ++k)
      for (int u = 0; u < int(n - i); ++u) s[u] += part[k * n + i + u];
  }
  store4(c, i, s[0], s[1], s[2], s[3], n - i, out_bf16);
}

}  // namespace

size_t matmul_workspace_bytes(int64_t M, int64_t N, int64_t K) {
  const int splits = std::max(plan_of(M, N, K, false).splits, plan_of(M, N, K, true).splits);  // an upper bound
  return splits > 1 ? align256(size_t(splits) * size_t(M) * size_t(N) * sizeof(float)) : 0;
}

hipError_t launch_matmul(const MatmulArgs& a) {
  const MatmulPlan plan = plan_of(a.M, a.N, a.K, a.out == DType::kF32);
  MatmulParams p{};
  p.a = a.a.v;
  p.b = a.b.v;
  p.sa = a.a.s;
  p.sb = a.b.s;
  p.sa_row = a.a.s_row;
  p.sa_block = a.a.s_block;
  p.sb_row = a.b.s_row;
  p.sb_block = a.b.s_block;
  p.M = a.M;
  p.N = a.N;
  p.ld_a = int(a.a.ld);
  p.ld_b = int(a.b.ld);
  p.K = int(a.K);
  p.blocks = int(up(a.K, kFp8Block));
  p.per_split = int(up(p.blocks, plan.splits));
  p.splits = int(up(p.blocks, p.per_split));
  p.ra = a.a.block_rows == 1 ? 0 : 7;
  p.rb = a.b.block_rows == 1 ? 0 : 7;
  p.e8m0 = a.st == Scale::kE8M0;
  const int64_t bm = plan.kind == 0 ? 32 : plan.kind == 1 ? 128 : 256, bn = plan.kind == 0 ? 128 : bm;
  p.tiles_m = int(up(a.M, bm));
  p.tiles_n = int(up(a.N, bn));
  p.c = a.c;
  p.part = static_cast<float*>(a.ws);
  p.out_bf16 = a.out == DType::kBf16;
  hipError_t e;
  if (a.a.format == 0)
    e = a.b.format == 0 ? launch_matmul_formats<0, 0>(a, p, plan) : launch_matmul_formats<0, 1>(a, p, plan);
  else
    e = a.b.format == 0 ? launch_matmul_formats<1, 0>(a, p, plan) : launch_matmul_formats<1, 1>(a, p, plan);
  if (e != hipSuccess || p.splits == 1) return e;
  const int64_t n = a.M * a.N;
  k_join<<<dim3(unsigned(up(n, 1024))), 256, 0, a.stream>>>(p.part, n, p.splits, a.c, p.out_bf16);
  return hipGetLastError();
}

}  // namespace aal
