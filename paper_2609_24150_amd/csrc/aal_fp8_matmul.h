// Kernels of the product of 8-bit operands (aal_fp8_matmul), by formats:
//
//   c[m, n] = sum_j sa[m, j] sb[n, j] sum_{k in block j} a[m, k] b[n, k]
//
// Rows of b go down the matrix instructions' tiles and rows of a across: a lane holds four
// consecutive columns n of one row m of c, and its row's scale is one value.  A block's 128 values are two
// instructions' worth, whose sum is scaled and added in fp32.
#pragma once

#include "aal_fp8_device.h"

#include <type_traits>

namespace aal {

// How a product is cut (plan_of): few rows of a, or tiles of 128 or 256 in both directions; the inner
// dimension in `splits` parts, whose sums are joined by a second kernel.
struct MatmulPlan {
  int kind;  // 0: few rows, 1: tiles of 128 x 128, 2: of 256 x 256
  int splits;
};

struct MatmulParams {
  const uint8_t* a;
  const uint8_t* b;
  const void* sa;
  const void* sb;
  int64_t sa_row, sa_block, sb_row, sb_block;
  int64_t M, N;
  int ld_a, ld_b, K;
  int blocks;        // of 128 of K
  int per_split;     // blocks of a part
  int ra, rb;        // rows of a scale's block, as shifts: 0 or 7
  int e8m0;
  int tiles_m, tiles_n;
  void* c;
  float* part;       // [splits][M][N] where there are several
  int out_bf16;
};

template <int FA, int FB>
hipError_t launch_matmul_formats(const MatmulArgs& a, const MatmulParams& p, const MatmulPlan& plan);

namespace {

typedef __attribute__((address_space(3))) void lds_t;
typedef __amdgpu_buffer_rsrc_t rsrc_t;

__device__ __forceinline__ float scale_at(const void* s, int64_t i, int e8m0) {
  return e8m0 ? load_scale<Scale::kE8M0>(s, i) : load_scale<Scale::kF32>(s, i);
}

// Four consecutive results of a row, of which n exist.
__device__ __forceinline__ void store4(void* c, int64_t at, float x, float y, float z, float w, int64_t n, bool bf16) {
  typedef u32x2 u32x2_e2 __attribute__((aligned(2)));
  typedef f32x4 f32x4_e4 __attribute__((aligned(4)));
  if (n >= 4) {
    if (bf16) {
      const u32x2 v = {pack_bf16x2(x, y), pack_bf16x2(z, w)};
      *reinterpret_cast<u32x2_e2*>(static_cast<uint16_t*>(c) + at) = v;
    } else {
      const f32x4 v = {x, y, z, w};
      *reinterpret_cast<f32x4_e4*>(static_cast<float*>(c) + at) = v;
    }
  } else {
    const float v[4] = {x, y, z, w};
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < n) {
        if (bf16)
          GBf16::store1(c, at + i, v[i]);
        else
          GF32::store1(c, at + i, v[i]);
      }
  }
}

// Waits for this wave's loads into LDS and its LDS accesses, then for the workgroup.
__device__ __forceinline__ void stage_barrier() {
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// ------------------------------------------------------------------ tiles
// A workgroup of WN x WM waves makes 32 TN WN x 32 TM WM results.  Both operands' rows of a block, 128 bytes
// each, are loaded straight into LDS, the next block's while one is being multiplied; 16-byte pieces
// of row r stand at place (piece ^ r % 8), so that the 8 lanes that read at a time meet no bank twice.
template <bool WIDE, int FA, int FB, bool SQUARE, int TN, int TM, int WN, int WM>
__global__ __launch_bounds__(64 * WN * WM) void k_tiles(MatmulParams p) {
  constexpr int NT = 64 * WN * WM, BN = 32 * TN * WN, BM = 32 * TM * WM, RP = NT / 8;  // RP: rows of a round of loads
  static_assert(BN <= NT && BM <= NT, "one scale of either side per thread");
  __shared__ __attribute__((aligned(16))) uint8_t tile[2][(BN + BM) * 128];
  __shared__ __attribute__((aligned(16))) float scales[2][BN + BM];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l = lane & 31, h = lane >> 5;
  // Workgroups go round over the 8 XCDs: each takes a stretch of tiles of its own, in which
  // groups of 8 tiles down run through all of those across, so that its L2 serves both operands' panels.
  const int total = p.tiles_m * p.tiles_n, id = blockIdx.x, x = id & 7, q = total >> 3, rest = total & 7;
  const int at = x * q + min(x, rest) + (id >> 3);
  const int group = at / (8 * p.tiles_n), first = group * 8, rows = min(8, p.tiles_m - first);
  const int in = at - group * 8 * p.tiles_n, tm = first + in % rows, tn = in / rows;
  const int64_t m0 = int64_t(tm) * BM, n0 = int64_t(tn) * BN;
  const int left_m = int(min(int64_t(BM), p.M - m0)), left_n = int(min(int64_t(BN), p.N - n0));
  // rows behind the last one repeat it: what they give is not stored
  const rsrc_t ra = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(p.a) + m0 * p.ld_a, short(0),
                                                      int(uint32_t(left_m) * uint32_t(p.ld_a)), 0x00020000);
  const rsrc_t rb = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(p.b) + n0 * p.ld_b, short(0),
                                                      int(uint32_t(left_n) * uint32_t(p.ld_b)), 0x00020000);
  const int row = tid >> 3, piece = ((tid & 7) ^ (row & 7)) << 4;
  uint32_t va[BM / RP], vb[BN / RP];
#pragma unroll
  for (int i = 0; i < BM / RP; ++i) va[i] = uint32_t(min(row + i * RP, left_m - 1)) * uint32_t(p.ld_a) + piece;
#pragma unroll
  for (int i = 0; i < BN / RP; ++i) vb[i] = uint32_t(min(row + i * RP, left_n - 1)) * uint32_t(p.ld_b) + piece;
  const int j0 = blockIdx.y * p.per_split, j1 = min(p.blocks, j0 + p.per_split);
  auto load = [&](int j, int to) {
    const uint32_t k = uint32_t(j) * 128u;
#pragma unroll
    for (int i = 0; i < BN / RP; ++i)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rb, (lds_t*)&tile[to][(i * RP + wave * 8) * 128], 16, int(vb[i] + k), 0, 0, 0);
#pragma unroll
    for (int i = 0; i < BM / RP; ++i)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(ra, (lds_t*)&tile[to][(BN + i * RP + wave * 8) * 128], 16, int(va[i] + k), 0, 0,
                                               0);
  };
  const int64_t sn = (n0 + min(tid, left_n - 1)) >> p.rb, sm = (m0 + min(tid, left_m - 1)) >> p.ra;
  float next_n = 0.f, next_m = 0.f;
  auto load_scales = [&](int j) {
    if (tid < BN) next_n = scale_at(p.sb, sn * p.sb_row + j * p.sb_block, p.e8m0);
    if (tid < BM) next_m = scale_at(p.sa, sm * p.sa_row + j * p.sa_block, p.e8m0);
  };
  auto put_scales = [&](int to) {
    if (tid < BN) scales[to][tid] = next_n;
    if (tid < BM) scales[to][BN + tid] = next_m;
  };
  // K ends inside the last block: zeros for what lies behind it
  auto clear_tail = [&](int to) {
    const int rem = p.K & 127;
    for (int r = tid; r < BN + BM; r += NT) {
      uint8_t* at = &tile[to][r * 128];
      for (int b = rem; b < 128;) {
        uint8_t* w = at + (((b >> 4) ^ (r & 7)) << 4);
        if ((b & 15) == 0) {
          *reinterpret_cast<u32x4*>(w) = u32x4{0, 0, 0, 0};
          b += 16;
        } else {
          w[b & 15] = 0;
          ++b;
        }
      }
    }
  };
  const int wn = wave % WN, wm = wave / WN;
  f32x16 acc[TN][TM];
#pragma unroll
  for (int i = 0; i < TN; ++i)
#pragma unroll
    for (int j = 0; j < TM; ++j) acc[i][j] = f32x16{};
  auto fragment = [&](const uint8_t* base, int r, int u) {
    const u32x4 lo = *reinterpret_cast<const u32x4*>(base + r * 128 + (((4 * u + 2 * h) ^ (l & 7)) << 4));
    const u32x4 hi = *reinterpret_cast<const u32x4*>(base + r * 128 + (((4 * u + 2 * h + 1) ^ (l & 7)) << 4));
    return i32x8{int(lo.x), int(lo.y), int(lo.z), int(lo.w), int(hi.x), int(hi.y), int(hi.z), int(hi.w)};
  };
  load_scales(j0);
  load(j0, 0);
  put_scales(0);
  stage_barrier();
  if ((p.K & 127) && j0 == p.blocks - 1) {
    clear_tail(0);
    stage_barrier();
  }
  for (int j = j0; j < j1; ++j) {
    const int cur = (j - j0) & 1;
    const bool more = j + 1 < j1;
    if (more) {
      load_scales(j + 1);
      load(j + 1, cur ^ 1);
    }
    const uint8_t* tb = tile[cur];
    const uint8_t* ta = tile[cur] + BN * 128;
    const float* sc = scales[cur];
    i32x8 xa[TM][2];
    float fa[TM];
#pragma unroll
    for (int m = 0; m < TM; ++m) {
      const int r = (wm * TM + m) * 32 + l;
      fa[m] = sc[BN + r];
      xa[m][0] = fragment(ta, r, 0);
      xa[m][1] = fragment(ta, r, 1);
    }
#pragma unroll
    for (int n = 0; n < TN; ++n) {
      const int r0 = (wn * TN + n) * 32;
      const i32x8 xb0 = fragment(tb, r0 + l, 0), xb1 = fragment(tb, r0 + l, 1);
      f32x4 fb[4];
      float fb1 = 0.f;
      if constexpr (SQUARE) {
        fb1 = sc[r0];
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) fb[i] = *reinterpret_cast<const f32x4*>(&sc[r0 + i * 8 + h * 4]);
      }
#pragma unroll
      for (int m = 0; m < TM; ++m) {
        f32x16 t = dot64<WIDE, FB, FA>(xb0, xa[m][0], f32x16{});
        t = dot64<WIDE, FB, FA>(xb1, xa[m][1], t);
        const float f = fa[m] * fb1;
#pragma unroll
        for (int i = 0; i < 16; ++i)
          acc[n][m][i] = __builtin_fmaf(t[i], SQUARE ? f : fa[m] * fb[i / 4][i % 4], acc[n][m][i]);
      }
    }
    if (more) {
      put_scales(cur ^ 1);
      stage_barrier();
      if ((p.K & 127) && j + 1 == p.blocks - 1) {
        clear_tail(cur ^ 1);
        stage_barrier();
      }
    }
  }
  const bool whole = gridDim.y == 1;
  void* c = whole ? p.c : p.part + int64_t(blockIdx.y) * p.M * p.N;
  const bool bf16 = whole && p.out_bf16;
#pragma unroll
  for (int m = 0; m < TM; ++m) {
    const int64_t gm = m0 + (wm * TM + m) * 32 + l;
    if (gm >= p.M) continue;
#pragma unroll
    for (int n = 0; n < TN; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int64_t gn = n0 + (wn * TN + n) * 32 + i * 8 + h * 4;
        if (gn < p.N)
          store4(c, gm * p.N + gn, acc[n][m][4 * i], acc[n][m][4 * i + 1], acc[n][m][4 * i + 2], acc[n][m][4 * i + 3],
                 p.N - gn, bf16);
      }
  }
}

// --------------------------------------------------------------- few rows
// Up to 32 rows of a.  A workgroup takes 64 rows of b, its four waves every fourth block each; b goes from
// memory to registers, since nothing else reads it, the next block's on its way while one is being multiplied.
template <bool WIDE, int FA, int FB, bool SQUARE>
__global__ __launch_bounds__(256) void k_few_rows(MatmulParams p) {
  __shared__ float sums[4][32][65];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l = lane & 31, h = lane >> 5;
  const int64_t n0 = int64_t(blockIdx.x) * 64;
  const int j0 = blockIdx.y * p.per_split, j1 = min(p.blocks, j0 + p.per_split);
  const int64_t m = min(int64_t(l), p.M - 1);
  const uint8_t* ra = p.a + m * p.ld_a;
  const uint8_t* rb[2];
  int64_t sn[2];
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const int64_t n = min(n0 + t * 32 + l, p.N - 1);
    rb[t] = p.b + n * p.ld_b;
    sn[t] = (SQUARE ? min(n0 + t * 32, p.N - 1) : n) >> p.rb;
  }
  struct Block {
    u32x4 a[4], b[2][4];
    float fa, fb[2];
  };
  // a lane's 64 bytes of a row: 16-byte pieces h, 2 + h, 4 + h and 6 + h, the same of either operand
  auto load = [&](int j, Block& r) {
    const int64_t k = int64_t(j) * 128 + h * 16;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const bool in = k + i * 32 < p.K;
#pragma unroll
      for (int t = 0; t < 2; ++t)
        r.b[t][i] = in ? __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(rb[t] + k + i * 32)) : u32x4{0, 0, 0, 0};
      r.a[i] = in ? *reinterpret_cast<const u32x4*>(ra + k + i * 32) : u32x4{0, 0, 0, 0};
    }
    r.fa = scale_at(p.sa, (m >> p.ra) * p.sa_row + j * p.sa_block, p.e8m0);
#pragma unroll
    for (int t = 0; t < 2; ++t) r.fb[t] = scale_at(p.sb, sn[t] * p.sb_row + j * p.sb_block, p.e8m0);
  };
  // bytes behind K, which only the last block has
  auto clear = [&](u32x4& v, int64_t k) {
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const int64_t n = p.K - k - 4 * w;
      v[w] = n >= 4 ? v[w] : n <= 0 ? 0u : v[w] & ((1u << (8 * n)) - 1u);
    }
  };
  auto join = [](const u32x4& lo, const u32x4& hi) {
    return i32x8{int(lo.x), int(lo.y), int(lo.z), int(lo.w), int(hi.x), int(hi.y), int(hi.z), int(hi.w)};
  };
  f32x16 acc[2] = {};
  auto multiply = [&](int j, Block& r) {
    if ((p.K & 127) && j == p.blocks - 1) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int64_t k = int64_t(j) * 128 + h * 16 + i * 32;
        clear(r.a[i], k);
        clear(r.b[0][i], k);
        clear(r.b[1][i], k);
      }
    }
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      f32x16 s = dot64<WIDE, FB, FA>(join(r.b[t][0], r.b[t][1]), join(r.a[0], r.a[1]), f32x16{});
      s = dot64<WIDE, FB, FA>(join(r.b[t][2], r.b[t][3]), join(r.a[2], r.a[3]), s);
      const float f = r.fa * r.fb[t];
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        if constexpr (SQUARE)
          acc[t][i] = __builtin_fmaf(s[i], f, acc[t][i]);
        else
          acc[t][i] = __builtin_fmaf(s[i], r.fa * __shfl(r.fb[t], (i / 4) * 8 + h * 4 + i % 4, 64), acc[t][i]);
      }
    }
  };
  Block one, two;
  int j = j0 + wave;
  if (j < j1) load(j, one);
  while (j < j1) {
    if (j + 4 < j1) load(j + 4, two);
    multiply(j, one);
    j += 4;
    if (j >= j1) break;
    if (j + 4 < j1) load(j + 4, one);
    multiply(j, two);
    j += 4;
  }
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int i = 0; i < 16; ++i) sums[wave][l][t * 32 + (i / 4) * 8 + h * 4 + i % 4] = acc[t][i];
  __syncthreads();
  const bool whole = gridDim.y == 1;
  void* c = whole ? p.c : p.part + int64_t(blockIdx.y) * p.M * p.N;
  const bool bf16 = whole && p.out_bf16;
  const int64_t n = n0 + (tid & 63);
  if (n >= p.N) return;
  for (int r = tid >> 6; r < p.M; r += 4) {
    const int i = tid & 63;
    const float s = (sums[0][r][i] + sums[1][r][i]) + (sums[2][r][i] + sums[3][r][i]);
    if (bf16)
      GBf16::store1(c, int64_t(r) * p.N + n, s);
    else
      GF32::store1(c, int64_t(r) * p.N + n, s);
  }
}

template <bool WIDE, int FA, int FB, bool SQUARE>
hipError_t launch_square(const MatmulParams& p, const MatmulPlan& plan, hipStream_t stream) {
  const dim3 grid(unsigned(int64_t(p.tiles_m) * p.tiles_n), unsigned(plan.splits));
  if (plan.kind == 0)
    k_few_rows<WIDE, FA, FB, SQUARE><<<grid, 256, 0, stream>>>(p);
  else if (plan.kind == 1)
    k_tiles<WIDE, FA, FB, SQUARE, 2, 2, 2, 2><<<grid, 256, 0, stream>>>(p);
  else
    k_tiles<WIDE, FA, FB, SQUARE, 4, 2, 2, 4><<<grid, 512, 0, stream>>>(p);
  return hipGetLastError();
}

}  // namespace

template <int FA, int FB>
hipError_t launch_matmul_formats(const MatmulArgs& a, const MatmulParams& p, const MatmulPlan& plan) {
  if (a.out == DType::kBf16)
    return p.rb ? launch_square<false, FA, FB, true>(p, plan, a.stream) : launch_square<false, FA, FB, false>(p, plan, a.stream);
  return p.rb ? launch_square<true, FA, FB, true>(p, plan, a.stream) : launch_square<true, FA, FB, false>(p, plan, a.stream);
}

}  // namespace aal
