// Kernels of the product of 8-bit operands (aal_fp8_matmul), by formats:
//
//   c[m, n] = sum_j sa[m, j] sb[n, j] sum_{k in block j} a[m, k] b[n, k]
//
// Rows of b go down the matrix instructions' tiles and rows of a across: a lane holds four
// consecutive columns n of one row m of c, and its row's scale is one value.  A block's 128 values are two
// instructions' worth, whose sum is scaled and added in fp32.
#pragma once

#include "aal_fp8_device.h"
#include "aal_fp8_plan.h"

#include <type_traits>

namespace aal {

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
  int splits;        // parts, none of them empty
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

// A scale as it is stored, and as a float: apart, so that its load is not waited for at once.
__device__ __forceinline__ uint32_t raw_scale(const void* s, int64_t i, int e8m0) {
  return e8m0 ? static_cast<const uint8_t*>(s)[i] : static_cast<const uint32_t*>(s)[i];
}
__device__ __forceinline__ float scale_of(uint32_t raw, int e8m0) {
  const uint32_t e = raw == 0u ? 0x400000u : raw == 255u ? 0x7fc00000u : raw << 23;
  return __builtin_bit_cast(float, e8m0 ? e : raw);
}

// Two scales may leave fp32's range together where the result does not.  Blocks with such scales are looked for and scaled
// in 64 bits, in two to four times a block's time: first whether any scale lies outside of [2^LESS, 2^HIGH], which
// rarely is so, and then what it meets: in range are two of 2^LESS, one of 2^LEAST and one of 2^SMALL, 0, and what lies above
// them up to 2^HIGH.  Looking costs 1% of a product (8,192^3 482 -> 483 us, 64 x 128,256 x 4,096 125 -> 127; 128,256 x 4,096 x 2,048
// into fp32 with any scales 2.55 -> 2.62 ms); once for a whole workgroup, through a flag in LDS, it cost 5%.
template <int HIGH, int SMALL, int LESS, int LEAST>
struct ScaleRange {
  static __device__ __forceinline__ uint32_t power(int e) { return uint32_t(e + 127) << 23; }
  // least and most: of scales' magnitudes (a NaN bears on neither, and ends as one either way)
  static __device__ __forceinline__ bool unusual(float least, float most) {
    return least < __builtin_bit_cast(float, power(LESS)) || most > __builtin_bit_cast(float, power(HIGH));
  }
  // a scale that is a power of two, as it is stored
  static __device__ __forceinline__ bool unusual(uint32_t e8m0) { return e8m0 - uint32_t(LESS + 127) > uint32_t(HIGH - LESS); }
  // bit 0: beyond it whatever the others are, 1: below 2^SMALL, 2: below 2^LESS
  static __device__ __forceinline__ uint32_t bits(float scale) {
    const uint32_t b = __builtin_bit_cast(uint32_t, scale) & 0x7fffffffu;
    auto below = [&](int e) { return b - 1u < power(e) - 1u ? 1u : 0u; };
    return (b > power(HIGH) ? 1u : below(LEAST)) | below(SMALL) << 1 | below(LESS) << 2;
  }
  // of a's scales and of b's, whatever lanes hold them
  static __device__ __forceinline__ bool left(uint32_t a, uint32_t b) {
    auto any = [](uint32_t v) { return __builtin_amdgcn_ballot_w64(v != 0u) != 0; };
    return any((a | b) & 1u) || (any(a & 4u) && any(b & 2u)) || (any(a & 2u) && any(b & 4u));
  }
};
typedef ScaleRange<63, -16, -62, -110> SumRange;   // of scales that sums are multiplied by
typedef ScaleRange<40, -16, -46, -78> ValueRange;  // and values of 2^-16 to 2^16 in bf16, whose products are normal numbers
// Of a product of two scales: 0 is none, since it may be what is left of two others.
__device__ __forceinline__ bool is_normal(float x) {
  return __builtin_amdgcn_classf(x, 0x108);
}
// sum + t x y for scales of any size.
__device__ __forceinline__ float add_far(float sum, float t, float x, float y) {
  return float(__builtin_fma(double(t) * double(x), double(y), double(sum)));
}

// 16 bytes per lane from base + voff (0 from `bytes` on) into LDS, lane l's at `to` + 16 l.  In assembly, since the
// compiler takes every later LDS read for one of these bytes and waits; nothing here has a result
// to wait for but LDS, which stage_barrier() does.  M0 is read one wait state after it is written at the soonest.
__device__ __forceinline__ void load_lds(u32x4 rsrc, uint32_t voff, uint32_t to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(to), "v"(voff), "s"(rsrc) : "m0");
}
// The same for what is read once.
__device__ __forceinline__ void load_lds_once(u32x4 rsrc, uint32_t voff, uint32_t to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen nt lds" ::"s"(to), "v"(voff), "s"(rsrc) : "m0");
}
__device__ __forceinline__ u32x4 buffer_of(const uint8_t* base, uint32_t bytes) {
  const uint64_t b = reinterpret_cast<uint64_t>(base);
  u32x4 r = {uint32_t(b), uint32_t(b >> 32), bytes, 0x00020000u};
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = uint32_t(__builtin_amdgcn_readfirstlane(int(r[i])));
  return r;
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

// Eight consecutive bf16 results of a row, of which n exist.
__device__ __forceinline__ void store8(void* c, int64_t at, u32x4 v, int64_t n) {
  typedef u32x4 u32x4_e2 __attribute__((aligned(2)));
  uint16_t* to = static_cast<uint16_t*>(c) + at;
  if (n >= 8) {
    *reinterpret_cast<u32x4_e2*>(to) = v;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) to[i] = uint16_t(v[i / 2] >> (16 * (i & 1)));
  }
}

// Waits for this wave's loads into LDS and its LDS accesses, then for the workgroup.
__device__ __forceinline__ void stage_barrier() {
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// A stage in LDS has the 128 bytes of each row side by side, the 16-byte piece i of row r at place i ^ r / 2 % 8: they are
// loaded as whole lines, and the 16 lanes that read at a time, rows l of pieces h and h + 1, meet none of the 64 banks
// twice.  A lane multiplies pieces h and h + 4 of its row, which are no neighbours in K, but the same of either operand.
// (Pieces 2 h and 2 h + 1 met four banks twice in every read, a third of LDS's time; an order without any swizzle that
// loads half lines took 5.6 ms for 8,192 x 128,256 x 4,096 instead of 4.4.)
__device__ __forceinline__ int place_in_stage(int row, int byte) {
  return row * 128 + (((byte >> 4) ^ ((row >> 1) & 7)) << 4) + (byte & 15);
}

// ------------------------------------------------------------------ tiles
// A workgroup of WN x WM waves makes 16 TN WN x 16 TM WM results.  Both operands' rows of a block, 128 bytes
// each, are loaded straight into LDS, the next block's while one is being multiplied.
//
// A CU has 64 KB of tiles a stage and two stages of them, so that one tile of 256 x 256 (eight waves) or two of 128 x 128
// (four each) are at work in it.  Bound by how fast stages arrive and by LDS: a block of 256 x 256 x 128 takes 3,700 to
// 4,000 cycles, 2,048 of them in the matrix unit; 8,192 x 128,256 x 4,096 4.2 ms, 2.0 PFLOP/s; 4.9 where
// both operands have a scale for each row, whose tiles of 256 x 256 spill 12 registers.  WIDE has half the
// matrix unit's rate, and 1.04 PFLOP/s at 8,192^3.  The library's products there: with one scale for all 2.6 to 3.2, bf16 1.3.
//
// POW (with WIDE, scales that are powers of two): the widening to bf16 applies them, which is exact, and sums stay in the
// matrix unit from block to block: no arithmetic on sums, a third of the instructions.  128,256 x 4,096 x 2,048 into fp32 2.37
// ms, with the scales applied to sums 2.66; 256 x 256 tiles, whose registers do not do, 3.11.
template <bool WIDE, bool POW, int FA, int FB, bool SQUARE, int TN, int TM, int WN, int WM>
__global__ __launch_bounds__(64 * WN * WM, 2) void k_tiles(MatmulParams p) {
  static_assert(WIDE || !POW, "products of 8-bit instructions take scales on their sums");
  constexpr int NT = 64 * WN * WM, BN = 16 * TN * WN, BM = 16 * TM * WM, RP = NT / 8;  // RP: rows of a round of loads
  static_assert(BN + BM == NT, "one scale per thread");
  static_assert(!SQUARE || 128 % (16 * TN) == 0, "a wave's columns have one scale");
  __shared__ __attribute__((aligned(16))) uint8_t tile[2][(BN + BM) * 128];
  __shared__ __attribute__((aligned(16))) float scales[2][BN + BM];
  __shared__ __attribute__((aligned(4))) uint8_t unusual[2][POW ? WN * WM : 1];  // a wave's scales of a stage are
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l = lane & 15, h = lane >> 4;
  // A tile of c, and the blocks of a part of K.  Workgroups go round over the 8 XCDs: each XCD takes a stretch of
  // tiles of its own, in which groups of 8 tiles down run through all of those across, so that its L2 serves
  // both operands' panels.
  struct Place {
    int down, across, split, j0, j1;
  };
  struct Sources {
    u32x4 ra, rb;
    int64_t scale;
  };
  const int tiles = p.tiles_m * p.tiles_n, total = tiles * p.splits;
  // a thread has one scale: of the first BN threads one of b's rows, of the others one of a's
  const bool is_b = wave < BN / 64;
  const void* scale_base = is_b ? p.sb : p.sa;
  const int64_t scale_step = is_b ? p.sb_block : p.sa_block;
  auto place_of = [&](int id) {
    const int x = id & 7, q = total >> 3, rest = total & 7, seq = x * q + min(x, rest) + (id >> 3);
    const int split = seq / tiles, at = seq - split * tiles;
    const int group = at / (8 * p.tiles_n), first = group * 8, rows = min(8, p.tiles_m - first);
    const int in = at - group * 8 * p.tiles_n, across = in / rows, j0 = split * p.per_split;
    return Place{first + in - across * rows, across, split, j0, min(p.blocks, j0 + p.per_split)};
  };
  auto sources_of = [&](const Place& t) {
    const int64_t m0 = int64_t(t.down) * BM, n0 = int64_t(t.across) * BN;
    const int left_m = int(min(int64_t(BM), p.M - m0)), left_n = int(min(int64_t(BN), p.N - n0));
    // rows behind the last one lie outside the buffers and are zeros
    return Sources{buffer_of(p.a + m0 * p.ld_a, uint32_t(left_m) * uint32_t(p.ld_a)),
                   buffer_of(p.b + n0 * p.ld_b, uint32_t(left_n) * uint32_t(p.ld_b)),
                   is_b ? ((n0 + min(tid, left_n - 1)) >> p.rb) * p.sb_row
                        : ((m0 + min(tid - BN, left_m - 1)) >> p.ra) * p.sa_row};
  };
  const int row = tid >> 3, piece = ((tid & 7) ^ ((row >> 1) & 7)) << 4;
  const uint32_t va = uint32_t(row) * uint32_t(p.ld_a) + piece, vb = uint32_t(row) * uint32_t(p.ld_b) + piece;
  const uint32_t lds0 = uint32_t(reinterpret_cast<uintptr_t>((lds_t*)&tile[0][0])) + wave * 1024;
  constexpr int kLoads = (BN + BM) / RP;  // of a stage; the first BN / RP are b's
  auto load = [&](const Sources& t, int j, int to, int i) {
    const uint32_t k = uint32_t(j) * 128u, base = lds0 + uint32_t(to) * ((BN + BM) * 128) + i * RP * 128;
    if (i < BN / RP)
      load_lds(t.rb, vb + (uint32_t(i * RP) * uint32_t(p.ld_b) + k), base);
    else
      load_lds(t.ra, va + (uint32_t(i * RP - BN) * uint32_t(p.ld_a) + k), base);
  };
  uint32_t next = 0;
  auto load_scales = [&](const Sources& t, int j) { next = raw_scale(scale_base, t.scale + j * scale_step, p.e8m0); };
  auto put_scales = [&](int to) {
    const float s = scale_of(next, p.e8m0);
    scales[to][tid] = s;
    if constexpr (POW) {
      const bool any = __builtin_amdgcn_ballot_w64(ValueRange::unusual(next)) != 0;
      if (lane == 0) unusual[to][wave] = any;
    }
  };
  // K ends inside the last block: zeros for what lies behind it
  auto clear_tail = [&](int to) {
    const int rem = p.K & 127;
    for (int r = tid; r < BN + BM; r += NT) {
      for (int b = rem; b < 128;) {
        uint8_t* at = &tile[to][place_in_stage(r, b)];
        if ((b & 15) == 0) {
          *reinterpret_cast<u32x4*>(at) = u32x4{0, 0, 0, 0};
          b += 16;
        } else {
          *at = 0;
          ++b;
        }
      }
    }
  };
  const int wn = wave % WN, wm = wave / WN;
  f32x4 acc[TN][TM];
#pragma unroll
  for (int i = 0; i < TN; ++i)
#pragma unroll
    for (int j = 0; j < TM; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int front = (h ^ (l >> 1)) << 4, back = ((h + 4) ^ (l >> 1)) << 4;
  auto fragment = [&](const uint8_t* at) {
    const u32x4 a = *reinterpret_cast<const u32x4*>(at + front), b = *reinterpret_cast<const u32x4*>(at + back);
    return i32x8{int(a.x), int(a.y), int(a.z), int(a.w), int(b.x), int(b.y), int(b.z), int(b.w)};
  };
  // The blocks of all tiles that the workgroup takes follow each other without a break, and nothing in it drains at the end
  // of one: when the last row of products of a block begins, all of the block is in registers; there the workgroup
  // meets, the next block has arrived, the one after it is sent for into the stage that has become free, and
  // the next block's first fragments are read into the registers of those that have had their last use.
  int load_id = blockIdx.x, load_j, stage = 0;
  Place ahead = place_of(load_id), t = ahead;
  Sources from = sources_of(ahead);
  bool live = true;  // there is a block to load
  load_j = ahead.j0;
  auto advance = [&] {
    if (++load_j < ahead.j1) return;
    load_id += gridDim.x;
    live = load_id < total;
    if (!live) return;
    ahead = place_of(load_id);
    from = sources_of(ahead);
    load_j = ahead.j0;
  };
  // A wave waits for each of its loads to be taken, and all eight waves send theirs at once: the first kFirst in the
  // last row and kSend of them in each of the next block's first ones leave the matrix unit at work, and
  // time to arrive (all eight in the last row: 1,000 of a block's 4,000 cycles; one a row: they come too late).
  constexpr int kFirst = TN == 8 ? 4 : 3, kSend = TN == 8 ? 2 : 3;
  auto send = [&](int to, int first, int count) {
    if (first == 0) load_scales(from, load_j);
#pragma unroll
    for (int i = first; i < first + count && i < kLoads; ++i) load(from, load_j, to, i);
  };
  auto arrived = [&](int at, int j) {
    put_scales(at);
    stage_barrier();
    if ((p.K & 127) && j == p.blocks - 1) {
      clear_tail(at);
      stage_barrier();
    }
  };
  send(0, 0, kLoads);
  arrived(0, t.j0);
  advance();
  if (live) send(1, 0, kLoads);
  bool sending = false;  // a block's loads are under way
  const int at_b = (wn * TN * 16 + l) * 128, at_a = (BN + wm * TM * 16 + l) * 128;
  // POW: half of a block at a time, a 16-byte piece of each row, and the scales of the lane's own rows
  constexpr int SB = SQUARE ? 1 : TN;
  u32x4 pa[TM], pb[TN];
  float sa[TM], sb[SB];
  bool plain = true;
  // POW: whether the stage's scales may be applied to values (four waves' flags are read at a time)
  auto is_plain = [&](int at) {
    static_assert(!POW || WN * WM == 4, "flags of four waves");
    if (__builtin_amdgcn_readfirstlane(*reinterpret_cast<const int*>(unusual[at])) == 0) return true;
    uint32_t of_a = 0, of_b = 0;
    for (int i = lane; i < BN; i += 64) of_b |= ValueRange::bits(scales[at][i]);
    for (int i = lane; i < BM; i += 64) of_a |= ValueRange::bits(scales[at][BN + i]);
    return !ValueRange::left(of_a, of_b);
  };
  auto scale_a = [&](int at, int m) { return plain ? scales[at][BN + (wm * TM + m) * 16 + l] : 1.f; };
  auto scale_b = [&](int at, int n) { return plain ? scales[at][wn * TN * 16 + (SQUARE ? 0 : n * 16 + l)] : 1.f; };
  auto piece_at = [&](const uint8_t* at, int back_half) { return *reinterpret_cast<const u32x4*>(at + (back_half ? back : front)); };
  i32x8 xa[TM], xb[2];
  if constexpr (!POW) {
    xb[0] = fragment(tile[0] + at_b);
    xb[1] = fragment(tile[0] + at_b + 16 * 128);
  }
  f32x4 made[TM], fb{}, fp{};
  float fa[TM];
  auto scales_b = [&](int at, int n) { return *reinterpret_cast<const f32x4*>(&scales[at][(wn * TN + n) * 16 + h * 4]); };
  if constexpr (!SQUARE && !POW) fb = scales_b(0, 0);
  if constexpr (POW) {
    plain = is_plain(0);
#pragma unroll
    for (int m = 0; m < TM; ++m) {
      sa[m] = scale_a(0, m);
      pa[m] = piece_at(tile[0] + at_a + m * 16 * 128, 0);
    }
#pragma unroll
    for (int n = 0; n < TN; ++n) {
      if (n < SB) sb[n] = scale_b(0, n);
      pb[n] = piece_at(tile[0] + at_b + n * 16 * 128, 0);
    }
  }
#pragma unroll
  for (int m = 0; m < TM; ++m) {
    if constexpr (!POW) xa[m] = fragment(tile[0] + at_a + m * 16 * 128);
    made[m] = f32x4{0.f, 0.f, 0.f, 0.f};
    fa[m] = 0.f;
  }
  auto add = [&](int n, int m, const f32x4& t, float f, const f32x4& g) {
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[n][m][i] = __builtin_fmaf(t[i], SQUARE ? f : f * g[i], acc[n][m][i]);
    // here, not where the compiler would rather have all of them: 128 registers of products
    asm volatile("" : "+v"(acc[n][m]));
  };
  // Whether the wave's scales of the block, of which fa has a's, leave fp32's range (SQUARE: fa has their products).
  auto scales_left = [&] {
    if constexpr (SQUARE) {
      bool any = false;
#pragma unroll
      for (int m = 0; m < TM; ++m) any |= !is_normal(fa[m]);
      return __builtin_amdgcn_ballot_w64(any) != 0;
    } else {
      float own[TN / 4], least = fabsf(fa[0]), most = least;
      auto meet = [&](float f) {
        least = fminf(least, fabsf(f));
        most = fmaxf(most, fabsf(f));
      };
#pragma unroll
      for (int i = 0; i < TN / 4; ++i) meet(own[i] = scales[stage][wn * TN * 16 + i * 64 + lane]);
#pragma unroll
      for (int m = 1; m < TM; ++m) meet(fa[m]);
      if (__builtin_amdgcn_ballot_w64(SumRange::unusual(least, most)) == 0) return false;
      uint32_t of_a = 0, of_b = 0;
#pragma unroll
      for (int i = 0; i < TN / 4; ++i) of_b |= SumRange::bits(own[i]);
#pragma unroll
      for (int m = 0; m < TM; ++m) of_a |= SumRange::bits(fa[m]);
      return SumRange::left(of_a, of_b);
    }
  };
  int id = blockIdx.x;
  for (int j = t.j0;;) {
    const bool last = j + 1 == t.j1;
    const bool more = !last || id + int(gridDim.x) < total;
    Place then = t;
    int next_j = j + 1;
    if (last && more) {
      id += gridDim.x;
      then = place_of(id);
      next_j = then.j0;
    }
    const uint8_t* tb = tile[stage] + at_b;
    const uint8_t* next_b = tile[stage ^ 1] + at_b;
    const uint8_t* next_a = tile[stage ^ 1] + at_a;
    float fn[TM];
    if constexpr (POW) {
      // A quarter of the block at a time, widened; a piece's registers take the next one when it has had its last use.
      const uint8_t* ta = tile[stage] + at_a;
      const bool apply = plain;
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        const int w0 = s % 2 * 2;
        bf16x8 wa[TM];
#pragma unroll
        for (int m = 0; m < TM; ++m) wa[m] = widen<FA>(int(pa[m][w0]), int(pa[m][w0 + 1]), sa[m]);
        if (!apply) {
          // widened as they are: sums times the scales, which are read before another wave may replace them
#pragma unroll
          for (int n = 0; n < TN; ++n) {
            const f32x4 g = SQUARE ? f32x4{1.f, 1.f, 1.f, 1.f} * scales[stage][wn * TN * 16] : scales_b(stage, n);
            const bf16x8 w = widen<FB>(int(pb[n][w0]), int(pb[n][w0 + 1]));
#pragma unroll
            for (int m = 0; m < TM; ++m) {
              const f32x4 u = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, wa[m], f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
              const float f = scales[stage][BN + (wm * TM + m) * 16 + l];
#pragma unroll
              for (int i = 0; i < 4; ++i) acc[n][m][i] = add_far(acc[n][m][i], u[i], f, g[i]);
              asm volatile("" : "+v"(acc[n][m]));
            }
            __builtin_amdgcn_sched_barrier(0);
          }
          // and nothing is left to add to them below, which has no branch
#pragma unroll
          for (int n = 0; n < TN; ++n) pb[n][w0] = pb[n][w0 + 1] = 0u;
#pragma unroll
          for (int m = 0; m < TM; ++m) wa[m] = bf16x8{};
        }
        if (s == 3) {
          if (more) {
            arrived(stage ^ 1, next_j);
            advance();
            sending = live;
          } else {
            sending = false;
          }
          plain = is_plain(stage ^ 1);
        }
        if (s % 2) {
#pragma unroll
          for (int m = 0; m < TM; ++m) {
            pa[m] = piece_at((s == 1 ? ta : next_a) + m * 16 * 128, s == 1);
            if (s == 3) sa[m] = scale_a(stage ^ 1, m);
          }
        }
#pragma unroll
        for (int n = 0; n < TN; ++n) {
          const bf16x8 w = widen<FB>(int(pb[n][w0]), int(pb[n][w0 + 1]), sb[SQUARE ? 0 : n]);
          if (s % 2) pb[n] = piece_at((s == 1 ? tb : next_b) + n * 16 * 128, s == 1);
          if (s == 3 && !SQUARE) sb[n] = scale_b(stage ^ 1, n);
          if (sending && n % (TN / 2) == 0) {
            constexpr int kPart = kLoads / 4;
            const int part = (s == 0 ? 2 : 0) + n / (TN / 2);
            if (s == 3 || s == 0) send(s == 3 ? stage : stage ^ 1, part * kPart, kPart);
          }
#pragma unroll
          for (int m = 0; m < TM; ++m) acc[n][m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, wa[m], acc[n][m], 0, 0, 0);
          __builtin_amdgcn_sched_barrier(0);
        }
        if (s == 3 && SQUARE) sb[0] = scale_b(stage ^ 1, 0);
      }
    } else {
    // each row of products is added while the next one is in the matrix unit
#pragma unroll
    for (int n = 0; n < TN; ++n) {
      const i32x8 x = xb[n & 1];
      const f32x4 g = fb;
      if (n == 0) {
#pragma unroll
        for (int m = 0; m < TM; ++m) {
          fn[m] = scales[stage][BN + (wm * TM + m) * 16 + l];
          if constexpr (SQUARE) fn[m] *= scales[stage][wn * TN * 16];
        }
      }
      if (n + 2 < TN) xb[n & 1] = fragment(tb + (n + 2) * 16 * 128);
      if (n + 1 < TN) {
        if constexpr (!SQUARE) fb = scales_b(stage, n + 1);
      } else {
        if (more) {
          arrived(stage ^ 1, next_j);
          advance();
          sending = live;
        } else {
          sending = false;
        }
        xb[0] = fragment(next_b);
        xb[1] = fragment(next_b + 16 * 128);
        if constexpr (!SQUARE) fb = scales_b(stage ^ 1, 0);
      }
#pragma unroll
      for (int m = 0; m < TM; ++m) {
        const f32x4 u = dot128<WIDE, FB, FA>(x, xa[m]);
        if (m == 1 && sending) {
          if (n + 1 == TN) send(stage, 0, kFirst);
          if (kFirst + n * kSend < kLoads) send(stage ^ 1, kFirst + n * kSend, kSend);
        }
        if (n + 1 == TN) xa[m] = fragment(next_a + m * 16 * 128);
        add(n > 0 ? n - 1 : TN - 1, m, made[m], fa[m], fp);
        made[m] = u;
        if (n == 0) fa[m] = fn[m];
        if constexpr (!WIDE) __builtin_amdgcn_sched_barrier(0);
      }
      fp = g;
      if (n == 0 && scales_left()) {
        // the block's sums are formed and added here, and what follows adds nothing (NaN where values are not finite)
#pragma unroll
        for (int k = 0; k < TN; ++k) {
          const i32x8 y = fragment(tb + k * 16 * 128);
          const f32x4 of_b = SQUARE ? f32x4{1.f, 1.f, 1.f, 1.f} * scales[stage][wn * TN * 16] : scales_b(stage, k);
#pragma unroll
          for (int m = 0; m < TM; ++m) {
            const f32x4 u = dot128<WIDE, FB, FA>(y, xa[m]);
            const float of_a = scales[stage][BN + (wm * TM + m) * 16 + l];
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[k][m][i] = add_far(acc[k][m][i], u[i], of_a, of_b[i]);
            asm volatile("" : "+v"(acc[k][m]));
            __builtin_amdgcn_sched_barrier(0);
          }
        }
#pragma unroll
        for (int m = 0; m < TM; ++m) fa[m] = 0.f;
      }
    }
    }
    stage ^= 1;
    j = next_j;
    if (!last) continue;
    const bool whole = p.splits == 1;
    void* c = whole ? p.c : p.part + t.split * (p.M * p.N);
    const bool bf16 = whole && p.out_bf16;
#pragma unroll
    for (int m = 0; m < TM; ++m) {
      if constexpr (!POW) {
        add(TN - 1, m, made[m], fa[m], fp);
        made[m] = f32x4{0.f, 0.f, 0.f, 0.f};
        fa[m] = 0.f;
      }
      const int64_t gm = int64_t(t.down) * BM + (wm * TM + m) * 16 + l, n0 = int64_t(t.across) * BN + wn * TN * 16;
      if (bf16) {
        // two tiles' columns change places between neighbouring rows of lanes: 8 side by side a lane, 64 bytes of a row of c
#pragma unroll
        for (int n = 0; n < TN; n += 2) {
          const f32x4 &a = acc[n][m], &b = acc[n + 1][m];
          const auto lo = __builtin_amdgcn_permlane16_swap(pack_bf16x2(a[0], a[1]), pack_bf16x2(b[0], b[1]), false, false);
          const auto hi = __builtin_amdgcn_permlane16_swap(pack_bf16x2(a[2], a[3]), pack_bf16x2(b[2], b[3]), false, false);
          const int64_t gn = n0 + (n + (h & 1)) * 16 + (h >> 1) * 8;
          if (gm < p.M && gn < p.N) store8(c, gm * p.N + gn, u32x4{lo[0], hi[0], lo[1], hi[1]}, p.N - gn);
        }
      } else if (gm < p.M) {
#pragma unroll
        for (int n = 0; n < TN; ++n) {
          const int64_t gn = n0 + n * 16 + h * 4;
          if (gn < p.N) store4(c, gm * p.N + gn, acc[n][m][0], acc[n][m][1], acc[n][m][2], acc[n][m][3], p.N - gn, false);
        }
      }
#pragma unroll
      for (int n = 0; n < TN; ++n) acc[n][m] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    fp = f32x4{0.f, 0.f, 0.f, 0.f};
    if (!more) return;
    t = then;
  }
}

// --------------------------------------------------------------- few rows
// Up to 16 TM rows of a: b is read once and bounds the time (7 x 128,256 x 4,096 85 us, 6.2 TB/s where a lone read has 7.1).
// A workgroup of four waves takes 128 rows of b and at most kFewBlocks blocks, which run through a ring of kRing stages in
// LDS, two of them on their way while one is being multiplied.  All its scales are in LDS before that, so that the
// loop waits for the stages alone.
constexpr int kRing = 3;

template <int N>
__device__ __forceinline__ void ring_barrier() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

template <bool WIDE, int FA, int FB, bool SQUARE, int TM>
__global__ __launch_bounds__(256, 2) void k_few_rows(MatmulParams p) {
  constexpr int BN = 128, BM = 32, RP = 32, kLoads = (BN + BM) / RP, SN = SQUARE ? 1 : BN;
  static_assert(kRing == 3, "one stage is waited for while another is on its way");
  __shared__ __attribute__((aligned(16))) uint8_t tile[kRing][(BN + BM) * 128];
  __shared__ float scale_m[kFewBlocks][BM];
  __shared__ __attribute__((aligned(16))) float scale_n[kFewBlocks][SN];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l = lane & 15, h = lane >> 4;
  const int64_t n0 = int64_t(blockIdx.x) * BN;
  const int left_n = int(min(int64_t(BN), p.N - n0)), M = int(p.M);
  const int j0 = blockIdx.y * p.per_split, j1 = min(p.blocks, j0 + p.per_split);
  const u32x4 ra = buffer_of(p.a, uint32_t(M) * uint32_t(p.ld_a));
  const u32x4 rb = buffer_of(p.b + n0 * p.ld_b, uint32_t(left_n) * uint32_t(p.ld_b));
  const int row = tid >> 3, piece = ((tid & 7) ^ ((row >> 1) & 7)) << 4;
  const uint32_t va = uint32_t(row) * uint32_t(p.ld_a) + piece, vb = uint32_t(row) * uint32_t(p.ld_b) + piece;
  const uint32_t lds0 = uint32_t(reinterpret_cast<uintptr_t>((lds_t*)&tile[0][0])) + wave * 1024;
  // workgroups start at blocks of their own: rows of one length would have them all at the same memory channels
  const int count = j1 - j0, turn = int(blockIdx.x % uint32_t(count));
  auto block = [&](int i) { return i + turn < count ? j0 + i + turn : j0 + i + turn - count; };
  auto load = [&](int i, int to) {
    const uint32_t k = uint32_t(block(i)) * 128u, base = lds0 + uint32_t(to) * ((BN + BM) * 128);
#pragma unroll
    for (int r = 0; r < BN / RP; ++r) load_lds_once(rb, vb + (uint32_t(r * RP) * uint32_t(p.ld_b) + k), base + r * RP * 128);
    load_lds(ra, va + k, base + BN * 128);
  };
  float least = 1.f, most = 1.f;
  for (int i = tid; i < (j1 - j0) * BM; i += 256) {
    const int j = i / BM, m = min(i % BM, M - 1);
    const float s = scale_of(raw_scale(p.sa, int64_t(m >> p.ra) * p.sa_row + (j0 + j) * p.sa_block, p.e8m0), p.e8m0);
    scale_m[j][i % BM] = s;
    least = fminf(least, fabsf(s));
    most = fmaxf(most, fabsf(s));
  }
  for (int i = tid; i < (j1 - j0) * SN; i += 256) {
    const int j = i / SN, n = min(i % SN, left_n - 1);
    const float s = scale_of(raw_scale(p.sb, ((n0 + n) >> p.rb) * p.sb_row + (j0 + j) * p.sb_block, p.e8m0), p.e8m0);
    scale_n[j][i % SN] = s;
    least = fminf(least, fabsf(s));
    most = fmaxf(most, fabsf(s));
  }
  // for each wave to read in the part of the last stage that it loads itself, later: the two workgroups of a CU take 160 KB to
  // the byte
  const bool unusual = __builtin_amdgcn_ballot_w64(SumRange::unusual(least, most)) != 0;
  if (lane < 4) tile[kRing - 1][lane * 1024 + wave] = unusual;
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  load(0, 0);
  if (count > 1) load(1, 1);
  const int front = (h ^ (l >> 1)) << 4, back = ((h + 4) ^ (l >> 1)) << 4;
  auto fragment = [&](const uint8_t* at) {
    const u32x4 a = *reinterpret_cast<const u32x4*>(at + front), b = *reinterpret_cast<const u32x4*>(at + back);
    return i32x8{int(a.x), int(a.y), int(a.z), int(a.w), int(b.x), int(b.y), int(b.z), int(b.w)};
  };
  f32x4 acc[2][TM];
#pragma unroll
  for (int n = 0; n < 2; ++n)
#pragma unroll
    for (int m = 0; m < TM; ++m) acc[n][m] = f32x4{0.f, 0.f, 0.f, 0.f};
  int at = 0;  // i's stage
  bool plain = true;
  for (int i = 0; i < count; ++i) {
    const int j = block(i);
    if (i + 1 < count)
      ring_barrier<kLoads>();
    else
      ring_barrier<0>();
    if (i == 0) {
      int any = __builtin_amdgcn_readfirstlane(*reinterpret_cast<const int*>(&tile[kRing - 1][wave * 1024]));
      asm volatile("" : "+s"(any)::"memory");  // read before the load below takes its place
      if (any) {
        uint32_t of_a = 0, of_b = 0;
        for (int k = lane; k < count * BM; k += 64) of_a |= SumRange::bits((&scale_m[0][0])[k]);
        for (int k = lane; k < count * SN; k += 64) of_b |= SumRange::bits((&scale_n[0][0])[k]);
        plain = !SumRange::left(of_a, of_b);
      }
    }
    if (i + 2 < count) load(i + 2, at == 0 ? 2 : at - 1);
    uint8_t* stage = tile[at];
    if ((p.K & 127) && j == p.blocks - 1) {
      // K ends inside the block: zeros for what lies behind it
      for (int r = tid; r < BN + BM; r += 256)
        for (int b = p.K & 127; b < 128; ++b) stage[place_in_stage(r, b)] = 0;
      __syncthreads();
    }
    const uint8_t* tb = stage + (wave * 32 + l) * 128;
    const uint8_t* ta = stage + (BN + l) * 128;
    const i32x8 xb[2] = {fragment(tb), fragment(tb + 2048)};
#pragma unroll
    for (int m = 0; m < TM; ++m) {
      const i32x8 xa = fragment(ta + m * 2048);
      const float fa = scale_m[j - j0][m * 16 + l];
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        const f32x4 t = dot128<WIDE, FB, FA>(xb[n], xa);
        f32x4 fb;
        if constexpr (SQUARE)
          fb = f32x4{1.f, 1.f, 1.f, 1.f} * scale_n[j - j0][0];
        else
          fb = *reinterpret_cast<const f32x4*>(&scale_n[j - j0][wave * 32 + n * 16 + h * 4]);
        if (plain) {
#pragma unroll
          for (int i = 0; i < 4; ++i) acc[n][m][i] = __builtin_fmaf(t[i], fa * fb[i], acc[n][m][i]);
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) acc[n][m][i] = add_far(acc[n][m][i], t[i], fa, fb[i]);
        }
      }
    }
    at = at == 2 ? 0 : at + 1;
  }
  const bool whole = gridDim.y == 1;
  void* c = whole ? p.c : p.part + int64_t(blockIdx.y) * p.M * p.N;
  const bool bf16 = whole && p.out_bf16;
#pragma unroll
  for (int m = 0; m < TM; ++m) {
    const int64_t gm = m * 16 + l;
    if (gm >= p.M) continue;
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      const int64_t gn = n0 + wave * 32 + n * 16 + h * 4;
      if (gn < p.N) store4(c, gm * p.N + gn, acc[n][m][0], acc[n][m][1], acc[n][m][2], acc[n][m][3], p.N - gn, bf16);
    }
  }
}

template <bool WIDE, int FA, int FB, bool SQUARE>
hipError_t launch_square(const MatmulParams& p, const MatmulPlan& plan, hipStream_t stream) {
  const unsigned total = unsigned(int64_t(p.tiles_m) * p.tiles_n * p.splits), most = plan.kind == 1 ? 2 * kCus : kCus;
  const dim3 grid(total < most ? total : most), few(unsigned(p.tiles_n), unsigned(p.splits));
  if (plan.kind == 0 && p.M <= 16)
    k_few_rows<WIDE, FA, FB, SQUARE, 1><<<few, 256, 0, stream>>>(p);
  else if (plan.kind == 0)
    k_few_rows<WIDE, FA, FB, SQUARE, 2><<<few, 256, 0, stream>>>(p);
  else if (WIDE && p.e8m0)
    k_tiles<WIDE, WIDE, FA, FB, SQUARE, 4, 4, 2, 2><<<grid, 256, 0, stream>>>(p);
  else if (plan.kind == 1)
    k_tiles<WIDE, false, FA, FB, SQUARE, 4, 4, 2, 2><<<grid, 256, 0, stream>>>(p);
  else if constexpr (!WIDE)
    k_tiles<WIDE, false, FA, FB, SQUARE, 8, 4, 2, 4><<<grid, 512, 0, stream>>>(p);
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
