// How a product of 8-bit operands is cut (aal_fp8_matmul).  Host code alone.
#pragma once

#include <algorithm>
#include <cstdint>

namespace aal {

constexpr unsigned kCus = 256;  // of an MI355X: workgroups of tiles of 256 x 256 that run at once, of 128 x 128 twice as many
constexpr int kFewBlocks = 32;  // of 128 of the inner dimension, that a workgroup takes where rows are few

// Few rows of a, or tiles of 128 or 256 in both directions; the inner
// dimension in `splits` parts, whose sums are joined by a second kernel.
struct MatmulPlan {
  int kind;  // 0: few rows, 1: tiles of 128 x 128, 2: of 256 x 256
  int splits;
};

inline int64_t up(int64_t a, int64_t b) { return (a + b - 1) / b; }

// The cut whose time is estimated to be the least.  Microseconds, measured over 1 to 2,048 rows of 250 to 128,256 columns and
// 512 to 128,256 values: a block of 128 takes a workgroup `step`, less where half the chip's places or fewer are
// taken, a tile `tile` besides; parts are written, read again and joined by another launch.  Against this, a rule by turns
// of the chip alone took 67 us instead of 46 for 256 x 32,000 x 4,096, 65 instead of 42 for 2,048 x 4,096 x 4,096.
struct TileTimes {
  int side, places;
  double step, step_few, tile;
};
constexpr TileTimes kSmall{128, 2 * kCus, 1.3, 1.1, 4.0}, kLarge{256, kCus, 1.75, 1.6, 8.0};
constexpr TileTimes kSmallWide{128, 2 * kCus, 2.0, 1.55, 6.0};

inline MatmulPlan plan_of(int64_t M, int64_t N, int64_t K, bool wide) {
  const int64_t blocks = up(K, 128);
  if (M <= 32) {
    // Few rows of a: b is read once, for which 250 workgroups do (32 x 32,000 x 4,096 24.8 us, in four parts 36.8); of
    // eight blocks at least.  33 rows of 128,256 x 4,096 take 120 us in tiles, up to 32 take 84 to 92 here.
    const int64_t s = std::min<int64_t>(kCus / up(N, 128), blocks / 8);
    return {0, int(std::max<int64_t>(up(blocks, kFewBlocks), std::min<int64_t>(s, 64)))};
  }
  MatmulPlan best{1, 1};
  double least = 1e300;
  auto consider = [&](int kind, const TileTimes& t) {
    const int64_t tiles = up(M, t.side) * up(N, t.side);
    for (int s : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64}) {
      if (s > 1 && (blocks < 4 * s || tiles * s > t.places)) break;
      const double turns = double(up(tiles * s, t.places)), steps = double(up(blocks, s));
      const double join = s > 1 ? 4.0 + double(s) * (0.4 + double(M) * double(N) * (8.0 / 7e6)) : 0.0;
      const double us = turns * (steps * (tiles * s <= t.places / 2 ? t.step_few : t.step) + t.tile) + join;
      if (us < least) {
        least = us;
        best = {kind, s};
      }
    }
  };
  consider(1, wide ? kSmallWide : kSmall);
  // fp32 results need widened operands, for which tiles of 256 x 256 have no registers left (3.1 ms instead of 2.3)
  if (!wide) consider(2, kLarge);
  return best;
}

}  // namespace aal
