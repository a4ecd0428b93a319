// Which tile a product of 8-bit codes takes. Plain C++, as CPU tests run it too.
#pragma once

#include <cstdint>

namespace sf {

// Tiles of the 8-bit products; all give the same bits (their sums are exact integers).
enum I8Tile { kI8Deep64, kI8Tile64, kI8Deep128, kI8Tile128, kI8Tile128x192, kI8Tile256x192 };

// What the workgroups of a tile cost that a CU runs side by side (`per` of them), in ns: so
// much per 128-wide slice of K and so much once. `alone` is what a single one takes of
// that, in percent, two or three lie between.
struct I8Cost {
  I8Tile tile;
  int bm, bn, per, slice, once, alone;
};

// Which tile: the one with the least work on its busiest CU. Fitted to launches of 240 shapes
// (1 to 32768 rows, N 64 to 8192, K 128 to 8192, bf16 outputs); the choice takes about 1.01 of the
// fastest tile's time on average, 1.2 in the worst case. Some times (us):
//   * 64 x 64 with four stages, three slices under way, where a CU has one or two of them:
//     64 x 4608 x 1152 4.6, with two stages 4.9, 128 x 128 7.5; 1023 x 777 x 4321 12.5, 15.4
//     and 37. With more per CU the four workgroups that two stages leave room for hide more:
//     4096 x 768 x 768 8.8 and 7.7.
//   * 128 x 128 with four stages, eight wavefronts, one per CU, where one round of it holds
//     everything: 4096 x 768 x 4608 19.9, with two stages 26.8, 64 x 64 23.8; 6000 x 384 x
//     8192 28.1, 40.5 and 38.5.
//   * 128 x 128 in pairs: 2048 x 2048 x 2048 11.7, 64 x 64 16, 128 x 192 15.7.
//   * 128 x 192: 16384 x 4608 x 1152 98, 128 x 128 108; 16384 x 1152 x 4608 83 and 97.
//   * 256 x 192, one per CU, where one round of it holds everything (beyond, pairs of smaller
//     ones hide each other's first loads and outputs): 4096 x 2304 x 768 13.1, 128 x 192 14.2.
// A residual epilogue reads and writes 8 bytes per output more, 1/4 ns of a CU's share of the
// bandwidth: the attention output of four 512^2 rows of width 768 takes 11.1 with 64 x 64 in
// fours, 12.7 with four stages, 14.2 with 128 x 128.
inline I8Tile choose_gemm_i8_tile(long M, long N, long K, bool residual) {
  constexpr I8Cost kTiles[] = {{kI8Deep64, 64, 64, 2, 327, 2626, 44},
                               {kI8Tile64, 64, 64, 4, 738, 3068, 29},
                               {kI8Deep128, 128, 128, 1, 427, 2350, 100},
                               {kI8Tile128, 128, 128, 2, 916, 4165, 54},
                               {kI8Tile128x192, 128, 192, 2, 1204, 6197, 57},
                               {kI8Tile256x192, 256, 192, 1, 915, 6000, 100}};
  const int64_t slices = ((int64_t)K + 127) / 128;
  double least = -1.0;  // the largest sizes pass 64-bit integers
  I8Tile best = kI8Tile128;
  for (const I8Cost& t : kTiles) {
    const int64_t tiles = (((int64_t)M + t.bm - 1) / t.bm) * (((int64_t)N + t.bn - 1) / t.bn);
    const int64_t k = (tiles + 255) / 256;
    if (t.per == 1 && k > 1) continue;
    const int64_t rest = k % t.per;
    const int64_t part = rest ? t.alone + (100 - t.alone) * (rest - 1) / (t.per > 1 ? t.per - 1 : 1) : 0;
    const int64_t once = t.once + (residual ? t.bm * t.bn * t.per / 4 : 0);
    const double cost = (double)(t.slice * slices + once) * ((double)(k / t.per) + 0.01 * (double)part);
    if (least < 0.0 || cost < least) {
      best = t.tile;
      least = cost;
    }
  }
  return best;
}

}  // namespace sf
