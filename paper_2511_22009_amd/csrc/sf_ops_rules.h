// Which tile a product of 8-bit codes takes. Plain C++, as CPU tests run it too.
#pragma once

#include <cstdint>

namespace sf {

// Tiles of the 8-bit products; all give the same bits (their sums are exact integers).
enum I8Tile { kI8Deep64, kI8Tile64, kI8Deep128, kI8Tile128, kI8Tile128x192, kI8Tile192x256, kI8Tile256x256 };

// What the workgroups of a tile cost that a CU runs side by side (`per` of them), in ns: so
// much per 128-wide slice of K and so much once. `alone` is what a single one takes of
// that, in percent, two or three lie between.
struct I8Cost {
  I8Tile tile;
  int bm, bn, per, slice, once, alone;
};

// Which tile: the one with the least work on its busiest CU. Fitted to launches of 260 shapes
// (1 to 32768 rows, N 64 to 8192, K 128 to 8192, bf16 outputs into memory that no cache holds);
// the choice takes about 1.01 of the fastest tile's time on average, 1.15 in the worst case but for
// two of 7 us. Some times (us):
//   * 64 x 64 with four stages, three slices under way, where a CU has one or two of them:
//     64 x 4608 x 1152 4.5, with two stages 4.8, 128 x 128 7.2; 1023 x 777 x 4321 13.7, 19.2
//     and 33. With more per CU the four workgroups that two stages leave room for hide more:
//     1024 x 4608 x 1152 14.0 and 14.8.
//   * 128 x 128 with four stages, eight wavefronts, one per CU, where one round of it holds
//     everything: 2048 x 2048 x 2048 12.9, with two stages 14.9, 64 x 64 16.6.
//   * 128 x 128 in pairs: 1024 x 4608 x 1152 12.0, 64 x 64 14.0.
//   * 128 x 192 in pairs: 16384 x 1152 x 4608 87, 128 x 128 99, 192 x 256 93; 4096 x 4608 x 1152
//     28.5, 31.7 and 30.7.
//   * 192 x 256: 4096 x 2304 x 768 12.7, 128 x 192 15.2, 256 x 256 14.9.
//   * 256 x 256, of large outputs: 16384 x 4608 x 1152 103, 128 x 192 109; 8192^3 440 and 500.
// `heavy`: an epilogue that takes long, so that a CU's other workgroup has to work under it:
// stores from the registers, whose pieces the large tiles write more slowly as well (16384 x 4608 x
// 1152: 192 x 256 132, 256 x 256 163, 128 x 192 124), and GELU (256 x 256 138 to 155, 128 x 192
// 122). The tiles that a CU holds one of are left to a single round then. A residual epilogue
// reads and writes 8 bytes per output more, 1/4 ns of a CU's share of the bandwidth: the
// attention output of four 512^2 rows of width 768 takes 11.1 with 64 x 64 in fours, 12.7 with
// four stages, 14.2 with 128 x 128.
inline I8Tile choose_gemm_i8_tile(long M, long N, long K, bool heavy, bool residual) {
  constexpr I8Cost kTiles[] = {{kI8Deep64, 64, 64, 2, 342, 2430, 46},
                               {kI8Tile64, 64, 64, 4, 805, 3072, 28},
                               {kI8Deep128, 128, 128, 1, 453, 3075, 100},
                               {kI8Tile128, 128, 128, 2, 930, 3697, 61},
                               {kI8Tile128x192, 128, 192, 2, 1267, 5995, 58},
                               {kI8Tile192x256, 192, 256, 1, 1006, 5618, 100},
                               {kI8Tile256x256, 256, 256, 1, 1191, 7780, 100}};
  const int64_t slices = ((int64_t)K + 127) / 128;
  double least = -1.0;  // the largest sizes pass 64-bit integers
  I8Tile best = kI8Tile128;
  for (const I8Cost& t : kTiles) {
    const int64_t tiles = (((int64_t)M + t.bm - 1) / t.bm) * (((int64_t)N + t.bn - 1) / t.bn);
    const int64_t k = (tiles + 255) / 256;
    if (heavy && ((t.per == 1 && k > 1) || t.tile == kI8Tile256x256)) continue;
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
