// Which tile a product of 8-bit codes takes, and how the rows around a block are shared out. Plain C++, as CPU
// tests run it too.
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

// Tiles of the products of e4m3 codes. Outputs that are codes need a tile that holds whole blocks of 128
// outputs, gated: 256 columns of both projections. `exact`: sums in fp32 (outputs in fp32, or codes).
enum F8Tile {
  kF8Few,
  kF8Split32,
  kF8Split32x4,
  kF8Split64,
  kF8Split64x4,
  kF8Deep128,
  kF8Tile128,
  kF8Tile128x256,
  kF8Tile256x256,
  kF8Codes32,
  kF8Codes64
};
constexpr bool f8_has_tile(F8Tile t, bool codes, bool exact) {
  return codes   ? t == kF8Codes32 || t == kF8Codes64
         : t == kF8Few ? true
         : exact ? t == kF8Split32x4 || t == kF8Split64x4 || t == kF8Tile128
                 : t == kF8Split32 || t == kF8Split64 || t == kF8Deep128 || t == kF8Tile128 || t == kF8Tile128x256 ||
                       t == kF8Tile256x256;
}

// What the workgroups of a tile cost that a CU runs side by side (`per` of them, or one alone), in ns: so much per
// 128-wide slice of K and so much once.
struct F8Cost {
  F8Tile tile;
  int bm, bn, per, slice, once, alone_slice, alone_once;
};

struct F8Choice {
  F8Tile tile;
  double cost;  // ns
};
// The tile among `from` to `to` with the least work on its busiest CU.
inline F8Choice cheapest_f8_tile(const F8Cost* from, const F8Cost* to, int64_t M, int64_t N, int64_t K) {
  const int64_t slices = (K + 127) / 128;
  F8Choice best{from->tile, -1.0};
  for (const F8Cost* t = from; t != to; ++t) {
    const int64_t tiles = ((M + t->bm - 1) / t->bm) * ((N + t->bn - 1) / t->bn);
    const int64_t k = (tiles + 255) / 256, rest = k % t->per;
    const double cost = (double)(k / t->per) * ((double)t->slice * (double)slices + t->once) +
                        (rest ? (double)t->alone_slice * (double)slices + t->alone_once : 0.0);
    if (best.cost < 0.0 || cost < best.cost) best = F8Choice{t->tile, cost};
  }
  return best;
}

// The tiles of each kind of output. Costs from launches of one and of two rounds of each tile at K = 1024 and 4096. Some times (us,
// all of one run: launches of one tile in a row on three sets of operands, codes of a bell as wide as e4m3 goes; codes with
// smaller magnitudes cost less power, and large products up to a tenth less time):
//   * 256 x 256, of large outputs: 16384 x 4608 x 1152 122, 128 x 256 134, 128 x 128 in pairs 136; 8192^3 508, 551
//     and 617.
//   * 128 x 128 in pairs where rounds of the large tiles are left half empty: 4100 x 2048 x 2048 in fp32.
//   * 128 x 128 with four stages, eight wavefronts, one per CU, for single rounds of it: 2048 x 2048 x 4096 23, in pairs
//     31, 128 x 256 31; half a round of 16384 x 128 x 4608 24, 64 x 64 25 (its cost is between what a whole and half a round take).
//   * 64 x 64 with K split over two groups of wavefronts for small grids: 1024 x 1024 x 4096 11.8, over four 12.7, 32 x 64
//     13.8; in fp32 517 x 1001 x 4321 over four 16.2, 32 x 64 23.
//   * 32 x 64 with one wavefront to a group, two groups (fp32: four) for the smallest: 512 x 1024 x 4352 10.6, 64 x 64 11.8,
//     128 x 128 19; 300 x 1152 x 1152 5.5 and 6.2; in fp32 100 x 1152 x 4608 11.7 and 14.1, 300 x 1152 x 1152 7.2 and 8.0. With four
//     groups bf16 10.8 and 6.2.
//   * codes: 64 x 256, two workgroups a CU: gated 16384 x 2 x 4608 x 1152 382, 1024 x 2 x 4608 x 1152 34; 128 x 256 with
//     eight wavefronts, one a CU, 400 and 42; 32 x 256 491 and 37. 32 x 256 while a CU gets one or
//     two of them: 300 x 2 x 1152 x 1152 11.1, 64 x 256 14.2; 2048 x 2 x 2048 x 1024 28 and 23.
// Up to 32 rows the weights' bytes count, which more and smaller workgroups fetch sooner: 32 x 3456 x 1152 4.5, 32 x 64 5.4,
// 64 x 64 6.1; but long weights that a tile's stages fetch faster: 32 x 8192 x 8192 26.2 and 15.7 (16 rows 17.7 and 15.4). Of
// 17 rows on each of those workgroups reads as many rows as columns, and a second round of them (fp32: a third) takes longer than
// 32 x 64: 32 x 4608 x 1152 6.4 and 5.4, 32 x 9216 x 1152 8.6 and 5.5 (fp32 3456 columns 4.7 and 6.9, 4608 6.6 and 7.1,
// 9216 8.7 and 7.2).
struct F8Tiles {
  const F8Cost *from, *to;
};
inline F8Tiles f8_tiles_of(bool codes, bool exact) {
  static constexpr F8Cost kTiles[] = {{kF8Split32, 32, 64, 2, 279, 4540, 193, 3740},
                                      {kF8Split64, 64, 64, 1, 242, 3700, 242, 3700},
                                      {kF8Deep128, 128, 128, 1, 540, 4200, 540, 4200},
                                      {kF8Tile128, 128, 128, 2, 1265, 2600, 834, 4000},
                                      {kF8Tile128x256, 128, 256, 1, 1000, 5200, 1000, 5200},
                                      {kF8Tile256x256, 256, 256, 1, 1900, 7300, 1900, 7300}};
  static constexpr F8Cost kExact[] = {{kF8Split32x4, 32, 64, 1, 215, 4800, 215, 4800},
                                      {kF8Split64x4, 64, 64, 1, 311, 4800, 311, 4800},
                                      {kF8Tile128, 128, 128, 2, 1930, 4900, 1165, 5560}};
  static constexpr F8Cost kCodes[] = {{kF8Codes32, 32, 256, 2, 1096, 6570, 776, 4510},
                                      {kF8Codes64, 64, 256, 2, 1891, 7940, 1092, 6700}};
  return codes ? F8Tiles{kCodes, kCodes + 2} : exact ? F8Tiles{kExact, kExact + 3} : F8Tiles{kTiles, kTiles + 6};
}
// N counts columns of the weights (gated: both projections).
inline F8Tile choose_gemm_f8_tile(long M, long N, long K, bool codes, bool exact, bool gated) {
  const bool few = M <= 16 ? (double)N * (double)K <= 4e7
                           : M <= 32 && (double)N * (double)K <= 1.6e7 && N / (gated ? 32 : 16) <= (exact ? 512 : 256);
  if (few && !codes) return kF8Few;
  const F8Tiles t = f8_tiles_of(codes, exact);
  return cheapest_f8_tile(t.from, t.to, M, N, K).tile;
}

// A product whose last round of tiles leaves most CUs idle is cheaper as two, one after the other: the rows, or the columns
// (multiples of 256), that a tile takes in whole rounds or without its last partial column, and the others, each with a tile of its
// own. 16384 x 1152 x 4608, in the run above: 1024 columns in one round of 256 x 256 tiles 83 us, 128 columns in 128 x 128 tiles 24,
// both 103, all of them in 2.25 rounds of 128 x 128 in pairs 123; 4224 x 4096 x 4096 81 and 104. rows, cols: the first part's; M and N where the whole is not to be parted. Products
// below 40 us stay whole (a second launch and its fixed part count there), and those that would gain less than a twelfth.
inline void choose_gemm_f8_parts(long M, long N, long K, bool codes, bool exact, long& rows, long& cols) {
  rows = M;
  cols = N;
  const F8Tiles t = f8_tiles_of(codes, exact);
  const double whole = cheapest_f8_tile(t.from, t.to, M, N, K).cost;
  if (M <= 32 || whole < 40e3) return;
  double least = whole * (11.0 / 12.0);
  for (const F8Cost* c = t.from; c != t.to; ++c) {
    const int64_t tm = ((int64_t)M + c->bm - 1) / c->bm, tn = ((int64_t)N + c->bn - 1) / c->bn, round = 256 * (int64_t)c->per;
    const int64_t full = tm * tn / round * round;
    const int64_t r = full / tn * c->bm, n[2] = {full / tm * c->bn / 256 * 256, (int64_t)N / c->bn * c->bn / 256 * 256};
    if (r > 0 && r < M) {
      const double two = cheapest_f8_tile(t.from, t.to, r, N, K).cost + cheapest_f8_tile(t.from, t.to, M - r, N, K).cost + 2e3;
      if (two < least) {
        least = two;
        rows = (long)r;
        cols = N;
      }
    }
    for (const int64_t first : n)
      if (first > 0 && first < N) {
        const double two = cheapest_f8_tile(t.from, t.to, M, first, K).cost + cheapest_f8_tile(t.from, t.to, M, N - first, K).cost + 2e3;
        if (two < least) {
          least = two;
          rows = M;
          cols = (long)first;
        }
      }
  }
}

// Columns (outputs) and rows of one launch of a product, whose grid holds less than 2^32 threads: longer calls are several.
// Grids this large have tiles of at least 32 outputs to a thread, so 2^36 outputs are 2^31 threads at most.
constexpr int64_t kF8MostColumns = 1 << 23;  // a multiple of 128
inline int64_t f8_most_rows(int64_t N) {
  const int64_t n = N < kF8MostColumns ? N : kF8MostColumns, most = (int64_t{1} << 36) / n / 256 * 256;
  return most < (1 << 23) ? most : 1 << 23;
}

// ---- rows around a block ---------------------------------------------------------------

// A count in parts of at most `most`: call(first, n) for each. In 64 bits, since counts go up to 2^31 - 1 and the
// first one past the last part does not fit 32.
template <typename F>
inline void in_parts(int64_t count, int64_t most, F call) {
  for (int64_t first = 0; first < count; first += most) call(first, count - first < most ? count - first : most);
}

// Pieces of four dims that a lane holds of a row, and wavefronts that share it. A wavefront takes a row where there are many,
// else a workgroup does, whose lanes each wait for less. `whole`: D is a multiple of four.
struct NormTile {
  int pieces, waves;
};
constexpr NormTile choose_norm_tile(int64_t rows, int D) {
  const bool whole = D % 4 == 0, many = whole && rows >= 2048;
  return D <= 256            ? NormTile{1, 1}
         : many && D <= 768  ? NormTile{3, 1}
         : many && D <= 1024 ? NormTile{4, 1}
         : many && D <= 1280 ? NormTile{5, 1}
         : D <= 1024         ? NormTile{1, 4}
         : D <= 2048         ? NormTile{2, 4}
         : whole && D <= 4096 ? NormTile{4, 4}
         : D <= 8192         ? NormTile{2, 16}
                             : NormTile{4, 16};
}
constexpr bool norm_has_tile(NormTile t, bool whole) { return whole || !(t.pieces > 2 && t.waves < 16); }

// Workgroups that take `step` rows at once, about `groups` of them: `span` rows of one sample each, `spans` to a
// sample, and `most` samples in a launch, since a grid holds less than 2^32 threads.
struct NormSpans {
  int span;
  uint32_t spans;
  int64_t most;
};
inline NormSpans norm_spans(int64_t samples, int64_t tokens, int step, int64_t groups) {
  const int64_t all = (samples * tokens + groups * step - 1) / (groups * step), one = (tokens + step - 1) / step;
  const int64_t span = (all < one ? all : one) * step, spans = (tokens + span - 1) / span;
  return NormSpans{(int)span, (uint32_t)spans, spans < (1 << 21) ? (1 << 21) / spans : 1};
}

// Rows of a sample from `start` on go to one workgroup, `span` of them or what is left: the first row past them. And
// the row that is read ahead: `step` rows further, or the last one again. Neither leaves 32 bits, whatever tokens is.
constexpr int span_end(int start, int span, int tokens) { return span < tokens - start ? start + span : tokens; }
constexpr int row_ahead(int token, int step, int end) { return step < end - token ? token + step : end - 1; }

}  // namespace sf
