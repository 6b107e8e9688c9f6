// Host plan of the packed products with packed tokens (mx4.hip): which tile, and how many ranges
// of its sum. A function of the sizes alone, and of the tokens by blocks of 64.
#pragma once

#include "common.h"

namespace optima {

// Tiles of outputs: 256 x 256 with eight waves, and 128 x 128, 64 x 128 and 64 x 64 (tokens x
// outputs) with four.
enum Mx4Tile { kMx4Tile256, kMx4Tile128, kMx4Tile64x128, kMx4Tile64, kMx4Tiles };
constexpr int kMx4TileM[kMx4Tiles] = {256, 128, 64, 64}, kMx4TileN[kMx4Tiles] = {256, 128, 128, 64};

constexpr int64_t kMx4PartBytes = int64_t(64) << 20;  // of split sums, at most

struct Mx4Plan {
  int tile, splits;
  int64_t tiles;
};

inline int64_t mx4_tiles(int tile, int64_t n_tok, int64_t d_out) {
  return ceil_div(n_tok, kMx4TileM[tile]) * ceil_div(d_out, kMx4TileN[tile]);
}
inline int64_t mx4_part_bytes(int tile, int splits, int64_t tiles) {
  return splits < 2 ? 0 : splits * tiles * kMx4TileM[tile] * kMx4TileN[tile] * 4;
}

constexpr int kMx4Splits[] = {1, 2, 3, 4, 6, 8, 12};

// The least estimate, in microseconds: a stage (256 values) of one workgroup alone on its CU, or of
// each of those that share it; what is around the stages; the operands and outputs at 6 TB/s; and
// the join with its parts at 8 TB/s. The constants fit 75 sizes of 17 to 16287 tokens, 64 to 14336
// wide, every tile and split timed with cold weights: the choice is 1.8 % off the best of them on
// average, 19 % at most. 777 tokens, 4097 -> 5001: 128 x 128 27 us, 64 x 128 30, 64 x 64 32,
// 256 x 256 35; 256 tokens, 1000 -> 768: 6.1, 5.0, 4.2, 11.6.
inline Mx4Plan mx4_plan(int64_t n_tok, int64_t d, int64_t d_out) {
  constexpr double kAlone[kMx4Tiles] = {1.31, 0.62, 0.51, 0.33}, kEach[kMx4Tiles] = {1.35, 0.55, 0.39, 0.27};
  constexpr double kAround[kMx4Tiles] = {6.0, 3.7, 3.1, 3.1};
  const int64_t stages = ceil_div(d, 256), pairs = ceil_div(d, 512);
  Mx4Plan best{};
  double best_us = 1e30;
  for (int t = 0; t < kMx4Tiles; ++t) {
    const int64_t tiles = mx4_tiles(t, round_up(n_tok, 64), d_out);
    for (const int splits : kMx4Splits) {
      if (splits > pairs || mx4_part_bytes(t, splits, tiles) > kMx4PartBytes) break;
      const double each = double(std::min(2 * ceil_div(pairs, splits), stages));
      const double us = kAround[t] + each * std::max(kAlone[t], kEach[t] * double(ceil_div(tiles * splits, 256))) +
                        (splits > 1 ? 2.3 + double(mx4_part_bytes(t, splits, tiles)) * 2 / 8e6 : 0);
      if (us < best_us) {
        best_us = us;
        best = Mx4Plan{t, splits, tiles};
      }
    }
  }
  return best;
}

// Room for the parts of any number of tokens up to these.
inline size_t mx4_tile_workspace(int64_t n_tok, int64_t d, int64_t d_out) {
  int64_t most = 0;
  for (int t = 0; t < kMx4Tiles; ++t) {
    const int64_t tiles = mx4_tiles(t, n_tok, d_out);
    for (const int splits : kMx4Splits)
      if (splits <= ceil_div(d, 512)) most = std::max(most, mx4_part_bytes(t, splits, tiles));
  }
  return size_t(std::min(most, kMx4PartBytes));
}

}  // namespace optima
