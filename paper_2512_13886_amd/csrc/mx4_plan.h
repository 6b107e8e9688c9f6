// Host plans of the packed products (mx4.hip): which kernel and tile, and how many ranges of its
// sum. Functions of the sizes alone.
#pragma once

#include "common.h"

namespace optima {

// Tiles of outputs: 256 x 256 with eight waves, and 128 x 128, 64 x 128 and 64 x 64 (tokens x
// outputs) with four.
enum Mx4Tile { kMx4Tile256, kMx4Tile128, kMx4Tile64x128, kMx4Tile64, kMx4Tiles };
constexpr int kMx4TileM[kMx4Tiles] = {256, 128, 64, 64}, kMx4TileN[kMx4Tiles] = {256, 128, 128, 64};

constexpr int64_t kMx4PartBytes = int64_t(64) << 20;  // of split sums, at most

constexpr int kMx4Few = 16;     // tokens of the few-token kernel, at most
constexpr int kMx4Fewest = 8;   // up to which 16-bit ones always take it, and no sum is split: no room

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
// each of those that share it; what is around the stages; and the join with its parts at 10 TB/s.
// (Operands and outputs take the same with every tile.) The constants fit 70 sizes of 17 to 16287
// tokens, 64 to 14336 wide, every tile and split timed with weights from HBM and from the cache: the
// choice is 1.7 % off the best of them on average, 26 % at most. 777 tokens, 4097 -> 5001: 128 x 128
// 27 us, 64 x 128 30, 64 x 64 32, 256 x 256 35; 256 tokens, 1000 -> 768: 6.1, 5.0, 4.0, 11.6.
inline Mx4Plan mx4_plan(int64_t n_tok, int64_t d, int64_t d_out) {
  constexpr double kAlone[kMx4Tiles] = {1.23, 0.60, 0.49, 0.25}, kEach[kMx4Tiles] = {1.24, 0.57, 0.42, 0.25};
  constexpr double kAround[kMx4Tiles] = {7.7, 3.5, 2.8, 2.8};
  const int64_t stages = ceil_div(d, 256), pairs = ceil_div(d, 512);
  Mx4Plan best{};
  double best_us = 1e30;
  for (int t = 0; t < kMx4Tiles; ++t) {
    const int64_t tiles = mx4_tiles(t, round_up(n_tok, 64), d_out);
    for (const int splits : kMx4Splits) {
      if (splits > pairs || mx4_part_bytes(t, splits, tiles) > kMx4PartBytes ||
          (splits > 1 && n_tok <= kMx4Fewest))
        break;
      const double each = double(std::min(2 * ceil_div(pairs, splits), stages));
      const double us = kAround[t] + each * std::max(kAlone[t], kEach[t] * double(ceil_div(tiles * splits, 256))) +
                        (splits > 1 ? 2.6 + double(mx4_part_bytes(t, splits, tiles)) * 2 / 10.2e6 : 0);
      if (us < best_us) {
        best_us = us;
        best = Mx4Plan{t, splits, tiles};
      }
    }
  }
  return best;
}

// Whether packed tokens go in tiles, or by 16 in the few-token kernel. Every 16 or 32 outputs of that one
// read all tokens again. us with it and in tiles: 16 tokens, 4096 -> 4096 5.5 and 9.4, -> 9000 10.8 and 10.1,
// -> 60000 35 and 33; 8 tokens, 8192 -> 28672 33 and 41, 4096 -> 60000 31.4 and 29.8, -> 128000 60 and 55;
// one token, -> 128000 53 and 56.
// Tiles bring scales into LDS by direct loads of 16 bytes, at multiples of 16; the other kernel takes them
// by dwords, so that other scales (of 4 bytes' alignment) go there whatever their number.
inline bool mx4_packed_tiles(int64_t n_tok, int64_t d_out, bool aligned) {
  return aligned && (n_tok > kMx4Few || n_tok * d_out >= (n_tok > 8 ? 100000 : 240000));
}

// The few-token kernel: blocks of 16 outputs that a workgroup takes, and its waves.
struct Mx4FewPlan {
  int blocks, waves;
};
constexpr int kMx4FewWaves = 16;
constexpr int kMx4FewPitch = 512 * 2 + 64;  // bytes of a 16-bit token's 512 values in LDS

// Two blocks halve what is read of the tokens, where that outweighs fewer workgroups than CUs can share
// evenly. us in one and two: 16 tokens, 4096 -> 9000 16.1 and 15.4, d = 1000 -> 1000 5.9 and 6.8; 8 tokens,
// 8192 -> 12288 19.6 and 20.4, -> 17000 28.5 and 27.7; 4 tokens, 4096 -> 12288 9.3 and 10.2, -> 128000 65
// and 60; one token, 8192 -> 10240 13.3 and 15.7, 4096 -> 128000 57 and 63.
// As many waves as there are batches of 512 values, and as the CU's LDS holds tokens for; eight where
// several workgroups of two blocks, or of more than four tokens, can share a CU (8 tokens, 8192 -> 10240
// 22.0 to 18.4 us; but one block of one token, 8192 -> 9000 14.4 in place of 14.0).
inline Mx4FewPlan mx4_few_plan(int64_t n_tok, int64_t d, int64_t d_out, bool packed) {
  const int64_t pairs = ceil_div(d_out, 32), batches = ceil_div(d, 512);
  const bool two = n_tok > 8 ? pairs > 255 : n_tok > 4 ? pairs > 384 : n_tok > 1 && pairs > 2048;
  const int cap = two || (ceil_div(d_out, 16) > 256 && n_tok > 4) ? 8 : kMx4FewWaves;
  const int64_t lds = packed ? cap : 163840 / (n_tok * kMx4FewPitch);
  return {two ? 2 : 1, int(std::min({batches, lds, int64_t(cap)}))};
}
// Of up to kMx4Few 16-bit tokens, in microseconds: rounds of the workgroups that the CUs hold, and the
// batches that a CU takes. The constants fit 84 sizes of 9 to 16 tokens, 4.6 % off on average.
inline double mx4_few_us(int64_t n_tok, int64_t d, int64_t d_out) {
  const Mx4FewPlan p = mx4_few_plan(n_tok, d, d_out, false);
  const int64_t batches = ceil_div(d, 512), each = ceil_div(ceil_div(d_out, 16 * p.blocks), 256);
  const int64_t share = std::min<int64_t>({32 / p.waves, 163840 / (p.waves * n_tok * kMx4FewPitch), 8});
  const double rounds = double(ceil_div(each, std::max<int64_t>(share, 1)));
  return 2.1 + rounds * (1.36 + 0.58 * double(ceil_div(batches, p.waves))) +
         (2.75 + 2.13 / 16 * double(n_tok)) * double(each * batches * p.blocks) / 16;
}

// 16-bit tokens: the few-token kernel (tokens 0), or slabs of 16, 32 or 64 tokens and 256 outputs.
struct Mx4SlabPlan {
  int tokens, splits;
};
constexpr int kMx4SlabRows = 256;
constexpr int kMx4SlabSplits[] = {1, 2, 3, 4, 6, 8, 12, 16, 24};

inline int64_t mx4_slab_parts(int tokens, int splits, int64_t n_tok, int64_t d_out) {
  return splits < 2 ? 0
                    : splits * ceil_div(n_tok, tokens) * ceil_div(d_out, kMx4SlabRows) * tokens * kMx4SlabRows * 4;
}

// The least estimate, in microseconds, as above: batches of 512 values of a slab's workgroup, one a
// CU, 9 TB/s for operands and outputs, and the join. The constants fit 90 sizes of 9 to 64 tokens; the
// choice is 1.7 % off the best on average, between slabs and the few-token kernel 0.2 % of 84 sizes of 9 to 16
// tokens, 5 % at most. 16 tokens, 4096 -> 4096: few 6.8 us, slabs 10.9; -> 128000 118 and 73. 64 tokens,
// 768 -> 14336 8.7 us in slabs of 16, 13.5 in slabs of 64; 4096 -> 14336 23 in slabs of 32, 22.4 of 64.
// More tokens: slabs of 32 where those of 64 leave a round nearly empty (777 tokens, 4097 -> 5001 64 us and
// 87; 128, 1000 -> 5000 9.9 and 13.1; but 1024, 4096 -> 14336 183 and 153).
inline Mx4SlabPlan mx4_slab_plan(int64_t n_tok, int64_t d, int64_t d_out) {
  Mx4SlabPlan best{0, 1};
  if (n_tok <= kMx4Fewest) return best;
  const int64_t batches = ceil_div(d, 512);
  const double bytes = double(d) * double(d_out) * 0.53 + 2.0 * double(n_tok) * double(d + d_out);
  double best_us = 1e30;
  if (n_tok <= kMx4Few) best_us = mx4_few_us(n_tok, d, d_out);
  for (const int tokens : {16, 32, 64}) {
    if (n_tok > 64 ? tokens < (n_tok > 16384 ? 64 : 32) : tokens > 16 && n_tok <= tokens / 2) continue;
    const double around = tokens == 16 ? 2.4 : tokens == 32 ? 3.2 : 4.0;
    const double batch = tokens == 16 ? 2.43 : tokens == 32 ? 2.66 : 3.62;
    const int64_t tiles = ceil_div(n_tok, tokens) * ceil_div(d_out, kMx4SlabRows);
    for (const int splits : kMx4SlabSplits) {
      const int64_t parts = mx4_slab_parts(tokens, splits, n_tok, d_out);
      if (splits > batches || parts > kMx4PartBytes) break;
      const double us = around + batch * double(ceil_div(batches, splits) * ceil_div(tiles * splits, 256)) +
                        bytes / 9e6 + (splits > 1 ? 3.2 + double(parts) * 2 / 5e6 : 0);
      if (us < best_us) {
        best_us = us;
        best = Mx4SlabPlan{tokens, splits};
      }
    }
  }
  return best;
}

// Room for the parts of any number of tokens up to these, of either kind.
inline size_t mx4_room(int64_t n_tok, int64_t d, int64_t d_out) {
  if (n_tok <= kMx4Fewest) return 0;
  int64_t most = 0;
  for (int t = 0; t < kMx4Tiles; ++t)
    for (const int splits : kMx4Splits)
      if (splits <= ceil_div(d, 512))
        most = std::max(most, mx4_part_bytes(t, splits, mx4_tiles(t, n_tok, d_out)));
  for (const int tokens : {16, 32, 64})
    for (const int splits : kMx4SlabSplits)
      if (splits <= ceil_div(d, 512)) most = std::max(most, mx4_slab_parts(tokens, splits, n_tok, d_out));
  return size_t(std::min(most, kMx4PartBytes));
}

}  // namespace optima
