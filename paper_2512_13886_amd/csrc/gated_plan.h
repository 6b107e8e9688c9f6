// Host plans of the gated product and its gradient (gated.hip): which kernel, which tiles,
// how many ranges of a sum. Functions of the sizes alone.
#pragma once

#include "common.h"

namespace optima {

constexpr int kFewTokens = 64;
constexpr int64_t kCus = 256;

// Partial sums of at most kPartTiles 128 x 128 tiles.
constexpr int64_t kPartTiles = 512;

// Microseconds that n[0] blocks of c[0] and then n[1] of c[1] each take over the CUs,
// the longer ones first.
inline double grad_makespan(const int64_t (&n)[2], const double (&c)[2], int first) {
  const int64_t n1 = n[first], n2 = n[1 - first];
  const double c1 = c[first], c2 = c[1 - first];
  const int64_t q = n1 / kCus, r = n1 % kCus;
  if (r == 0) return double(q) * c1 + double(ceil_div(n2, kCus)) * c2;
  const int64_t light = kCus - r, room = light * int64_t(c1 / c2);
  if (n2 <= room)
    return std::max(double(q + 1) * c1, double(q) * c1 + double(ceil_div(n2, light)) * c2);
  return double(q + 1) * c1 + double(ceil_div(n2 - room, kCus)) * c2;
}

// Tile side, and the ranges that the sums of dX (0) and dW (1) are split into, by the time
// that both in one launch should take: 1.4 us a stage and 6 around them for a 256 x 256 tile, 0.56
// and 3.5 for a 128 x 128 one, 3 us and 5 TB/s for the join. By the sizes alone, so that an output
// has the same bits whether or not the other one is wanted beside it.
struct GradPlan {
  int side, splits[2];
};
inline GradPlan plan_grad(int64_t n_tok, int64_t d, int64_t ff) {
  // Stages of 64 values of the contraction, of both parts of the operand that has two.
  const int64_t rows[2] = {n_tok, 2 * ff}, stages[2] = {4 * ceil_div(ff, 64), 2 * ceil_div(n_tok, 64)};
  GradPlan best{256, {1, 1}};
  double best_us = 1e30;
  for (const int side : {256, 128}) {
    const double stage = side == 256 ? 1.4 : 0.56, around = side == 256 ? 6 : 3.5;
    const int64_t most = kPartTiles * 16384 / (side * side);
    int64_t tiles[2];
    for (int k = 0; k < 2; ++k) tiles[k] = ceil_div(rows[k], side) * ceil_div(d, side);
    for (const int sx : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32})
      for (const int sw : {1, 2, 3, 4}) {
        const int64_t parts = (sx > 1 ? sx * tiles[0] : 0) + (sw > 1 ? sw * tiles[1] : 0);
        if (parts > most || (sx > 1 && sx > stages[0]) || (sw > 1 && sw > stages[1])) continue;
        const int64_t n[2] = {tiles[0] * sx, tiles[1] * sw};
        const double c[2] = {stage * double(ceil_div(stages[0], sx)) + around,
                             stage * double(ceil_div(stages[1], sw)) + around};
        const double join = parts ? 3 + double(parts) * side * side * 8 / 5e6 : 0;
        const double us = grad_makespan(n, c, c[0] >= c[1] ? 0 : 1) + join;
        if (us < best_us) {
          best_us = us;
          best = GradPlan{side, {sx, sw}};
        }
      }
  }
  return best;
}

// The tiles of the forward product: the first `wide` outputs take 256 tokens x 128
// outputs, the others 128 x 64, with the sum in `splits` ranges where they are all. By what
// the rounds over the CUs should take: 1.4 us a stage and 6 around them for the large tile,
// 0.56 and 3.5 for the small one, 3 us and 5 TB/s for the join. Small tiles after whole
// rounds of large ones take 4 us and 1.3 times that, since one launch ends before the other
// begins, and are worth it from 7 % on: 2048 -> 5632, 1500 tokens 104 us in two rounds, 83
// in one and small tiles; 1984 -> 12529, 700 tokens 115 and 93; but 4096 -> 14336, 2500
// tokens 532 and 547.
struct GatedPlan {
  int64_t wide;
  int splits;
  double us;
};
inline GatedPlan plan_gated(int64_t n_tok, int64_t d, int64_t ff) {
  const int64_t stages = ceil_div(d, 64);
  const double large_us = 1.4 * double(stages) + 6, small_us = 0.56 * double(stages) + 3.5;
  const int64_t rows = ceil_div(n_tok, 256), cols = ceil_div(ff, 128);
  GatedPlan best{ff, 1, double(ceil_div(rows * cols, kCus)) * large_us};
  const int64_t rounds = rows * cols / kCus, whole = rounds * kCus / rows;
  if (rounds && whole < cols) {
    const int64_t rest = ceil_div(n_tok, 128) * ceil_div(ff - 128 * whole, 64);
    const double us = double(rounds) * large_us + 1.3 * double(ceil_div(rest, kCus)) * small_us + 4;
    if (us < 0.93 * best.us) best = GatedPlan{128 * whole, 1, us};
  }
  const int64_t small = ceil_div(n_tok, 128) * ceil_div(ff, 64);
  for (const int splits : {1, 2, 3, 4, 6, 8, 12, 16}) {
    if (splits > stages || (splits > 1 && splits * small > kPartTiles)) break;
    const double range = 0.56 * double(ceil_div(stages, splits)) + 3.5;
    const double us = double(ceil_div(small * splits, kCus)) * range +
                      (splits > 1 ? 3 + double(small) * splits * 131072 / 5e6 : 0);
    if (us < best.us) best = GatedPlan{0, splits, us};
  }
  return best;
}

// Whether the weights are streamed once for all tokens, or tiles take them. Streamed
// they come at 6 TB/s, and every 16 outputs read all tokens again, at 10 TB/s out of
// the caches; with few outputs a CU's workgroups' own way through d is what counts. To tiles
// they come at 5.5 TB/s at most, and rows that do not suit them are copied first. Measured,
// streamed against tiles: 4096 -> 14336, 4 tokens 39 to 42 us, 16 tokens 49 to 43, 64 tokens
// 91 to 45; 1024 -> 8192, 32 tokens 10.7 to 12.2, 64 tokens 15.1 to 13.1; 2048 -> 5632, 32
// tokens 18 to 20, 64 tokens 25 to 20; 4096 -> 2048, 16 tokens 11 to 17, 64 tokens 26 to 17;
// 1001 -> 2731, 64 tokens 13 to 21.
inline bool few_tokens(int64_t n_tok, int64_t d, int64_t ff) {
  if (n_tok > kFewTokens) return false;
  const double weights = 4e-6 * double(d) * double(ff);  // MB
  const int64_t rounds = ceil_div(ff, 16 * kCus);
  const double streamed = std::max(weights / 6 + double(n_tok) * weights / 320,
                                   4 + double(rounds * n_tok * d) / 13000);
  const double tiles = std::max(plan_gated(kFewTokens, d, ff).us, weights / 5.5 + 1);
  return streamed <= tiles + (d % 64 ? 2 * weights / 5 + 4 : 0);
}

}  // namespace optima
