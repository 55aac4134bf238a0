// Which tiles and splits the weight gradient of a linear layer takes.  Host code without a GPU in it, so that a test can ask it.
#pragma once
#include <cstdint>

namespace qa {

constexpr int kWeightStep = 32;                    // rows that a work-group multiplies at a time

// Tiles of 256 x 256 or 128 x 128, and the rows whole or split: whichever is estimated to take the least time.  Measured
// for a step of 32 rows and bfloat16: a 128-tile 0.38 us where it has its compute unit to itself, 0.65 where two share
// one; a 256-tile 0.62 us where few run and 0.9 where all do, which the card's power bounds; times the parts of dY, but
// for 0.1 of the small one's.  A round of work-groups takes 4 us more, and the splits' sums are written and read at
// some 6 TB/s.  (2048 x 2048 columns, 16384 rows: 145 us with four splits of 256-tiles, 322 in one piece, 185 with two of
// 128-tiles; 2048 rows: 40, 48 and 39, and 30 with 128-tiles in one piece.)
struct WeightPlan { int tile; int64_t tiles_n, tiles, splits; };
inline WeightPlan weight_plan(int64_t rows, int64_t cols, int64_t n, int parts) {
  const auto over = [](int64_t a, int64_t b) { return (a + b - 1) / b; };
  WeightPlan best = {};
  double least = 0.0;
  for (int tile = 128; tile <= 256; tile *= 2) {
    if (tile == 256 && n < 8) break;
    const int64_t tiles_n = over(n, tile), tiles = tiles_n * over(cols, tile), at_once = tile == 256 ? 256 : 512;
    for (int64_t splits = 1; splits <= 64 && (splits == 1 || splits * 64 <= rows); ++splits) {
      const int64_t groups = tiles * splits, steps = over(over(rows, splits), kWeightStep);
      const double step = tile == 256 ? parts * (0.6 + 0.3 * (groups < 256 ? (double)groups / 256.0 : 1.0))
                                      : 0.1 + parts * (groups <= 256 ? 0.28 : 0.55);
      const double us = (double)over(groups, at_once) * ((double)steps * step + 4.0) +
                        (splits > 1 ? 4.0 + (double)(2 * splits + 1) * (double)n * (double)cols * (4.0 / 6e6) : 0.0);
      if (least == 0.0 || us < least) {
        least = us;
        best = {tile, tiles_n, tiles, splits};
      }
    }
  }
  return best;
}

}  // namespace qa
