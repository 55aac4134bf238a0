// Which tiles a product takes, and into how many splits its sums go.  Host code without a GPU in it, so that a test can ask it.
#pragma once
#include <cstdint>

namespace qa {

// Tiles of a work-group, in columns and rows; with k shared by two or four lots of its waves.
enum Tiles { kTiles256, kTiles192, kTiles128, kTiles128Two, kTiles64Two, kTiles64Four };
constexpr unsigned tiles_bit(Tiles t) { return 1u << t; }

struct TileForm {
  int side;
  int at_once;                                     // tiles that run at a time
  double alone, full;                              // us per step of three products of 16: where few tiles run, and where all do
  double round;                                    // us per round beside the steps
};
// Measured with products of 1 x 1 to 4096 x 4096 numbers in two parts; a step of a large tile takes longer where all run, which the
// card's power bounds.  (4096 x 4096 A = X X^T: 250 us with tiles of 256, 193 with 192, 234 with 128 shared by two, 257 with 128; 2048 x 8192:
// 395, 242, 124, 153; 1024 x 1024: 59, 37, 19, 20, and 11.5 with 64 shared by two, 9.9 by four.)  What becomes of the sums there is a store: a tile of logits
// takes longer behind its steps, and estimates are low for few steps (2060 rows, 16384 x 1024 in tiles of 256, with their gradient: 164 us, 106 estimated).
constexpr TileForm kTileForms[] = {{256, 256, 0.70, 1.24, 9.0}, {192, 256, 0.38, 0.75, 6.5}, {128, 512, 0.20, 0.71, 4.5},
                                   {128, 256, 0.19, 0.37, 5.0}, {64, 512, 0.11, 0.24, 3.6}, {64, 256, 0.07, 0.115, 4.6}};

struct ProductShape {
  int64_t m, n, steps, count;                      // count: products side by side
  bool lower;                                      // tiles on and below the diagonal only (m = n)
  double step;                                     // time of a step beside one of three products of 16
};
inline double product_us(Tiles form, const ProductShape& S, int64_t splits) {
  const auto over = [](int64_t a, int64_t b) { return (a + b - 1) / b; };
  const TileForm& F = kTileForms[form];
  const int64_t tm = over(S.m, F.side), tn = over(S.n, F.side), tiles = S.count * splits * (S.lower ? tm * (tm + 1) / 2 : tm * tn);
  const int64_t rounds = tiles / F.at_once, rest = tiles % F.at_once;
  const double step = (double)rounds * F.full + (rest ? F.alone + (F.full - F.alone) * (double)rest / F.at_once : 0.0);
  return (double)over(S.steps, splits) * S.step * step + F.round * (double)(rounds + (rest != 0)) +
         (splits > 1 ? 5.0 + (double)(2 * splits + 1) * (double)S.m * (double)S.n * (4.0 / 5e6) : 0.0);       // written, read and joined at 5 TB/s
}

// Products side by side in one launch, whose work-items number less than 2^32 in tiles of any form (64 x 64 by 512 are the most).
inline int64_t most_side_by_side(int64_t m, int64_t n) {
  const int64_t each = (m + 63) / 64 * ((n + 63) / 64) * 512, most = ((int64_t(1) << 32) - 1) / each;
  return most > 1 ? most : 1;
}

struct ProductPlan { Tiles tiles; int64_t splits; };
// What is estimated to take the least time, of the forms in `allowed` and up to `most` splits, each of eight steps at least and none without any.
inline ProductPlan product_plan(unsigned allowed, const ProductShape& S, int64_t most) {
  ProductPlan best = {kTiles256, 0};
  double least = 0.0;
  for (int f = 0; f < (int)(sizeof kTileForms / sizeof *kTileForms); ++f) {
    if (!(allowed >> f & 1)) continue;
    for (int64_t s = 1; s <= most && (s == 1 || s * 8 <= S.steps); ++s) {
      const double us = product_us((Tiles)f, S, s);
      if (best.splits && us >= least) continue;
      least = us;
      best = {(Tiles)f, s};
    }
  }
  const int64_t each = (S.steps + best.splits - 1) / best.splits;
  best.splits = (S.steps + each - 1) / each;
  return best;
}

}  // namespace qa
