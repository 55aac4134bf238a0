// Which tiles a product of parts takes.  Host code without a GPU in it, so that a test can ask it.
#pragma once
#include <cstdint>

namespace qa {

// Tiles of a work-group, in columns and rows; with k shared by two or four lots of its waves.
enum Tiles { kTiles256, kTiles192, kTiles128, kTiles128Two, kTiles64Two, kTiles64Four };

struct TileForm {
  int side;
  int at_once;                                     // tiles that run at a time
  double alone, full;                              // us per step of 16: where few tiles run, and where all do
  double round;                                    // us per round beside the steps
};
// Measured with products of 1 x 1 to 4096 x 4096 numbers in two parts; a step of a large tile takes longer where all run, which the
// card's power bounds.  (4096 x 4096 A = X X^T: 250 us with tiles of 256, 193 with 192, 234 with 128 shared by two, 257 with 128; 2048 x 8192:
// 395, 242, 124, 153; 1024 x 1024: 59, 37, 19, 20, and 11.5 with 64 shared by two, 9.9 by four.)
constexpr TileForm kTileForms[] = {{256, 256, 0.70, 1.24, 9.0}, {192, 256, 0.38, 0.75, 6.5}, {128, 512, 0.20, 0.71, 4.5},
                                   {128, 256, 0.19, 0.37, 5.0}, {64, 512, 0.11, 0.24, 3.6}, {64, 256, 0.07, 0.115, 4.6}};

// The form out of `allowed` (bits) that is estimated to take the least time for `count` products of m x n over `steps` steps; lower: tiles on and below
// the diagonal only (m = n).
inline Tiles tiles_for(unsigned allowed, int64_t m, int64_t n, int64_t steps, int64_t count, bool lower) {
  int best = -1;
  double least = 0.0;
  for (int f = 0; f < (int)(sizeof kTileForms / sizeof *kTileForms); ++f) {
    if (!(allowed >> f & 1)) continue;
    const TileForm& F = kTileForms[f];
    const int64_t tm = (m + F.side - 1) / F.side, tn = (n + F.side - 1) / F.side, tiles = count * (lower ? tm * (tm + 1) / 2 : tm * tn);
    const int64_t rounds = tiles / F.at_once, rest = tiles % F.at_once;
    const double step = (double)rounds * F.full + (rest ? F.alone + (F.full - F.alone) * (double)rest / F.at_once : 0.0);
    const double us = (double)steps * step + F.round * (double)(rounds + (rest != 0));
    if (best < 0 || us < least) {
      least = us;
      best = f;
    }
  }
  return (Tiles)best;
}

}  // namespace qa
