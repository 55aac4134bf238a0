// Products side by side in one launch (csrc/qa_product_plan.h), for tests/test_product_grid.py.
#include "qa_product_plan.h"

extern "C" int64_t most_side_by_side(int64_t m, int64_t n) { return qa::most_side_by_side(m, n); }
// Tiles of a product's launch in the form of the given number.
extern "C" int64_t tiles_of(int form, int64_t m, int64_t n, int64_t count) {
  const int64_t side = qa::kTileForms[form].side;
  return (m + side - 1) / side * ((n + side - 1) / side) * count;
}
