// Tiles and splits of products (csrc/qa_product_plan.h), for tests/test_product_plan.py.
#include "qa_product_plan.h"

extern "C" void product_plan(unsigned allowed, int64_t m, int64_t n, int64_t steps, int64_t count, int lower, double step, int64_t most, int64_t out[2]) {
  const qa::ProductPlan p = qa::product_plan(allowed, qa::ProductShape{m, n, steps, count, lower != 0, step}, most);
  out[0] = p.tiles;
  out[1] = p.splits;
}
