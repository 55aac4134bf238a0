// Tiles and splits of the weight gradient (csrc/qa_weight_plan.h), for tests/test_weight_plan.py.
#include "qa_weight_plan.h"

extern "C" void weight_plan(int64_t rows, int64_t cols, int64_t n, int parts, int64_t out[2]) {
  const qa::WeightPlan p = qa::weight_plan(rows, cols, n, parts);
  out[0] = p.tile;
  out[1] = p.splits;
}
