// Which tiles a product of 8-bit rows takes.  A slice of 128 bytes costs what a slice of 64 bf16 columns does (gemm_q8.hpp), so the estimates are
// those of the bf16 projections (launch_plan.hpp) over half as many slices.
#pragma once
#include "launch_plan.hpp"

namespace pab {

// kernel numbers as in GemmPlan; 32: 32 tokens x 128 features (quantised outputs of few tokens: their tiles are whole blocks of 128)
inline GemmPlan plan_q8(int M, int N, int nk, bool out8) {
  GemmPlan best{0, 0, 0, 0, 0, 1e30, 0};
  if (!out8) {
    plan_tile(64, 2.9, 0.26, 0.25, 0.55, M, N, nk, &best);
    plan_tile(65, 2.95, 0.185, 0.17, 0.55, M, N, nk, &best);
  }
  plan_tile(128, 3.5, 0.55, 0.52, 2.2, M, N, nk, &best);
  if (!out8 || N % 128 == 0) plan_stream(8, M, N, nk, &best);   // tiles moved back to the edge start at whole blocks
  if (!out8) plan_stream(9, M, N, nk, &best);
  return best;
}

}  // namespace pab
