// Which kernel serves a product of the 8-bit linear layers (linear_q8.hip).  Host code only.
#pragma once
#include "linear_plan.h"

namespace tvm {

constexpr int kBKQ = 128;     // contraction entries (bytes) per LDS tile
constexpr int kFewRows = 16;  // x's and tx's rows together that linear_q8_few.hip takes

// Tile shape (k192, k128 or k64) of `sets` products [R][K] x [F][K]: the model of product_ns (linear_plan.h), with contraction tiles
// of 128.  The weights are fits to times of all three shapes at 400 products of R = 9 ... 16384 rows, K = 64 ... 4608 and F = 64 ...
// 6912, one and two sets, bf16 and float32 results; of 500 others the choice is 0.01 % behind the fastest shape on average and
// 3.4 % at most.  Some of the times, back to back (us; 256 x 192 | 128 | 64):
//   64 x 4608 -> 1152:         33 | 21 | 10      few tiles: small ones fill the chip
//   2 x 256 x 1152 -> 1152:    14 | 9.4 | 5.4
//   2 x 642 x 4528 -> 2248:    39 | 26 | 39      one round of 128, two of 64
//   2 x 1000 x 1152 -> 3456:   17 | 19 | 23
//   2 x 4096 x 1152 -> 1152:   19 | 29 | 28
//   2 x 16384 x 1152 -> 3456: 142 | 241 | 288
inline int pick_shape_q8(int sets, int R, int F, int K) {
  constexpr ShapeCost kCost[] = {{-1597, 9137, 859}, {-132, 6103, 413}, {2048, 1277, 185}};
  constexpr int kShape[] = {k192, k128, k64};
  const int steps = (K + kBKQ - 1) / kBKQ;
  int best = k192;
  long long best_ns = product_ns(kCost[0], sets * tiles_of(k192, R, F), steps);
  for (int n = 1; n < 3; ++n) {
    const long long tiles = sets * tiles_of(kShape[n], R, F), ns = product_ns(kCost[n], tiles, steps);
    if (ns < best_ns && grid_fits(kShape[n], tiles)) {
      best = kShape[n];
      best_ns = ns;
    }
  }
  return best;
}

}  // namespace tvm
