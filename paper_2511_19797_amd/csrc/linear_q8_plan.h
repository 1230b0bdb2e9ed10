// Which kernel serves a product of the 8-bit linear layers (linear_q8.hip).  Host code only.
#pragma once
#include "linear_plan.h"

namespace tvm {

constexpr int kBKQ = 128;     // contraction entries (bytes) per LDS tile
constexpr int kFewRows = 16;  // x's and tx's rows together that linear_q8_few.hip takes

// Output tiles
enum { kQ256x192, kQ256x128, kQ128, kQ64, kShapesQ8 };
constexpr int kTileRowsQ8[kShapesQ8] = {256, 256, 128, 64}, kTileColsQ8[kShapesQ8] = {192, 128, 128, 64};
inline long long tiles_q8(int n, int R, int F) {
  return ((long long)R + kTileRowsQ8[n] - 1) / kTileRowsQ8[n] * (((long long)F + kTileColsQ8[n] - 1) / kTileColsQ8[n]);
}
// The 256-row shapes are persistent, 256 workgroups at most; the others a workgroup per tile.
inline bool grid_fits_q8(int n, long long tiles) { return n <= kQ256x128 || small_workgroups(tiles) * kSmallThreads < (1ll << 32); }
// Tile shape of `sets` products [R][K] x [F][K]: the model of product_ns (linear_plan.h), with contraction tiles of 128.  The weights are
// fits to times of all four shapes at 1100 products of R = 9 ... 16384 rows, K = 64 ... 4608 and F = 64 ... 6912, one and two sets,
// bf16 and float32 results; the choice is 0.05 % behind the fastest shape on average and 7.7 % at most, and more than 1 % at 14 of them
// (always 64 x 64: 10 % on average, 256 x 192: 106 %).  Some of the times, back to back (us; 256 x 192 | 256 x 128 | 128 | 64):
//   2 x 256 x 1152 -> 1152:    14.0 | 11.1 |  8.9 | 5.7    few tiles: small ones fill the chip
//   512 x 1152 -> 4608:        14.1 | 11.5 |  9.7 | 10.0   one round of 128, two of 64
//   2 x 1000 x 1152 -> 3456:   14.4 | 12.1 | 16.7 | 19.0   216 tiles of 256 x 128, one round of 256 workgroups, against 144 of 192
//   2 x 4096 x 1152 -> 1152:   15.1 | 21.4 | 24.5 | 23.5   288 of them, two rounds, against 192
//   2 x 16384 x 1152 -> 3456:   146 |  151 |  213 |  275
inline int pick_shape_q8(int sets, int R, int F, int K) {
  constexpr ShapeCost kCost[kShapesQ8] = {{-849, 8420, 832}, {488, 5210, 659}, {108, 4680, 503}, {1944, 1210, 193}};
  const int steps = (K + kBKQ - 1) / kBKQ;
  int best = kQ256x192;
  long long best_ns = product_ns(kCost[best], sets * tiles_q8(best, R, F), steps);
  for (int n = best + 1; n < kShapesQ8; ++n) {
    const long long tiles = sets * tiles_q8(n, R, F), ns = product_ns(kCost[n], tiles, steps);
    if (ns < best_ns && grid_fits_q8(n, tiles)) {
      best = n;
      best_ns = ns;
    }
  }
  return best;
}

}  // namespace tvm
