// What the kernels of the 8-bit linear layers (linear_q8.hip, linear_q8_pipe.hip) share.
#pragma once
#include "linear_gemm.h"
#include "q8.h"

namespace tvm {

typedef __attribute__((ext_vector_type(4))) int i32x4;
typedef __attribute__((ext_vector_type(16))) int i32x16;
typedef __attribute__((ext_vector_type(4))) float f32x4;

constexpr int kBKQ = 128;  // contraction entries (bytes) per LDS tile

// Which 16 bytes of an operand row's 128 a lane of the loads fetches (Operand::setup), the same for all its loads.
__device__ __forceinline__ int lane_chunk(int wave, int lane) {
  const int pos = wave * 64 + lane;
  return (pos & 7) ^ ((pos >> 4) & 7);
}

// Four consecutive floats or bf16 values as floats
__device__ __forceinline__ f32x4 four(const float* p) { return *reinterpret_cast<const f32x4*>(p); }
__device__ __forceinline__ f32x4 four(const bf16* p) {
  const bf16x4 v = *reinterpret_cast<const bf16x4*>(p);
  return f32x4{(float)v[0], (float)v[1], (float)v[2], (float)v[3]};
}

// The order of the output tiles (linear_gemm.h)
struct TileOrder {
  int sets;
  Divisor by_set, by_group, by_rest;
};
inline TileOrder tile_order(int shape, int sets, int R, int F) {
  GemmArgs g{};
  g.I = R;
  g.J = F;
  g.set_divisors(shape, false);
  return TileOrder{sets, g.by_set, g.by_group, g.by_rest};
}

// x's and tx's rows together at most kFewRows (linear_q8_few.hip).
constexpr int kFewRows = 16;
hipError_t launch_linear_q8_few(const LinearQ8Args& a, int dtype, hipStream_t st);
// 256 x 192 tiles (linear_q8_pipe.hip).
hipError_t launch_linear_q8_pipe(const LinearQ8Args& a, int dtype, hipStream_t st);

// Tile shape (k192, k128 or k64; linear_plan.h has the model): time in ns of rounds of 256 workgroups, each its contraction tiles of
// 128 and a fixed part, behind a start-up.
inline int pick_shape_q8(int sets, int R, int F, int K) {
  constexpr ShapeCost kCost[] = {{2000, 5000, 1100}, {1000, 3600, 610}, {1000, 700, 200}};
  constexpr int kShape[] = {k192, k128, k64};
  const int steps = (K + kBKQ - 1) / kBKQ;
  int best = k192;
  long long best_ns = -1;
  for (int n = 0; n < 3; ++n) {
    const long long tiles = sets * tiles_of(kShape[n], R, F), ns = product_ns(kCost[n], tiles, steps);
    if ((best_ns < 0 || ns < best_ns) && grid_fits(kShape[n], tiles)) {
      best = kShape[n];
      best_ns = ns;
    }
  }
  return best;
}

}  // namespace tvm
