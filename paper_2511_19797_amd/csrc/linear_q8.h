// What the kernels of the 8-bit linear layers (linear_q8.hip, linear_q8_pipe.hip) share.
#pragma once
#include "linear_gemm.h"
#include "linear_q8_plan.h"
#include "q8.h"

namespace tvm {

typedef __attribute__((ext_vector_type(4))) int i32x4;
typedef __attribute__((ext_vector_type(16))) int i32x16;
typedef __attribute__((ext_vector_type(4))) float f32x4;

// Which 16 bytes of an operand row's 128 a lane of the loads fetches (Operand::setup), the same for all its loads.
__device__ __forceinline__ int lane_chunk(int wave, int lane) {
  const int pos = wave * 64 + lane;
  return (pos & 7) ^ ((pos >> 4) & 7);
}

// A result is fma(fl(fl(sum) xs), ws, bias): three roundings in float32, a fourth to bf16.  The sum (below 2^30) times a token's scale may
// leave float32's range where the result does not, so the scales are taken as xs 2^-24 and ws 2^24: the same bits for xs from 2^-102 (below,
// xs 2^-24 is denormal and loses up to five of its bits) to 2^122 (max / 127 is smaller) and for ws below 2^104.
constexpr float kRowShift = 5.9604644775390625e-08f, kChannelShift = 16777216.0f;

// Four consecutive floats or bf16 values: loaded as they are, bounds-checked (zeros beyond), and as floats.
template <typename T>
struct Four {
  typedef __attribute__((ext_vector_type(sizeof(T)))) unsigned Raw;
  Raw raw;
  __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t rs, int at) {
    if constexpr (sizeof(T) == 4) raw = __builtin_amdgcn_raw_buffer_load_b128(rs, at * 4, 0, 0);
    else raw = __builtin_amdgcn_raw_buffer_load_b64(rs, at * 2, 0, 0);
  }
  __device__ __forceinline__ f32x4 values() const {
    if constexpr (sizeof(T) == 4) return __builtin_bit_cast(f32x4, raw);
    else return __builtin_bit_cast(f32x4, u32x4{raw[0] << 16, raw[0] & 0xffff0000u, raw[1] << 16, raw[1] & 0xffff0000u});
  }
};

// The order of the output tiles (linear_gemm.h)
struct TileOrder {
  int sets;
  Divisor by_set, by_group, by_rest;
  bool stream;  // (256-row tiles: how results are stored)
};
inline TileOrder tile_order(int shape, int sets, int R, int F) {
  const long long nI = ((long long)R + kTileRowsQ8[shape] - 1) / kTileRowsQ8[shape], nJ = ((long long)F + kTileColsQ8[shape] - 1) / kTileColsQ8[shape];
  return TileOrder{sets, Divisor::of((unsigned)(nI * nJ)), Divisor::of((unsigned)(kGI * nJ)), Divisor::of(nI % kGI == 0 ? 1u : (unsigned)(nI % kGI)), false};
}

// A handful of rows (linear_q8_few.hip).
hipError_t launch_linear_q8_few(const LinearQ8Args& a, int dtype, hipStream_t st);
// The 256-row tile shapes (linear_q8_pipe.hip).
hipError_t launch_linear_q8_pipe(int shape, const LinearQ8Args& a, int dtype, hipStream_t st);

}  // namespace tvm
