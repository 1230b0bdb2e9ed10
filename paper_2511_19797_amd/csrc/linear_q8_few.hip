// The 8-bit linear layers (linear_q8.hip) for a handful of rows, x and tx together: the modulation vectors of a batch from its time
// embedding, single tokens.  What bounds them is the weight, read once from memory, and the latencies in front of it.
//
// A workgroup takes 16 output channels and all rows; its waves take every NW-th 64 bytes of the contraction, straight from memory
// into fragments (16 rows x 64 bytes of the weight per load: whole 64-byte segments, no LDS), several loads in flight, and add
// their exact integer sums in LDS.  v_mfma_i32_16x16x64_i8, D = W-fragment x X-fragment: a lane ends up with four consecutive
// channels of one row.
// One row, K = 1152, F = 6912: 3.8 us from the caches, 4.7 from memory (8 MB), of which an empty launch is 1.4; on 64 x 64 tiles 5.3.
// K = 4608, F = 1152: 4.7 and 4.6 against 11.1.  Sixteen rows, F = 6912: 4.5 against 5.4.  From 17 rows on the tiles are as fast (32 rows,
// K = 1152: 5.0 against 5.8 here, every workgroup reading all rows).
#include "linear_q8.h"

namespace tvm {
namespace {

__device__ __forceinline__ void store_four(float* p, f32x4 v) { *reinterpret_cast<f32x4*>(p) = v; }
__device__ __forceinline__ void store_four(bf16* p, f32x4 v) {
  *reinterpret_cast<bf16x4*>(p) = bf16x4{(bf16)v[0], (bf16)v[1], (bf16)v[2], (bf16)v[3]};
}

template <typename T, int NW>
__global__ __launch_bounds__(64 * NW) void linear_q8_few_kernel(LinearQ8Args g, int rows) {
  constexpr int U = 5;  // steps of 64 bytes in flight per wave
  __shared__ i32x4 part[NW][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 15, q = lane >> 4, f0 = blockIdx.x * 16;
  const __amdgpu_buffer_rsrc_t rw = __builtin_amdgcn_make_buffer_rsrc(const_cast<signed char*>(g.w) + (long long)f0 * g.K, 0,
                                                                      min(16, g.F - f0) * g.K, 0x00027000);
  const int s = c < rows ? c : 0;  // (lanes past the last row: the first one again, not stored)
  const bool first = s < g.R;
  const int r = first ? s : s - g.R;
  const signed char* const x = (first ? g.x[0] : g.x[1]) + (long long)r * g.ldx;
  // scales and biases (not on the tangent) of what this lane ends up with, asked for first; beyond the edges zeros
  const int f = f0 + 4 * q;
  const float xs = (first ? g.xs[0] : g.xs[1])[r];
  const f32x4 ws = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(
                                                 __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(g.ws), 0, g.F * 4, 0x00027000), f * 4, 0, 0));
  Four<T> bias;
  bias.load(__builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(g.bias), 0, g.bias != nullptr ? g.F * (int)sizeof(T) : 0, 0x00027000),
            first ? f : g.F);
  i32x4 acc = {0, 0, 0, 0};
  const int steps = (g.K + 63) >> 6;
  for (int t0 = wave; t0 < steps; t0 += NW * U) {
    i32x4 w[U], xv[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {  // 16 bytes past the row's end: the weight's are zeros, the other's do not matter
      const int k = (t0 + u * NW) * 64 + q * 16;
      const bool in = k < g.K;
      w[u] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(rw, in ? c * g.K + k : (int)kNowhere, 0, 0));
      xv[u] = *reinterpret_cast<const i32x4*>(x + (in ? k : 0));
    }
    __builtin_amdgcn_sched_barrier(0);  // all loads first
#pragma unroll
    for (int u = 0; u < U; ++u) acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[u], xv[u], acc, 0, 0, 0);
  }
  part[wave][lane] = acc;
  __syncthreads();
  if (wave != 0 || c >= rows || f >= g.F) return;  // (F is a multiple of 8: four channels are in range together)
#pragma unroll
  for (int w = 1; w < NW; ++w) acc += part[w][lane];
  const f32x4 b4 = bias.values();
  f32x4 o;
#pragma unroll
  for (int e = 0; e < 4; ++e) o[e] = fmaf((float)acc[e] * (xs * kRowShift), ws[e] * kChannelShift, b4[e]);
  store_four(static_cast<T*>(first ? g.y[0] : g.y[1]) + (long long)r * g.ldy + f, o);
}

template <typename T>
hipError_t launch(const LinearQ8Args& a, int rows, hipStream_t st) {
  const dim3 grid((unsigned)((a.F + 15) / 16));
  // longer rows to more waves (one row, weight not in a cache, us of 4 | 8 waves: K = 1152, F = 1152 4.7 | 4.6; K = 2048, F = 2048
  // 4.6 | 4.6; K = 4608, F = 1152 6.3 | 5.4; sixteen rows, K = 1152, F = 6912 5.1 | 5.5)
  if (a.K > 2048) hipLaunchKernelGGL((linear_q8_few_kernel<T, 8>), grid, dim3(512), 0, st, a, rows);
  else hipLaunchKernelGGL((linear_q8_few_kernel<T, 4>), grid, dim3(256), 0, st, a, rows);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_linear_q8_few(const LinearQ8Args& a, int dtype, hipStream_t st) {
  const int rows = (a.x[1] != nullptr ? 2 : 1) * a.R;
  return dtype == 1 ? launch<bf16>(a, rows, st) : launch<float>(a, rows, st);
}

}  // namespace tvm
