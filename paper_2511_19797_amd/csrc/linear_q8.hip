// The block's linear layers on 8-bit rows (gfx950): y = (xq wq^T) o (xs ws^T) + b, ty = (txq wq^T) o (txs ws^T), with a float32 scale
// for each token row and each output channel (q8.h).  The products are exact: 8-bit integers into 32-bit sums, which K <= 2^16 keeps
// in range; one rounding takes the sum to float32, and one the result to its type.
//
// A 16-byte fragment holds 16 entries of a row where bf16 has 8, and one 32 x 32 x 32 product takes the cycles of a 32 x 32 x 16 one in
// bf16: tiles of 128 bytes x N rows lie in LDS as they do there (Operand, linear_gemm.h, with two entries to its one), and a
// contraction tile is 128 entries.  Computed transposed, D = W-fragment x X-fragment: a lane owns one token and 16 channels of a block.
#include "linear_q8.h"

namespace tvm {
namespace {

__device__ __forceinline__ i32x16 mfma_q8(bf16x8 a, bf16x8 b, i32x16 c) {
  return __builtin_amdgcn_mfma_i32_32x32x32_i8(__builtin_bit_cast(i32x4, a), __builtin_bit_cast(i32x4, b), c, 0, 0, 0);
}
// All waves of the workgroup.  (Not __syncthreads, which waits for every load in flight.)
__device__ __forceinline__ void barrier() { asm volatile("s_barrier" ::: "memory"); }


template <typename T, int N, int NST, int OCC>
__global__ __launch_bounds__(256, OCC) void linear_q8_kernel(LinearQ8Args g) {
  constexpr int W = N / 64;  // blocks of 32 x 32 per wave, either way
  using OP = Operand<false, N>;
  constexpr unsigned HALF = N * 128u, BUF = 2 * HALF;  // a stage: X tile, W tile
  constexpr int LOADS = OP::LOADS, BOTH = 2 * LOADS;
  constexpr unsigned OUT_REGION = 32 * (64 * W + 16);  // per wave, for store_tile_coalesced
  static_assert((NST - 2) * BOTH < 64 && 4 * OUT_REGION <= NST * BUF && NST * BUF * OCC <= 160 * 1024, "stages");
  __shared__ __attribute__((aligned(1024))) char lds[NST * BUF];
  const int nI = (g.R + N - 1) / N, nJ = (g.F + N - 1) / N;
  const int lane = threadIdx.x & 63, ic = lane & 31, hh = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wi = wave & 1, wj = wave >> 1;
  const int it = (int)(blockIdx.x % (unsigned)nI), jt = (int)(blockIdx.x / (unsigned)nI), set = blockIdx.y;
  if (jt >= nJ) return;
  const int i0 = it * N, j0 = jt * N, nct = (g.K + kBKQ - 1) / kBKQ, last = g.K - (nct - 1) * kBKQ;
  const signed char* const x = set == 0 ? g.x[0] : g.x[1];
  const float* const xs = set == 0 ? g.xs[0] : g.xs[1];
  T* const y = static_cast<T*>(set == 0 ? g.y[0] : g.y[1]);
  const unsigned pitchX = (unsigned)g.ldx, pitchW = (unsigned)g.K;
  const int validX = min(g.R - i0, N), validW = min(g.F - j0, N);
  const unsigned lds0 = lds_addr_of(lds);
  OP ox, ow;
  ox.setup(lds0, wi, wave, lane, pitchX);
  ow.setup(lds0 + HALF, wj, wave, lane, pitchW);
  const unsigned cut = lane_chunk(wave, lane) * 16 >= last ? kNowhere : 0u;  // of a row's last tile
  auto issue = [&](int t) {
    const bool end = t >= nct;  // beyond the end: loads that fetch nothing, so that the count of loads in flight stays the same
    const long long c0 = (long long)t * kBKQ;
    const u32x4 sx = descriptor((unsigned long long)(uintptr_t)(x + (long long)i0 * g.ldx + c0),
                                end ? 0u : (unsigned)(validX - 1) * pitchX + (unsigned)(g.K - (int)c0));
    const u32x4 sw = descriptor((unsigned long long)(uintptr_t)(g.w + (long long)j0 * g.K + c0),
                                end ? 0u : (unsigned)(validW - 1) * pitchW + (unsigned)(g.K - (int)c0));
    const unsigned l = lds0 + (unsigned)(t % NST) * BUF + (unsigned)wave * 1024u, c = t == nct - 1 ? cut : 0u;
#pragma unroll
    for (int n = 0; n < LOADS; ++n) load_lds(sx, ox.voff[0] | c, (unsigned)(n * OP::ROWS_STEP) * pitchX, l, n * 4096);
#pragma unroll
    for (int n = 0; n < LOADS; ++n) load_lds(sw, ow.voff[0] | c, (unsigned)(n * OP::ROWS_STEP) * pitchW, l, (int)HALF + n * 4096);
  };
  i32x16 acc[W][W];
#pragma unroll
  for (int a = 0; a < W; ++a)
#pragma unroll
    for (int b = 0; b < W; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[a][b][r] = 0;
  for (int t = 0; t < NST - 1; ++t) issue(t);
  for (int t = 0; t < nct; ++t) {
    dma_wait_keep<(NST - 2) * BOTH>();
    barrier();  // tile t is there for everyone, and everyone is done with tile t - 1: its stage is refilled now
    issue(t + NST - 1);
    const unsigned at = (unsigned)(t % NST) * BUF;
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) {
      bf16x8 xf[W], wf[W];
#pragma unroll
      for (int a = 0; a < W; ++a) xf[a] = ox.frag(a, kk, at);
#pragma unroll
      for (int b = 0; b < W; ++b) wf[b] = ow.frag(b, kk, at);
#pragma unroll
      for (int a = 0; a < W; ++a)
#pragma unroll
        for (int b = 0; b < W; ++b) acc[a][b] = mfma_q8(wf[b], xf[a], acc[a][b]);
    }
  }
  dma_wait();  // the loads past the end land in stages that the results are about to go through
  __syncthreads();
  const int jw = j0 + wj * (W * 32);
  if (jw >= g.F) return;
  const unsigned lw = lds0 + (unsigned)wave * OUT_REGION;
  const bool biased = g.bias != nullptr && set == 0;
#pragma unroll
  for (int a = 0; a < W; ++a) {
    const int i = i0 + (wi * W + a) * 32 + ic;
    const float s = xs[min(i, g.R - 1)];
    f32x16 out[W];
#pragma unroll
    for (int b = 0; b < W; ++b)
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4) {
        const int f = min(jw + b * 32 + 8 * q4 + 4 * hh, g.F - 4);  // (F is a multiple of 8: four channels are in range together)
        const f32x4 ws = four(g.ws + f), bias = biased ? four(static_cast<const T*>(g.bias) + f) : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int e = 0; e < 4; ++e) out[b][4 * q4 + e] = fmaf((float)acc[a][b][4 * q4 + e] * s, ws[e], bias[e]);
      }
    if constexpr (sizeof(T) == 2) {
      store_tile_coalesced<W>(lw, y + jw, g.ldy, i0 + (wi * W + a) * 32, g.R, g.F - jw, out, 1.f, lane);
    } else if (i < g.R) {
#pragma unroll
      for (int b = 0; b < W; ++b)
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4) {
          const int f = jw + b * 32 + 8 * q4 + 4 * hh;
          if (f < g.F)
            *reinterpret_cast<f32x4*>(y + (long long)i * g.ldy + f) = f32x4{out[b][4 * q4], out[b][4 * q4 + 1], out[b][4 * q4 + 2], out[b][4 * q4 + 3]};
        }
    }
  }
}

template <typename T>
hipError_t launch_tiles(int shape, const LinearQ8Args& a, hipStream_t st) {
  const int sets = a.x[1] != nullptr ? 2 : 1;
  const dim3 grid((unsigned)tiles_of(shape, a.R, a.F), sets), block(256);
  if (shape == k128) hipLaunchKernelGGL((linear_q8_kernel<T, 128, 4, 1>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((linear_q8_kernel<T, 64, 4, 2>), grid, block, 0, st, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_linear_q8(const LinearQ8Args& a, int dtype, hipStream_t st) {
  const int sets = a.x[1] != nullptr ? 2 : 1;
  if ((long long)sets * a.R <= kFewRows) return launch_linear_q8_few(a, dtype, st);
  const int shape = pick_shape_q8(sets, a.R, a.F, a.K);
  if (shape == k192) return launch_linear_q8_pipe(a, dtype, st);
  return dtype == 1 ? launch_tiles<bf16>(shape, a, st) : launch_tiles<float>(shape, a, st);
}

}  // namespace tvm
