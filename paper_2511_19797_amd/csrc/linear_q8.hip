// The block's linear layers on 8-bit rows (gfx950): y = (xq wq^T) o (xs ws^T) + b, ty = (txq wq^T) o (txs ws^T), with a float32 scale
// for each token row and each output channel (q8.h).  The products are exact: 8-bit integers into 32-bit sums, which K <= 2^16 keeps
// in range.  A sum is rounded to float32 (from 2^24 on), times its row's scale, and once more with its channel's scale and the bias (fused);
// a bf16 result is then rounded to its type.
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


// N x N output tiles, one to a workgroup of four waves, for shapes with few of the 256-row tiles.  As in gemm_small_kernel (linear.hip):
// a wave reads the fragments of the next contraction tile between the products of this one, the loads run NST - 2 tiles ahead,
// counted rather than drained, and their descriptors move by additions.  Scales and biases are asked for first of all.
// What bounds them is LDS latency and a barrier per contraction tile, 0.17 us on 64 x 64 where the products take 0.06, behind 3.3 us of
// launch, first loads and results: 2 x 256 x 1152 -> 1152 5.4 us, 64 x 4608 -> 1152 9.3.  (Two groups of waves, each every other contraction
// tile, sums added in the end: 5.8 and 8.4.)  128 x 128: 512 x 1152 -> 4608 10.0.
template <typename T, int N, int NST, int OCC>
__global__ __launch_bounds__(256, OCC) void linear_q8_kernel(LinearQ8Args g, TileOrder order) {
  constexpr int W = N / 64;  // blocks of 32 x 32 per wave, either way
  using OP = Operand<false, N>;
  constexpr unsigned HALF = N * 128u, BUF = 2 * HALF;  // a stage: X tile, W tile
  constexpr int LOADS = 2 * OP::LOADS;                 // wave-loads per wave and contraction tile
  constexpr unsigned OUT_REGION = 32 * (64 * W + 16);  // per wave, for store_tile_coalesced
  static_assert(NST >= 4 && (NST - 2) * LOADS < 64 && 4 * OUT_REGION <= NST * BUF && NST * BUF * OCC <= 160 * 1024, "stages");
  __shared__ __attribute__((aligned(1024))) char lds[NST * BUF];
  const int nI = (g.R + N - 1) / N, nJ = (g.F + N - 1) / N, total = order.sets * nI * nJ;
  // XCD x owns the x-th eighth of the tiles, which run in groups of kGI tile rows, down the group first (linear_pipe.hip)
  const int wg = (int)(blockIdx.x & 7) * ((total + 7) >> 3) + (int)(blockIdx.x >> 3);
  if (wg >= min(total, ((int)(blockIdx.x & 7) + 1) * ((total + 7) >> 3))) return;
  const int lane = threadIdx.x & 63, ic = lane & 31, hh = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wi = wave & 1, wj = wave >> 1;
  const Quotient z = divide((unsigned)wg, order.by_set), grp = divide(z.r, order.by_group);
  const int it_first = (int)grp.q * kGI;
  const Quotient tile = nI - it_first >= kGI ? Quotient{grp.r / kGI, grp.r % kGI} : divide(grp.r, order.by_rest);
  const bool second = z.q != 0;
  const int i0 = (it_first + (int)tile.r) * N, j0 = (int)tile.q * N, jw = j0 + wj * (W * 32);
  const int nct = (g.K + kBKQ - 1) / kBKQ, last = g.K - (nct - 1) * kBKQ;  // contraction tiles, bytes of a row in the last one
  const signed char* const x = second ? g.x[1] : g.x[0];
  const unsigned pitchX = (unsigned)g.ldx, pitchW = (unsigned)g.K;
  const unsigned lds0 = lds_addr_of(lds);
  OP ox, ow;
  ox.setup(lds0, wi, wave, lane, pitchX);
  ow.setup(lds0 + HALF, wj, wave, lane, pitchW);

  // Scales and biases (set 0 only), beyond the edges zeros.  As loaded: anything done to them here would make the compiler wait.
  float xs[W];
  f32x4 ws[W][4];
  Four<T> bias[W][4];
  {
    const __amdgpu_buffer_rsrc_t rx = __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(second ? g.xs[1] : g.xs[0]) + i0, 0,
                                                                        min(g.R - i0, N) * 4, 0x00027000);
    const __amdgpu_buffer_rsrc_t rw = __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(g.ws), 0, g.F * 4, 0x00027000);
    const __amdgpu_buffer_rsrc_t rb = __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(g.bias), 0,
                                                                        g.bias != nullptr && !second ? g.F * (int)sizeof(T) : 0, 0x00027000);
#pragma unroll
    for (int a = 0; a < W; ++a)
      xs[a] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(rx, ((wi * W + a) * 32 + ic) * 4, 0, 0));
#pragma unroll
    for (int b = 0; b < W; ++b)
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4) {
        const int f = jw + b * 32 + 8 * q4 + 4 * hh;
        ws[b][q4] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(rw, f * 4, 0, 0));
        bias[b][q4].load(rb, f);
      }
  }

  // The loads' cursor: descriptors (first byte, size for the bounds check) and lane offsets of contraction tile c_t
  u32x4 sx = descriptor((unsigned long long)(uintptr_t)(x + (long long)i0 * g.ldx), (unsigned)(min(g.R - i0, N) - 1) * pitchX + (unsigned)g.K);
  u32x4 sw = descriptor((unsigned long long)(uintptr_t)(g.w + (long long)j0 * g.K), (unsigned)(min(g.F - j0, N) - 1) * pitchW + (unsigned)g.K);
  const unsigned cut = lane_chunk(wave, lane) * 16 >= last ? kNowhere : 0u;  // of a row's last tile
  unsigned vx = ox.voff[0], vw = ow.voff[0];
  int c_t = 0;
  auto settle = [&]() {
    if (c_t == nct - 1) {
      vx |= cut;
      vw |= cut;
    }
    if (c_t >= nct) sx[2] = sw[2] = 0;  // beyond the end: loads that fetch nothing, so that the count of loads in flight stays the same
  };
  auto move = [&]() {
    ++c_t;
    sx = descriptor(((unsigned long long)sx[1] << 32 | sx[0]) + 128ull, sx[2] - 128u);
    sw = descriptor(((unsigned long long)sw[1] << 32 | sw[0]) + 128ull, sw[2] - 128u);
    settle();
  };
  // wave-load n of the cursor's tile into the stage at `to`
  auto issue = [&](unsigned to, int n) __attribute__((always_inline)) {
    const unsigned l = lds0 + to + (unsigned)wave * 1024u;
    if (n < OP::LOADS) load_lds(sx, vx, (unsigned)(n * OP::ROWS_STEP) * pitchX, l, n * 4096);
    else load_lds(sw, vw, (unsigned)((n - OP::LOADS) * OP::ROWS_STEP) * pitchW, l, (int)HALF + (n - OP::LOADS) * 4096);
  };
  bf16x8 xf[2][4][W], wf[2][4][W];
  auto fetch = [&](int set, int kk, unsigned at) {
#pragma unroll
    for (int a = 0; a < W; ++a) xf[set][kk][a] = ox.frag(a, kk, at);
#pragma unroll
    for (int b = 0; b < W; ++b) wf[set][kk][b] = ow.frag(b, kk, at);
  };
  settle();
#pragma unroll
  for (int n = 0; n < NST - 1; ++n) {
#pragma unroll
    for (int y = 0; y < LOADS; ++y) issue(n * BUF, y);
    move();
  }
  i32x16 acc[W][W];
#pragma unroll
  for (int a = 0; a < W; ++a)
#pragma unroll
    for (int b = 0; b < W; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[a][b][r] = 0;
  dma_wait_keep<(NST - 2) * LOADS>();
  barrier();
#pragma unroll
  for (int kk = 0; kk < 4; ++kk) fetch(0, kk, 0);
  unsigned at = 0;  // tile t's stage
  auto turn = [&](int set) {
    const unsigned next = at + BUF == NST * BUF ? 0 : at + BUF, before = at == 0 ? (NST - 1) * BUF : at - BUF;
    dma_wait_keep<(NST - 3) * LOADS>();
    barrier();  // tile t + 1 is there for everyone, and everyone has tile t - 1 in registers: its stage is refilled now
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) {
      fetch(set ^ 1, kk, next);
#pragma unroll
      for (int n = kk * LOADS / 4; n < (kk + 1) * LOADS / 4; ++n) issue(before, n);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int a = 0; a < W; ++a)
#pragma unroll
        for (int b = 0; b < W; ++b) acc[a][b] = mfma_q8(wf[set][kk][b], xf[set][kk][a], acc[a][b]);
      __builtin_amdgcn_sched_barrier(0);
    }
    move();
    at = next;
  };
  for (int t = 0; t < nct; t += 2) {
    turn(0);
    if (t + 1 < nct) turn(1);
  }
  dma_wait();  // the loads past the end land in stages that the results are about to go through
  __syncthreads();
  if (jw >= g.F) return;
  T* const y = static_cast<T*>(second ? g.y[1] : g.y[0]);
  f32x4 bf[W][4];
#pragma unroll
  for (int b = 0; b < W; ++b)
#pragma unroll
    for (int q4 = 0; q4 < 4; ++q4) bf[b][q4] = bias[b][q4].values();
  const unsigned lw = lds0 + (unsigned)wave * OUT_REGION;
#pragma unroll
  for (int a = 0; a < W; ++a) {
    const int i = i0 + (wi * W + a) * 32 + ic;
    f32x16 out[W];
#pragma unroll
    for (int b = 0; b < W; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r)
        out[b][r] = fmaf((float)acc[a][b][r] * (xs[a] * kRowShift), ws[b][r >> 2][r & 3] * kChannelShift, bf[b][r >> 2][r & 3]);
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
  const dim3 grid((unsigned)small_workgroups(sets * tiles_q8(shape, a.R, a.F))), block(kSmallThreads);
  const TileOrder order = tile_order(shape, sets, a.R, a.F);
  if (shape == kQ128) hipLaunchKernelGGL((linear_q8_kernel<T, 128, 4, 1>), grid, block, 0, st, a, order);
  else hipLaunchKernelGGL((linear_q8_kernel<T, 64, 5, 2>), grid, block, 0, st, a, order);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_linear_q8(const LinearQ8Args& a, int dtype, hipStream_t st) {
  const int sets = a.x[1] != nullptr ? 2 : 1;
  if ((long long)sets * a.R <= kFewRows) return launch_linear_q8_few(a, dtype, st);
  const int shape = pick_shape_q8(sets, a.R, a.F, a.K);
  if (shape <= kQ256x128) return launch_linear_q8_pipe(shape, a, dtype, st);
  return dtype == 1 ? launch_tiles<bf16>(shape, a, st) : launch_tiles<float>(shape, a, st);
}

}  // namespace tvm
