// The 8-bit linear layers (linear_q8.hip) on 256 x 192 and 256 x 128 output tiles, hand-scheduled like the bf16 ones
// (linear_pipe.hip, whose layout of LDS, fragment reads and loads this is: 128 bytes of a row per contraction tile, here 128 entries).
//
// Four waves, one per SIMD, as 2 x 2, each with 4 x 3 (4 x 2) blocks of 32 x 32 in AGPRs; three X tiles and two W tiles in LDS; the
// fragments of two contraction steps ahead are read between the products, the loads of later tiles in the slots between.
// Results: a lane owns a token and 16 channels of a block.  The token's scale is a register per block row.  A channel's scale and
// bias belong to a register index, so every row of 16 lanes holds the 16 of its half, one per lane, and the arithmetic takes them
// as row broadcasts (a data-parallel-primitive operand): two registers per block instead of 32.  They come by asynchronous loads
// into LDS, asked for when the output tile begins: with loads into registers the compiler waited, at the tile's end, for every
// load in flight.
// us (POP/s) on 256 x 192, bf16 results, on one card (by card the first takes 140 to 165): 2 x 16384 x 1152 -> 3456 146 (1.8), -> 1152 52 (1.7), -> 4608 188 (1.85), 2 x 16384 x 4608 -> 1152
// 145 (2.4), 8192 x 4608 -> 1152 42 (2.1); float32 results, 1152 -> 3456 162; on 128 x 128 tiles 213, 76, 293, 213, 67; 260.  What bounds it is
// power at K = 4608: at 2.4 POP/s the clock is 1.75 GHz with the matrix cores 64 % busy, and changes that save cycles (the barrier's slot,
// the order of fragment reads, of tiles) leave the times as they are.  At K = 1152 the clock is 1.97 GHz and they are 47 % busy: an output
// tile's end is a third of its cycles, 12 k of 30 k, and what hides it costs as much in LDS traffic.  256 x 256 tiles are no faster there (146 against 144 at -> 3456) and lose where they do not divide the layer (167 against 148
// at 4608 -> 1152).  256 x 128 is for shapes whose tiles it deals out better: 2 x 1000 x 1152 -> 3456 12.1 us, 14.4 on 256 x 192.
#include <type_traits>

#include "linear_gemm.h"
#include "linear_q8.h"

namespace tvm {
namespace {

constexpr int kWI = 4;              // 32-row blocks of a wave
constexpr unsigned kXTile = 32768;  // LDS: three X tiles, then two W tiles
constexpr unsigned kScales = 3 * 1024;
// Results whose rows are whole 64-byte pieces of memory are streamed past the L2 (sc1 nt), which then is the operands': us without | with,
// 2 x 16384 x 1152 -> 4608 on buffers that change from call to call 189 | 175, on the same ones 184 | 185, 4619 x 624 -> 5376 31.2 |
// 30.6, float32 2 x 16384 x 1152 -> 3456 166 | 155.  Where pieces of rows share their 64 bytes, every one of them goes to
// memory twice: 2 x 5103 x 192 -> 6408 47 | 114.
constexpr int kStreamed = 18;

__device__ __forceinline__ void mfma_acc_q8(i32x16& acc, bf16x8 a, bf16x8 b) {
  asm volatile("v_mfma_i32_32x32x32_i8 %0, %1, %2, %0" : "+a"(acc) : "v"(a), "v"(b));
}
// Eight results of a block: registers 8 H ... 8 H + 7 of its sums, times the token's scale, times the channels' scales, plus their
// biases.  (Assembly: the compiler would broadcast every channel's scale and bias once and keep them all, in registers it does not
// have.  The eight reads in front are more than the two slots due between a register copy that it may put there and the broadcasts
// that read the copy.)
template <int H>
__device__ __forceinline__ void results(float (&v)[8], const i32x16& t, float xs, float ws, float bias) {
  float u[8];
  asm volatile(
      "v_accvgpr_read_b32 %8, %16\n\t"
      "v_accvgpr_read_b32 %9, %17\n\t"
      "v_accvgpr_read_b32 %10, %18\n\t"
      "v_accvgpr_read_b32 %11, %19\n\t"
      "v_accvgpr_read_b32 %12, %20\n\t"
      "v_accvgpr_read_b32 %13, %21\n\t"
      "v_accvgpr_read_b32 %14, %22\n\t"
      "v_accvgpr_read_b32 %15, %23\n\t"
      "v_cvt_f32_i32 %8, %8\n\t"
      "v_cvt_f32_i32 %9, %9\n\t"
      "v_cvt_f32_i32 %10, %10\n\t"
      "v_cvt_f32_i32 %11, %11\n\t"
      "v_cvt_f32_i32 %12, %12\n\t"
      "v_cvt_f32_i32 %13, %13\n\t"
      "v_cvt_f32_i32 %14, %14\n\t"
      "v_cvt_f32_i32 %15, %15\n\t"
      "v_mov_b32_dpp %0, %26 row_newbcast:%27 row_mask:0xf bank_mask:0xf\n\t"
      "v_mov_b32_dpp %1, %26 row_newbcast:%28 row_mask:0xf bank_mask:0xf\n\t"
      "v_mov_b32_dpp %2, %26 row_newbcast:%29 row_mask:0xf bank_mask:0xf\n\t"
      "v_mov_b32_dpp %3, %26 row_newbcast:%30 row_mask:0xf bank_mask:0xf\n\t"
      "v_mov_b32_dpp %4, %26 row_newbcast:%31 row_mask:0xf bank_mask:0xf\n\t"
      "v_mov_b32_dpp %5, %26 row_newbcast:%32 row_mask:0xf bank_mask:0xf\n\t"
      "v_mov_b32_dpp %6, %26 row_newbcast:%33 row_mask:0xf bank_mask:0xf\n\t"
      "v_mov_b32_dpp %7, %26 row_newbcast:%34 row_mask:0xf bank_mask:0xf\n\t"
      "v_mul_f32 %8, %8, %24\n\t"
      "v_mul_f32 %9, %9, %24\n\t"
      "v_mul_f32 %10, %10, %24\n\t"
      "v_mul_f32 %11, %11, %24\n\t"
      "v_mul_f32 %12, %12, %24\n\t"
      "v_mul_f32 %13, %13, %24\n\t"
      "v_mul_f32 %14, %14, %24\n\t"
      "v_mul_f32 %15, %15, %24\n\t"
      "v_fmac_f32_dpp %0, %25, %8 row_newbcast:%27 row_mask:0xf bank_mask:0xf\n\t"
      "v_fmac_f32_dpp %1, %25, %9 row_newbcast:%28 row_mask:0xf bank_mask:0xf\n\t"
      "v_fmac_f32_dpp %2, %25, %10 row_newbcast:%29 row_mask:0xf bank_mask:0xf\n\t"
      "v_fmac_f32_dpp %3, %25, %11 row_newbcast:%30 row_mask:0xf bank_mask:0xf\n\t"
      "v_fmac_f32_dpp %4, %25, %12 row_newbcast:%31 row_mask:0xf bank_mask:0xf\n\t"
      "v_fmac_f32_dpp %5, %25, %13 row_newbcast:%32 row_mask:0xf bank_mask:0xf\n\t"
      "v_fmac_f32_dpp %6, %25, %14 row_newbcast:%33 row_mask:0xf bank_mask:0xf\n\t"
      "v_fmac_f32_dpp %7, %25, %15 row_newbcast:%34 row_mask:0xf bank_mask:0xf"
      : "=&v"(v[0]), "=&v"(v[1]), "=&v"(v[2]), "=&v"(v[3]), "=&v"(v[4]), "=&v"(v[5]), "=&v"(v[6]), "=&v"(v[7]),
        "=&v"(u[0]), "=&v"(u[1]), "=&v"(u[2]), "=&v"(u[3]), "=&v"(u[4]), "=&v"(u[5]), "=&v"(u[6]), "=&v"(u[7])
      : "a"(t[8 * H + 0]), "a"(t[8 * H + 1]), "a"(t[8 * H + 2]), "a"(t[8 * H + 3]), "a"(t[8 * H + 4]), "a"(t[8 * H + 5]), "a"(t[8 * H + 6]), "a"(t[8 * H + 7]),
        "v"(xs), "v"(ws), "v"(bias), "n"(8 * H + 0), "n"(8 * H + 1), "n"(8 * H + 2), "n"(8 * H + 3), "n"(8 * H + 4), "n"(8 * H + 5), "n"(8 * H + 6), "n"(8 * H + 7));
}

// load_lds (linear_gemm.h) with 4 bytes per lane
__device__ __forceinline__ void load_lds4(u32x4 srd, unsigned voff, unsigned lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"s"(lds), "v"(voff), "s"(srd) : "memory", "m0");
}

template <typename T, int WJ>
__global__ __launch_bounds__(256, 1) void q8_pipe_kernel(LinearQ8Args g, TileOrder order) {
  constexpr int kTI = 256, kTJ = 64 * WJ;
  constexpr unsigned kWTile = kTJ * 128u;
  constexpr bool WIDE = sizeof(T) == 4;        // float32 results
  using OX = Operand<false, kTI>;
  using OW = Operand<false, kTJ>;
  constexpr int NP = kWI * WJ;                 // products per contraction step
  constexpr int NF = kWI + WJ;                 // fragments per contraction step
  constexpr int LX = OX::LOADS, LW = OW::LOADS;
  constexpr int STORES = (WIDE ? 4 : 2) * NP;  // stores of a wave per output tile
  constexpr int SCALES = 3;                    // loads of scales and biases of a wave per output tile
  constexpr int YOUNGER = LX + STORES + SCALES;
  static_assert(YOUNGER < 64, "vmcnt is six bits");
  // (behind the tiles, twice: the scales of an output tile's 256 rows and 192 columns and the columns' biases, 1 KB each)
  __shared__ __attribute__((aligned(1024))) char lds[3 * kXTile + 2 * kWTile + 2 * kScales];
  const int lane = threadIdx.x & 63, ic = lane & 31, hh = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wi = wave & 1, wj = wave >> 1;
  const unsigned lds0 = lds_addr_of(lds), ldsw = lds0 + 3 * kXTile;
  const int nI = (g.R + kTI - 1) / kTI, nJ = (g.F + kTJ - 1) / kTJ;
  const int nct = (g.K + kBKQ - 1) / kBKQ, last = g.K - (nct - 1) * kBKQ;  // contraction tiles, bytes of a row in the last one
  const unsigned pitchX = (unsigned)g.ldx, pitchW = (unsigned)g.K;

  // Persistent workgroups; XCD x owns the x-th eighth of the tiles, which run in groups of kGI tile rows, down the group first
  // (linear_pipe.hip).
  const int total = order.sets * nI * nJ;
  const int per_xcd = (total + 7) >> 3, wg_per_xcd = (int)(gridDim.x >> 3);
  const int id_end = min(total, ((int)(blockIdx.x & 7) + 1) * per_xcd);
  struct Where {
    int i0, j0, set;
  };
  auto locate = [&](int wg) {
    Where c;
    const Quotient z = divide((unsigned)wg, order.by_set), grp = divide(z.r, order.by_group);
    const int it_first = (int)grp.q * kGI;
    const Quotient jt = nI - it_first >= kGI ? Quotient{grp.r / kGI, grp.r % kGI} : divide(grp.r, order.by_rest);
    c.set = (int)z.q;
    c.i0 = (it_first + (int)jt.r) * kTI;
    c.j0 = (int)jt.q * kTJ;
    return c;
  };
  int wg = (int)(blockIdx.x & 7) * per_xcd + (int)(blockIdx.x >> 3);
  if (wg >= id_end) return;

  OX ox;
  OW ow;
  ox.setup(lds0, wi, wave, lane, pitchX);
  ow.setup(ldsw, wj, wave, lane, pitchW);
  const unsigned cut = lane_chunk(wave, lane) * 16 >= last ? kNowhere : 0u;  // of a row's last tile

  // The loads run two contraction tiles ahead of the products, over the ends of output tiles.
  u32x4 srd_x, srd_w;              // descriptors: first byte, size for the bounds check
  unsigned vx, vw;                 // lane offsets
  int c_left, c_wg = wg;           // tiles left of the cursor's output tile
  auto lanes = [&]() {             // lane offsets of the cursor's tile
    const unsigned c = c_left == 1 ? cut : 0u;
    vx = ox.voff[0] | c;
    vw = ow.voff[0] | c;
  };
  auto open = [&](const Where& w) {
    srd_x = descriptor((unsigned long long)(uintptr_t)((w.set == 0 ? g.x[0] : g.x[1]) + (long long)w.i0 * g.ldx),
                       (unsigned)(min(g.R - w.i0, kTI) - 1) * pitchX + (unsigned)g.K);
    srd_w = descriptor((unsigned long long)(uintptr_t)(g.w + (long long)w.j0 * g.K),
                       (unsigned)(min(g.F - w.j0, kTJ) - 1) * pitchW + (unsigned)g.K);
    c_left = nct;
    lanes();
  };
  auto further_x = [&]() { srd_x = descriptor(((unsigned long long)srd_x[1] << 32 | srd_x[0]) + 128ull, srd_x[2] - 128u); };
  auto further_w = [&]() { srd_w = descriptor(((unsigned long long)srd_w[1] << 32 | srd_w[0]) + 128ull, srd_w[2] - 128u); };
  auto advance = [&]() {  // behind further_x, further_w: where the output tile goes on differently, or has ended
    if (--c_left > 0) {
      lanes();
    } else if (c_wg + wg_per_xcd < id_end) {
      c_wg += wg_per_xcd;
      open(locate(c_wg));
    } else {  // nothing more: size 0, loads that fetch nothing, so that the count of loads in flight stays the same
      srd_x = srd_w = descriptor(0, 0);
      c_left = 1;
      c_wg = id_end;
    }
  };
  unsigned slot_x = lds0 + (unsigned)wave * 1024u, slot_w = ldsw + (unsigned)wave * 1024u;  // where the next tile's loads go
  auto issue_x = [&](int n) { load_lds(srd_x, vx, (unsigned)(n * OX::ROWS_STEP) * pitchX, slot_x, n * 4096); };
  auto issue_w = [&](int n) { load_lds(srd_w, vw, (unsigned)(n * OW::ROWS_STEP) * pitchW, slot_w, n * 4096); };

  i32x16 acc[kWI][WJ];
  bf16x8 xf[4][kWI], wf[4][WJ];
  auto fetch = [&](int kk, int f) {  // fragment number f of contraction step kk of the tile at the read addresses
    if (f < WJ) wf[kk][f] = ow.frag(f, kk);
    else xf[kk][f - WJ] = ox.frag(f - WJ, kk);
  };

  // Scales of the output tile's rows and columns, and biases (set 0 only), into half `par` of their place; beyond the edges zeros.
  // Every wave fetches 64 values' worth of each.
  const unsigned ldss = ldsw + 2 * kWTile;
  auto scales_load = [&](const Where& w, unsigned par) {
    const unsigned at = ldss + par * kScales + (unsigned)wave * 256u, v = (unsigned)(wave * 64 + lane) * 4u;
    const int cols = min(g.F - w.j0, kTJ);
    load_lds4(descriptor((unsigned long long)(uintptr_t)((w.set == 0 ? g.xs[0] : g.xs[1]) + w.i0), (unsigned)min(g.R - w.i0, kTI) * 4u), v, at);
    load_lds4(descriptor((unsigned long long)(uintptr_t)(g.ws + w.j0), (unsigned)cols * 4u), v, at + 1024u);
    load_lds4(descriptor((unsigned long long)(uintptr_t)(static_cast<const T*>(g.bias) + w.j0),
                         g.bias != nullptr && w.set == 0 ? (unsigned)(cols * (int)sizeof(T)) : 0u), v, at + 2048u);
  };
  auto start = [&](int a) {  // accumulators of block row a from 0, by a product of zeros
    const bf16x8 zero = __builtin_bit_cast(bf16x8, u32x4{0u, 0u, 0u, 0u});
#pragma unroll
    for (int b = 0; b < WJ; ++b) asm volatile("s_nop 1\n\tv_mfma_i32_32x32x32_i8 %0, %1, %1, 0" : "=a"(acc[a][b]) : "v"(zero));
  };

  // Results of output tile w: [32 rows x 128 bytes] at a time (two blocks of bf16, one of float32; a last single block of bf16:
  // 64 bytes a row) through LDS, so that they leave as whole cache lines.  The place: the X tile that was just worked on is
  // free, and of the slot that the next X tile goes to, the chunks that this wave's own loads will fill are its own: 1 KB every
  // 4 KB.  A chunk holds 8 rows (16 of 64 bytes); 16-byte chunks within them are swizzled, and in rows 16 to 31 the 8-byte
  // halves that the two half-waves write change places, so that no two lanes meet in a bank.
  typedef __attribute__((ext_vector_type(2))) unsigned u32x2;
  auto write_out = [&](const Where& w, unsigned par) {
    typedef u32x2 __attribute__((address_space(3))) * wp2;
    typedef f32x4 __attribute__((address_space(3))) * wp4;
    typedef const u32x4 __attribute__((address_space(3))) * rp;
    const int i_first = w.i0 + wi * (kWI * 32), j_first = w.j0 + wj * (WJ * 32);
    const int rows = max(0, min(g.R - i_first, kWI * 32)), cols = max(0, min(g.F - j_first, WJ * 32));
    constexpr int E = (int)sizeof(T);
    const unsigned pitch = (unsigned)(g.ldy * E);
    char* const base = static_cast<char*>(w.set == 0 ? g.y[0] : g.y[1]) + ((long long)i_first * g.ldy + j_first) * E;
    const int bytes = rows > 0 && cols > 0 ? (int)((unsigned)(rows - 1) * pitch + (unsigned)cols * E) : 0;
    const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(base, 0, bytes, 0x00027000);
    constexpr int WB = WIDE ? 1 : 2;                  // blocks of a piece
    constexpr int NS = (WJ + WB - 1) / WB;            // pieces per block row
    const unsigned at128 = slot_x + (unsigned)(ic >> 3) * 4096u + (unsigned)(ic & 7) * 128u, sw128 = (unsigned)(ic >> 1) & 7u;
    const unsigned at64 = slot_x + (unsigned)(ic >> 4) * 4096u + (unsigned)(ic & 15) * 64u, sw64 = (unsigned)(ic >> 2) & 3u;
    const unsigned half = (unsigned)(hh ^ (ic >> 4)) * 8u;
    // read side: lane -> row r8 of 8 (16), chunk
    const unsigned rd128 = slot_x + (unsigned)(lane >> 3) * 128u, rd64 = slot_x + (unsigned)(lane >> 2) * 64u;
    const unsigned out128 = (unsigned)(lane >> 3) * pitch + (unsigned)(lane & 7) * 16u, out64 = (unsigned)(lane >> 2) * pitch + (unsigned)(lane & 3) * 16u;
    typedef const float __attribute__((address_space(3))) * fp;
    typedef const unsigned short __attribute__((address_space(3))) * sp;
    // A column's scale and bias belong to register 8 q4 + e of its half's lanes: lane 4 q4 + e of each row of 16.
    const unsigned sc = ldss + par * kScales, column = (unsigned)(wj * (WJ * 32) + 8 * ((lane & 15) >> 2) + 4 * hh + (lane & 3));
    float xs[kWI], ws[WJ], bias[WJ];
#pragma unroll
    for (int a = 0; a < kWI; ++a) xs[a] = *(fp)(uintptr_t)(sc + (unsigned)((wi * kWI + a) * 32 + ic) * 4u) * kRowShift;
#pragma unroll
    for (int b = 0; b < WJ; ++b) {
      ws[b] = *(fp)(uintptr_t)(sc + 1024u + (column + b * 32) * 4u) * kChannelShift;
      if constexpr (WIDE) bias[b] = *(fp)(uintptr_t)(sc + 2048u + (column + b * 32) * 4u);
      else bias[b] = __builtin_bit_cast(float, (unsigned)*(sp)(uintptr_t)(sc + 2048u + (column + b * 32) * 2u) << 16);
    }
    u32x4 v[4];
    auto park = [&](int n) __attribute__((always_inline)) {     // piece n into its half of the place
      const int a = n / NS, b0 = n % NS * WB, nb = WJ - b0 < WB ? WJ - b0 : WB;
      const unsigned buf = (unsigned)(n & 1) * 16384u;
#pragma unroll
      for (int b = b0; b < b0 + nb; ++b) {
        auto eight = [&](auto hc) __attribute__((always_inline)) {
          constexpr int h = decltype(hc)::value;
          float t[8];
          results<h>(t, acc[a][b], xs[a], ws[b], bias[b]);
          if constexpr (WIDE) {
#pragma unroll
            for (int q = 0; q < 2; ++q)
              *(wp4)(uintptr_t)(at128 + buf + (((unsigned)(2 * (2 * h + q) + hh)) ^ sw128) * 16u) = f32x4{t[4 * q], t[4 * q + 1], t[4 * q + 2], t[4 * q + 3]};
          } else {
            const unsigned c = (unsigned)((b - b0) * 4 + 2 * h);
            const unsigned at = (nb == 2 ? at128 : at64) + buf + half, sw = nb == 2 ? sw128 : sw64;
            const bf16x8 o = {(bf16)t[0], (bf16)t[1], (bf16)t[2], (bf16)t[3], (bf16)t[4], (bf16)t[5], (bf16)t[6], (bf16)t[7]};
            const u32x4 r = __builtin_bit_cast(u32x4, o);
            *(wp2)(uintptr_t)(at + (c ^ sw) * 16u) = u32x2{r[0], r[1]};
            *(wp2)(uintptr_t)(at + ((c + 1) ^ sw) * 16u) = u32x2{r[2], r[3]};
          }
        };
        eight(std::integral_constant<int, 0>{});
        eight(std::integral_constant<int, 1>{});
      }
      if (n % NS == NS - 1) start(a);
    };
    auto fetch_back = [&](int n) __attribute__((always_inline)) {
      const bool wide = WIDE || n % NS * WB + WB <= WJ;
      const unsigned buf = (unsigned)(n & 1) * 16384u;
#pragma unroll
      for (int it = 0; it < (wide ? 4 : 2); ++it) {
        const unsigned sw = wide ? (unsigned)(4 * it + (lane >> 4)) & 7u : (unsigned)(lane >> 4) & 3u;  // (row >> 1) & 7, (row >> 2) & 3
        v[it] = *(rp)(uintptr_t)((wide ? rd128 : rd64) + buf + (unsigned)it * 4096u + (((unsigned)(wide ? lane & 7 : lane & 3)) ^ sw) * 16u);
      }
    };
    auto store = [&](int n) __attribute__((always_inline)) {
      const int a = n / NS, b0 = n % NS * WB;
      const bool wide = WIDE || b0 + WB <= WJ;
      // (F is a multiple of 8: a lane's 16 bytes are in range together)
      const bool in = b0 * 32 * E + (wide ? lane & 7 : lane & 3) * 16 < cols * E;
#pragma unroll
      for (int it = 0; it < (wide ? 4 : 2); ++it) {
        const bool swapped = !WIDE && it >= (wide ? 2 : 1);
        const u32x4 o = swapped ? u32x4{v[it][2], v[it][3], v[it][0], v[it][1]} : v[it];
        const unsigned off = (wide ? out128 : out64) + (unsigned)(a * 32 + it * (wide ? 8 : 16)) * pitch + (unsigned)(b0 * 32 * E);
        if (order.stream) __builtin_amdgcn_raw_buffer_store_b128(o, rs, (int)(in ? off : kNowhere), 0, kStreamed);
        else __builtin_amdgcn_raw_buffer_store_b128(o, rs, (int)(in ? off : kNowhere), 0, 0);
      }
    };
    park(0);
    fetch_back(0);
#pragma unroll
    for (int n = 1; n < kWI * NS; ++n) {
      park(n);
      store(n - 1);
      fetch_back(n);
    }
    store(kWI * NS - 1);
  };

  // Start: tiles 0 and 1 on their way, the accumulators at 0, the first fragments.
  Where w = locate(wg);
  unsigned par = 0;
  scales_load(w, par);
  open(w);
#pragma unroll
  for (int n = 0; n < 2; ++n) {
#pragma unroll
    for (int x = 0; x < LX; ++x) issue_x(x);
#pragma unroll
    for (int x = 0; x < LW; ++x) issue_w(x);
    slot_x += kXTile;
    slot_w += n == 0 ? kWTile : 0u - kWTile;
    further_x();
    further_w();
    advance();
  }
  asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(LX + LW) : "memory");
#pragma unroll
  for (int a = 0; a < kWI; ++a) start(a);
#pragma unroll
  for (int f = 0; f < NF; ++f) fetch(0, f);
#pragma unroll
  for (int f = 0; f < NF; ++f) fetch(1, f);
  int left = nct;                      // contraction tiles of this output tile yet to be worked on
  int quiet = 1, passed = 1;           // tiles until something other than further() is due, and their number
  // byte offsets of the X tile being read and the next one; from the W tile being read to the other one
  unsigned x_now = 0, x_next = kXTile, w_step = kWTile;
  int fresh = 0;                       // results left in front of this tile
  for (;;) {
    // Products of contraction step kk.  Behind product m: the fragments of step kk + 2, and the loads of the tile two ahead
    // (X in steps 0 and 1, W in steps 2 and 3), in slots without fragment reads.
    auto step = [&](auto kkc) {
      constexpr int kk = decltype(kkc)::value;
      constexpr int sync = 1;                          // step 2: the barrier's slot
      constexpr int f0 = kk == 2 ? sync + 1 : 0;       // first slot with fragment reads (step 2: behind the barrier)
      constexpr FreeSlots<NP> slots = free_slots<NP, NF>(f0);
      constexpr int nfree = NP - f0 - NF, L = kk < 2 ? LX / 2 : LW / 2, x0 = (kk & 1) * L;
#pragma unroll
      for (int m = 0; m < NP; ++m) {
        mfma_acc_q8(acc[m / WJ][m % WJ], wf[kk][m % WJ], xf[kk][m / WJ]);
        if (kk == 2 && m == sync) {
          // Everyone has read its last fragments of this tile, and the next tile is there for everyone.  Younger than its
          // loads: the stores of an output tile's results, the loads of the next one's scales, and those of the X tile behind it.
          // (Branch in the assembly: the tile stays one basic block, over which the compiler keeps the order.)
          asm volatile(
              "s_cmp_lg_u32 %0, 0\n\t"
              "s_cbranch_scc1 .Ltvm_fresh_%=\n\t"
              "s_waitcnt vmcnt(%1)\n"
              ".Ltvm_fresh_%=:\n\t"
              "s_waitcnt vmcnt(%2) lgkmcnt(0)\n\t"
              "s_barrier" ::"s"(__builtin_amdgcn_readfirstlane(fresh)), "n"(LX), "n"(YOUNGER)
              : "memory", "scc");
          ox.move(x_next - x_now);
          ow.move(w_step);
        }
#pragma unroll
        for (int f = 0; f < NF; ++f)
          if (m == f0 + f * (NP - f0) / NF) fetch((kk + 2) & 3, f);
#pragma unroll
        for (int x = 0; x < L; ++x)
          if (m == slots.at[x * nfree / L]) {
            if (kk < 2) issue_x(x0 + x);
            else issue_w(x0 + x);
          }
        if (kk == 3 && m == 2) {  // the bookkeeping of a plain move to the next tile, in slots that have room
          const unsigned x_free = 3 * kXTile - x_now - x_next;
          slot_x += x_now - x_free;
          x_now = x_next;
          x_next = x_free;
          fresh = 0;
        }
        // (the descriptors move behind the tile's last loads: at the very end they are of size 0, which the move lets wrap)
        static_assert(kk != 3 || slots.at[(L - 1) * nfree / L] <= NP - 1, "W loads in front of their descriptor's move");
        if (kk == 3 && m == NP / 2) further_x();
        if (kk == 3 && m == NP - 1) {
          slot_w += w_step;
          w_step = 0u - w_step;
          further_w();
        }
      }
    };
    step(std::integral_constant<int, 0>{});
    step(std::integral_constant<int, 1>{});
    step(std::integral_constant<int, 2>{});
    step(std::integral_constant<int, 3>{});
    if (--quiet == 0) {
      c_left -= passed - 1;
      left -= passed;
      advance();
      // the cursor's moves are plain until it reaches the output tile's last one
      passed = quiet = max(1, c_left - 2);
      if (left > 0) passed = quiet = min(quiet, left);
      __builtin_amdgcn_s_waitcnt(0xc07f);  // scalar loads, here: with one on its way the fragments behind would all be waited for
    }
    if (left == 0) {
      mfma_settle();
      if (nct == 1) {  // (no other barrier since the scales were asked for)
        dma_wait();
        asm volatile("s_barrier" ::: "memory");
      }
      write_out(locate(wg), par);
      fresh = 1;
      wg += wg_per_xcd;
      if (wg >= id_end) break;
      par ^= 1;
      scales_load(locate(wg), par);
      left = nct;
      passed = quiet = min(quiet, left);
      __builtin_amdgcn_s_waitcnt(0xc07f);
    }
  }
  dma_wait();  // (no load may land in LDS that the next workgroup owns)
}

template <typename T>
hipError_t launch(int shape, const LinearQ8Args& a, hipStream_t st) {
  const int sets = a.x[1] != nullptr ? 2 : 1;
  const long long tiles = sets * tiles_q8(shape, a.R, a.F), per = (tiles + 7) / 8;
  const dim3 grid((unsigned)(8 * (per < 32 ? per : 32)));  // 8 XCDs x at most 32 CUs, fewer where an XCD's share of the tiles is smaller
  TileOrder order = tile_order(shape, sets, a.R, a.F);
  order.stream = ((a.ldy * (long long)sizeof(T)) | (long long)(reinterpret_cast<uintptr_t>(a.y[0]) | reinterpret_cast<uintptr_t>(a.y[1]))) % 64 == 0;
  if (shape == kQ256x192) hipLaunchKernelGGL((q8_pipe_kernel<T, 3>), grid, dim3(256), 0, st, a, order);
  else hipLaunchKernelGGL((q8_pipe_kernel<T, 2>), grid, dim3(256), 0, st, a, order);
  return hipGetLastError();
}
static_assert(kTileColsQ8[kQ256x192] == 64 * 3 && kTileColsQ8[kQ256x128] == 64 * 2, "the plan's tiles");

}  // namespace

hipError_t launch_linear_q8_pipe(int shape, const LinearQ8Args& a, int dtype, hipStream_t st) {
  return dtype == 1 ? launch<bf16>(shape, a, st) : launch<float>(shape, a, st);
}

}  // namespace tvm
