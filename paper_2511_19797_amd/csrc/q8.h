// The 8-bit operators around the block's linear layers (rows_q8.hip, linear_q8.hip): arguments and launchers.
//
// An 8-bit row: s = max|v| / 127 in float32 and q_j = round(v_j 127 / max|v|) to the nearest integer, ties to even; it stands for
// q s.  Exactly so for values that came in; values that are worked out first are float32 with a few roundings of their own, and next to
// the border between two integers either may come out (the rounding itself is off by 2^-17 of a step at most).  A row of zeros (or with nothing of 2^-100 or more) has
// s = 0 and q = 0; one that holds a NaN or an infinity has s = NaN and q = 0, so that whatever is made of it is NaN.
#pragma once
#include "tvm_common.h"

namespace tvm {

// [R][C] rows (pitch ld elements) and, where tx is there, as many of its tangent
struct RowsQ8Args {
  const void *x, *tx;
  long long ld;
  int R, C;
  signed char *q, *tq;  // dense
  float *s, *ts;
};
struct GateAdalnQ8Args {
  const void *x, *tx, *h, *th;             // [B][T][C]; tx, th null: no tangent; h null: no residual
  const float *a, *ta, *b, *tb, *c, *tc;   // [B][C]
  void *z, *tz;
  signed char *q, *tq;
  float *s, *ts;
  int B, T, C;
  float eps;
};
struct LinearQ8Args {
  const signed char* x[2];  // [R][K], pitch ldx; [1] null: no tangent
  const float* xs[2];       // [R]
  const signed char* w;     // [F][K]
  const float* ws;          // [F]
  const void* bias;         // [F] of the output's type, or null; not on the tangent
  void* y[2];               // [R][F], pitch ldy elements
  long long ldx, ldy;
  int R, K, F;
};

// Widest row: 4 chunks of 16 bytes per thread of 16 waves; of the norm, which keeps a row in one wave, 8 per lane.
constexpr int kMaxChunksQ8 = 4096, kMaxChunksNormQ8 = 512;
inline int vec_of(int dtype) { return dtype == 1 ? 8 : 4; }
inline bool rows_q8_supported(int C, int dtype) { return C % vec_of(dtype) == 0 && C / vec_of(dtype) <= kMaxChunksQ8; }
inline bool norm_q8_supported(int C, int dtype) { return C % vec_of(dtype) == 0 && C / vec_of(dtype) <= kMaxChunksNormQ8; }
// A sum of K products of magnitude 2^14 at most stays inside 32 bits for K <= 2^16.  Pitches up to 2^20: a tile's byte offsets
// (256 rows x pitch) stay inside 32 bits.  At most 2^30 rows and 2^38 results: rows and output tiles of any shape are
// counted in 31 bits, past the last one too.
inline bool linear_q8_supported(int R, int K, int F, long long ldx, long long ldy) {
  return R <= (1 << 30) && (long long)R * F <= (1ll << 38) && K % 16 == 0 && K <= (1 << 16) && F % 8 == 0 && F <= (1 << 20) && ldx % 16 == 0 && ldx <= (1ll << 20) && ldy % 8 == 0 &&
         ldy <= (1ll << 20);
}

hipError_t launch_rowquant(const RowsQ8Args& a, int dtype, hipStream_t st);
hipError_t launch_gelu_q8(const RowsQ8Args& a, int dtype, hipStream_t st);
hipError_t launch_gate_adaln_q8(const GateAdalnQ8Args& a, int dtype, hipStream_t st);
hipError_t launch_linear_q8(const LinearQ8Args& a, int dtype, hipStream_t st);

}  // namespace tvm
