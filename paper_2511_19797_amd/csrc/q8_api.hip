// C-ABI entry points of the 8-bit operators: argument validation and dispatch.  No allocation, no synchronisation.
#include <math.h>

#include "api_checks.h"
#include "q8.h"

namespace {

bool dtype_ok(int dtype) { return dtype == TVMATTN_F32 || dtype == TVMATTN_BF16; }
// R rows of `cols` elements at a pitch of `ld` elements
Buf pitched(const void* p, int R, int cols, long long ld, long long esz) { return Buf{p, 1, {R, 0, 0}, {ld * esz, 0, 0}, cols * esz}; }
// scales: one float per row or channel, as aligned as floats are (a range of rows of a longer vector)
Buf scales(const void* p, long long n) {
  Buf b = plain(p, 4 * n);
  b.align = 4;
  return b;
}

// The rows of tvmattn_rowquant_fwd and tvmattn_gelu_jvp_fwd_q8.
int rows_args(int R, int C, int dtype, const void* x, const void* tx, long long ldx, void* q, float* s, void* tq, float* ts,
              tvm::RowsQ8Args& g) {
  if (R < 1 || C < 1 || ldx < 0) return TVMATTN_INVALID_ARG;
  if (!dtype_ok(dtype)) return TVMATTN_UNSUPPORTED;
  if (ldx == 0) ldx = C;
  if (ldx < C) return TVMATTN_INVALID_ARG;
  const bool none = tx == nullptr;
  if (none != (tq == nullptr) || none != (ts == nullptr)) return TVMATTN_INVALID_ARG;
  if (!tvm::rows_q8_supported(C, dtype) || ldx % tvm::vec_of(dtype) != 0 || ldx > (1ll << 45) / R) return TVMATTN_UNSUPPORTED;
  const long long e = esz_of(dtype), n = (long long)R * C;
  const Buf in[] = {pitched(x, R, C, ldx, e), unless(none, pitched(tx, R, C, ldx, e))};
  const Buf out[] = {plain(q, n), scales(s, R), unless(none, plain(tq, n)), unless(none, scales(ts, R))};
  const int rc = check_bufs(in, out);
  if (rc) return rc;
  g = tvm::RowsQ8Args{x, tx, ldx, R, C, static_cast<signed char*>(q), static_cast<signed char*>(tq), s, ts};
  return TVMATTN_OK;
}
int status(hipError_t e) { return e == hipSuccess ? TVMATTN_OK : TVMATTN_LAUNCH_FAILED; }

}  // namespace

extern "C" {

int tvmattn_rowquant_fwd(int R, int C, int dtype, const void* x, const void* tx, long long ldx, void* q, float* s, void* tq,
                         float* ts, void* hip_stream) {
  tvm::RowsQ8Args g;
  const int rc = rows_args(R, C, dtype, x, tx, ldx, q, s, tq, ts, g);
  return rc ? rc : status(tvm::launch_rowquant(g, dtype, static_cast<hipStream_t>(hip_stream)));
}

int tvmattn_gelu_jvp_fwd_q8(int R, int C, int dtype, const void* u, const void* tu, long long ldu, void* q, float* s, void* tq,
                            float* ts, void* hip_stream) {
  tvm::RowsQ8Args g;
  const int rc = rows_args(R, C, dtype, u, tu, ldu, q, s, tq, ts, g);
  return rc ? rc : status(tvm::launch_gelu_q8(g, dtype, static_cast<hipStream_t>(hip_stream)));
}

int tvmattn_gate_adaln_jvp_fwd_q8(int B, int T, int C, int dtype, const void* x, const void* tx, const void* h, const void* th,
                                  const float* c, const float* tc, const float* a, const float* ta, const float* b,
                                  const float* tb, float eps, void* z, void* tz, void* q, float* s, void* tq, float* ts,
                                  void* hip_stream) {
  if (B < 1 || T < 1 || C < 1) return TVMATTN_INVALID_ARG;
  if (!dtype_ok(dtype)) return TVMATTN_UNSUPPORTED;
  if (!(eps >= 0.f) || isinf(eps)) return TVMATTN_INVALID_ARG;
  const bool gate = h != nullptr, tan = tx != nullptr;
  // the residual's operands and outputs come together, and so do those of the tangent
  if (gate != (c != nullptr) || gate != (z != nullptr)) return TVMATTN_INVALID_ARG;
  if (tan != (ta != nullptr) || tan != (tb != nullptr) || tan != (tq != nullptr) || tan != (ts != nullptr)) return TVMATTN_INVALID_ARG;
  if ((gate && tan) != (th != nullptr) || (gate && tan) != (tc != nullptr) || (gate && tan) != (tz != nullptr)) return TVMATTN_INVALID_ARG;
  if (!tvm::norm_q8_supported(C, dtype) || (long long)B * T >= (1ll << 31) || B > 65535) return TVMATTN_UNSUPPORTED;
  const long long n = (long long)B * T * C, e = esz_of(dtype), mb = (long long)B * C * 4, rows = (long long)B * T;
  const Buf in[] = {plain(x, n * e),  unless(!tan, plain(tx, n * e)), unless(!gate, plain(h, n * e)), unless(!gate || !tan, plain(th, n * e)),
                    plain(a, mb),     unless(!tan, plain(ta, mb)),    plain(b, mb),                   unless(!tan, plain(tb, mb)),
                    unless(!gate, plain(c, mb)), unless(!gate || !tan, plain(tc, mb))};
  const Buf out[] = {unless(!gate, plain(z, n * e)), unless(!gate || !tan, plain(tz, n * e)), plain(q, n), scales(s, rows),
                     unless(!tan, plain(tq, n)), unless(!tan, scales(ts, rows))};
  // z may be x itself and tz tx itself: a wave has a row's x and tx in registers before it writes that row, and nobody else touches it
  const int rc = check_bufs(in, out, 0, 0, 1, 1);
  if (rc) return rc;
  const tvm::GateAdalnQ8Args g{x, tx, h, th, a, ta, b, tb, c, tc, z, tz, static_cast<signed char*>(q), static_cast<signed char*>(tq),
                               s, ts, B, T, C, eps};
  return status(tvm::launch_gate_adaln_q8(g, dtype, static_cast<hipStream_t>(hip_stream)));
}

int tvmattn_linear_jvp_fwd_q8(int R, int K, int F, int dtype, const void* xq, const float* xs, const void* txq, const float* txs,
                              long long ldx, const void* wq, const float* ws, const void* bias, void* y, void* ty, long long ldy,
                              void* hip_stream) {
  if (R < 1 || K < 1 || F < 1 || ldx < 0 || ldy < 0) return TVMATTN_INVALID_ARG;
  if (!dtype_ok(dtype)) return TVMATTN_UNSUPPORTED;
  if (ldx == 0) ldx = K;
  if (ldy == 0) ldy = F;
  if (ldx < K || ldy < F) return TVMATTN_INVALID_ARG;
  const bool none = txq == nullptr;
  if (none != (txs == nullptr) || none != (ty == nullptr)) return TVMATTN_INVALID_ARG;
  if (!tvm::linear_q8_supported(R, K, F, ldx, ldy)) return TVMATTN_UNSUPPORTED;
  const long long e = esz_of(dtype);
  Buf wscales = scales(ws, F);
  wscales.align = 16;  // (read four at a time)
  const Buf in[] = {pitched(xq, R, K, ldx, 1), scales(xs, R), unless(none, pitched(txq, R, K, ldx, 1)), unless(none, scales(txs, R)),
                    plain(wq, (long long)F * K), wscales, unless(!bias, plain(bias, F * e))};
  const Buf out[] = {pitched(y, R, F, ldy, e), unless(none, pitched(ty, R, F, ldy, e))};
  const int rc = check_bufs(in, out);
  if (rc) return rc;
  const tvm::LinearQ8Args g{{static_cast<const signed char*>(xq), static_cast<const signed char*>(txq)}, {xs, txs},
                            static_cast<const signed char*>(wq), ws, bias, {y, ty}, ldx, ldy, R, K, F};
  return status(tvm::launch_linear_q8(g, dtype, static_cast<hipStream_t>(hip_stream)));
}

}  // extern "C"
