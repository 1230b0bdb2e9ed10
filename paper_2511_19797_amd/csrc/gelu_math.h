// The GELU in its tanh form with its first two derivatives (gelu.hip has the formulas).
#pragma once
#include "tvm_common.h"

namespace tvm {
namespace {

constexpr float kK = 0.7978845608028654f, kC = 0.044715f, kTwoLog2e = 2.8853900817779268f;

struct Gelu {
  float half_1pt, g1, g2;  // (1 + t)/2, gelu', gelu''
};
// With e = exp(2w) and r = 1/(e + 1):  t = 1 - 2r,  (1 + t)/2 = 1 - r =: h,  1 - t^2 = 4 r h.  For large |w| the
// exponential overflows to inf (r = 0, h = 1) or underflows to 0 (r = 1, h = 0): the limits come out exact.
template <bool SECOND>
__device__ __forceinline__ Gelu gelu_parts(float u) {
  const float u2 = u * u;
  const float e = __builtin_amdgcn_exp2f(u * fmaf(kTwoLog2e * kK * kC, u2, kTwoLog2e * kK));  // exp(2w)
  const float r = __builtin_amdgcn_rcpf(e + 1.0f);
  const float h = 1.0f - r;
  const float q = u * r * h;                               // u (1 - t^2) / 4
  const float wp = fmaf(3.0f * kK * kC, u2, kK);           // w'
  Gelu g;
  g.half_1pt = h;
  g.g1 = fmaf(2.0f * q, wp, h);
  // gelu'' = (1 - t^2) w' + u/2 (1 - t^2) (w'' - 2 t w'^2),  t = 1 - 2r
  g.g2 = SECOND ? fmaf(2.0f * q, fmaf(wp * wp, fmaf(4.0f, r, -2.0f), 6.0f * kK * kC * u), 4.0f * r * h * wp) : 0.f;
  return g;
}

}  // namespace
}  // namespace tvm
