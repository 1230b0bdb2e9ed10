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

// gelu and gelu' to a few float32 roundings of their own size, also where they are tiny (u at -9: 2^-93): what an 8-bit row needs, whose
// step is its largest value's.  (Above, 1 - r for r near 1 has an error of 2^-24 whatever its size; rows around u = -4.5 came out 4 steps
// off and rows around -6 lost.)  (1 + tanh w)/2 =: s = 1/(1 + exp(-2w)), a sum of positive numbers, is 0 or 1 where exp leaves the range;
// gelu = u s,  gelu' = s + 2 u w' (s - s^2): the difference is as good as s for u < 0, and for u > 0, where s is near 1, off by 2^-24 of
// gelu' times 2 u w' (35 at u = 5; behind that s is 1).  From |u| = 16 on s is 0 or 1, s - s^2 is 0, and w' is
// taken at 16: no finite u makes an infinity there to multiply with 0.
struct GeluSmall {
  float s, g1;
};
template <bool FIRST>
__device__ __forceinline__ GeluSmall gelu_small(float u) {
  constexpr double kW = 0.79788456080286535588, kL = -2.0 * kW * 1.44269504088896340736;  // -2 w log2 e = kL (u + c u^3)
  const float u2 = u * u;
  GeluSmall g;
  g.s = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(u * fmaf((float)(kL * 0.044715), u2, (float)kL)));
  g.g1 = FIRST ? fmaf(u, fmaf((float)(6.0 * kW * 0.044715), fminf(u2, 256.0f), (float)(2.0 * kW)) * fmaf(-g.s, g.s, g.s), g.s) : 0.f;
  return g;
}

}  // namespace
}  // namespace tvm
