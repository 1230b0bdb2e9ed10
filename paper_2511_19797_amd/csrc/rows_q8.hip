// Rows of tokens into 8 bits with a float32 scale per row (q8.h has the definition), with what comes before it in the block's
// forward: nothing (weights, the attention's output), the MLP's activation, or the gated residual and the normalised modulation.
// Every operator carries an optional tangent, whose rows have scales of their own.  Memory-bound: one pass, everything between
// the loads and the stores in float32 registers.
//
// A row belongs to one wave where it fits (4 chunks of 16 bytes per lane: 2048 bf16 values), so that its maximum and its sums
// are lane exchanges, with no barrier; longer rows belong to 4 or 16 waves, which meet once in LDS.
// us (TB/s of what has to be read and written): rows of 16384 x 1152 with tangent, bf16, 19.6 (5.8), float32 34.8 (5.4); activation 16384 x
// 4608 with tangent 77 (5.9), without 41 (5.5), 250 x 1536 float32 2.7; norm with residual 16 x 1024 x 1152 with tangent 50.4 (5.2), without
// 24.5 (5.4), float32 with tangent 99 (5.0), 1 x 256 x 1152 6.4.
#include <algorithm>

#include "gelu_math.h"
#include "q8.h"
#include "row_ops.h"

namespace tvm {
namespace {

// ---- a row's largest magnitude.  Magnitudes are compared as the integers of their bits: the order of the floats, with infinity
// and then every NaN on top.
__device__ __forceinline__ unsigned mag(float v) { return __builtin_bit_cast(unsigned, v) & 0x7fffffffu; }
template <int CTRL, int ROWS>
__device__ __forceinline__ unsigned dpp_bits(unsigned x) {
  return (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, ROWS, 0xf, false);
}
__device__ __forceinline__ unsigned wave_max_dpp(unsigned x) {  // the moves of wave_sum_dpp; 0 is neutral here too
  x = max(x, dpp_bits<0xB1, 0xf>(x));
  x = max(x, dpp_bits<0x4E, 0xf>(x));
  x = max(x, dpp_bits<0x141, 0xf>(x));
  x = max(x, dpp_bits<0x140, 0xf>(x));
  x = max(x, dpp_bits<0x142, 0xa>(x));
  x = max(x, dpp_bits<0x143, 0xc>(x));
  return (unsigned)__builtin_amdgcn_readlane((int)x, 63);
}

struct Scale {
  float s, inv;    // what a step stands for, steps per unit
  unsigned keep;   // 0: the row's values are all to be 0
};
__device__ __forceinline__ Scale scale_of(unsigned m) {
  const float top = __builtin_bit_cast(float, m);
  if (m >= 0x7f800000u) return {__builtin_nanf(""), 0.f, 0u};
  if (m < 0x0d800000u) return {0.f, 0.f, 0u};  // below 2^-100: 127 / top would leave float32's range
  return {top / 127.0f, 127.0f / top, ~0u};
}
// Four values as bytes.  v inv + 1.5 2^23 in one rounding leaves round(v inv) in the low bits (two's complement).  (inv is off by 2^-24:
// for values that were worked out in float32 and are off by as much.)
__device__ __forceinline__ unsigned pack4(float v0, float v1, float v2, float v3, const Scale& k) {
  constexpr float kMagic = 12582912.0f;
  const unsigned b0 = __builtin_bit_cast(unsigned, fmaf(v0, k.inv, kMagic)), b1 = __builtin_bit_cast(unsigned, fmaf(v1, k.inv, kMagic));
  const unsigned b2 = __builtin_bit_cast(unsigned, fmaf(v2, k.inv, kMagic)), b3 = __builtin_bit_cast(unsigned, fmaf(v3, k.inv, kMagic));
  return (__builtin_amdgcn_perm(b1, b0, 0x0c0c0400u) | __builtin_amdgcn_perm(b3, b2, 0x04000c0cu)) & k.keep;
}
template <int VEC>
__device__ __forceinline__ void store_q8(signed char* p, const float (&v)[VEC], const Scale& k) {
  if constexpr (VEC == 8) *reinterpret_cast<uint2*>(p) = make_uint2(pack4(v[0], v[1], v[2], v[3], k), pack4(v[4], v[5], v[6], v[7], k));
  else *reinterpret_cast<unsigned*>(p) = pack4(v[0], v[1], v[2], v[3], k);
}
// The nearest step to v 127 / top, ties to even, of values as they came in.  127 / top is not a float32, so that the product above goes to
// either side of a tie (top / 2, 63.5 steps, is one whatever top is, and common in bf16).  Instead: with an inverse surely too
// large and one surely too small, by 2^-22, all but one value in 60 000 come out the same, and then the exact quotient, which lies
// strictly between, does too.  The others are next to n + 1/2 steps.
//   bf16: v = V and top = M 2^k as integers, V and M below 2^8, k >= 0: 254 V and (2 n + 1) M 2^k are equal or 1 apart at least, 2^-16 of
//     themselves.  So it is a tie, and of the two integers the even one is taken, byte by byte.
//   float32: 254 v and (2 n + 1) top decide, whole numbers of at most 32 bits times one power of two, exact in float64.
// us of one product | of this: bf16 4608 x 1152 5.9 | 5.6, 16384 x 1152 of a pitch of 3456 with tangent 19.8 | 19.4, 16384 x 2304 with
// tangent 36.8 | 38.5; float32 with tangent 16384 x 1152 33.5 | 34.3, 4096 x 4608 38.0 | 40.8.  (bf16 by the branch into float64: 21.1 for 19.4.)
__device__ __forceinline__ int nearest(float v, float top, int a, int b) {
  const double x = 254.0 * (double)v, border = (double)(a + b) * (double)top;
  return x > border ? max(a, b) : x < border ? min(a, b) : (a & 1) == 0 ? a : b;
}
// All of a thread's chunks of a row: w gets the bytes.
template <typename T, int NCH>
__device__ __forceinline__ void pack_exact(unsigned (&w)[NCH][2], const float (&v)[NCH][Chunk<T>::VEC], const Scale& k, float top) {
  constexpr int WORDS = Chunk<T>::VEC / 4;
  constexpr float kOff = 2.384185791015625e-07f;  // 2^-22
  const Scale up = {k.s, k.inv * (1.0f + kOff), k.keep}, down = {k.s, k.inv * (1.0f - kOff), k.keep};
  unsigned other[NCH][2], differ = 0;
#pragma unroll
  for (int j = 0; j < NCH; ++j)
#pragma unroll
    for (int n = 0; n < WORDS; ++n) {
      const float* const f = v[j] + 4 * n;
      w[j][n] = pack4(f[0], f[1], f[2], f[3], up);
      other[j][n] = pack4(f[0], f[1], f[2], f[3], down);
      if constexpr (sizeof(T) == 2) {
        const unsigned odd = w[j][n] & 0x01010101u, take = (odd << 8) - odd;  // 255 in the bytes that are odd
        w[j][n] = (w[j][n] & ~take) | (other[j][n] & take);
      } else {
        differ |= w[j][n] ^ other[j][n];
      }
    }
  if (sizeof(T) == 4 && differ != 0) {
#pragma unroll
    for (int j = 0; j < NCH; ++j) {
      unsigned exact = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        exact |= (unsigned)(nearest(v[j][e], top, (signed char)(w[j][0] >> 8 * e), (signed char)(other[j][0] >> 8 * e)) & 255) << 8 * e;
      w[j][0] = exact;
    }
  }
}
template <int VEC>
__device__ __forceinline__ unsigned mag_of(const float (&v)[VEC], unsigned m) {
#pragma unroll
  for (int e = 0; e < VEC; ++e) m = max(m, mag(v[e]));
  return m;
}

// ---- rows as they are (GELU false), or through the activation.  NW waves to a row, NCH chunks per thread.  Without the
// activation the tangent's rows are rows like the others: blockIdx.y.
// Five waves per SIMD at most for the bf16 activation with tangent: with the six to eight that its registers would allow, 16384 x 4608
// takes 78.8 us instead of 76.5, 16384 x 3456 58.7 instead of 56.9, 16384 x 512 12.0 instead of 11.2.
template <typename T, bool GELU, bool TAN, int NCH, int NW>
__global__ __launch_bounds__(NW == 1 ? 256 : 64 * NW) __attribute__((amdgpu_waves_per_eu(1, sizeof(T) == 2 && GELU && TAN ? 5 : 8))) void rows_q8_kernel(RowsQ8Args a) {
  constexpr int VEC = Chunk<T>::VEC, SETS = GELU && TAN ? 2 : 1, PER_WG = NW == 1 ? 4 : 1;
  __shared__ unsigned red[SETS][NW];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const long long row = ((long long)blockIdx.z * gridDim.x + blockIdx.x) * PER_WG + (NW == 1 ? wave : 0);
  if (row >= a.R) return;  // (NW > 1: the whole workgroup or nobody)
  const bool second = !GELU && blockIdx.y == 1;
  const T* x = static_cast<const T*>(second ? a.tx : a.x) + row * a.ld;
  const T* tx = static_cast<const T*>(a.tx) + row * a.ld;
  signed char* const q[2] = {(second ? a.tq : a.q) + row * a.C, a.tq + row * a.C};
  const int first = NW == 1 ? lane : (int)threadIdx.x, chunks = a.C / VEC;
  Raw<T> raw[SETS][NCH];
#pragma unroll
  for (int j = 0; j < NCH; ++j) {  // chunks past the row's end are read as the first one and take no further part
    const int c = first + j * 64 * NW, at = c < chunks ? c * VEC : 0;
    raw[0][j] = load_raw<T>(x + at);
    if constexpr (SETS == 2) raw[1][j] = load_raw<T>(tx + at);
  }
  // All loads first: with the work below some came behind a wait for the one before (16384 x 1152 float32 with tangent 39.6 us, 34.3
  // with the fence).  The activation's loads come first without it, and its arithmetic loses by it (43 | 45 us).
  if constexpr (!GELU) __builtin_amdgcn_sched_barrier(0);
  float v[SETS][NCH][VEC];
  unsigned m[SETS] = {};
#pragma unroll
  for (int j = 0; j < NCH; ++j) {
    const bool live = first + j * 64 * NW < chunks;
    widen<T>(v[0][j], raw[0][j]);
    if constexpr (GELU) {
      float t[VEC];
      if constexpr (SETS == 2) widen<T>(t, raw[1][j]);
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const GeluSmall g = gelu_small<SETS == 2>(v[0][j][e]);
        v[0][j][e] *= g.s;
        if constexpr (SETS == 2) v[1][j][e] = g.g1 * t[e];
      }
    }
#pragma unroll
    for (int k = 0; k < SETS; ++k) m[k] = live ? mag_of<VEC>(v[k][j], m[k]) : m[k];
  }
#pragma unroll
  for (int k = 0; k < SETS; ++k) m[k] = wave_max_dpp(m[k]);
  if constexpr (NW > 1) {
    if (lane == 0) {
#pragma unroll
      for (int k = 0; k < SETS; ++k) red[k][wave] = m[k];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < SETS; ++k)
#pragma unroll
      for (int w = 0; w < NW; ++w) m[k] = max(m[k], red[k][w]);
  }
#pragma unroll
  for (int k = 0; k < SETS; ++k) {
    const Scale sc = scale_of(m[k]);
    if (first == 0) (second || k == 1 ? a.ts : a.s)[row] = sc.s;
    unsigned exact[NCH][2];
    if constexpr (!GELU) pack_exact<T, NCH>(exact, v[k], sc, __builtin_bit_cast(float, m[k]));
#pragma unroll
    for (int j = 0; j < NCH; ++j) {
      const int c = first + j * 64 * NW;
      if (c >= chunks) continue;
      signed char* const p = q[k] + c * VEC;
      if constexpr (GELU) store_q8<VEC>(p, v[k][j], sc);
      else if constexpr (VEC == 8) *reinterpret_cast<uint2*>(p) = make_uint2(exact[j][0], exact[j][1]);
      else *reinterpret_cast<unsigned*>(p) = exact[j][0];
    }
  }
}

// ---- z = x + RMSNorm^-(c) o h,  y = RMSNorm^-(z) o RMSNorm^-(a) + RMSNorm^-(b)  (adaln.hip), y and ty in 8 bits; z, tz are
// rounded on their way out and used as they were before.  A workgroup works out its batch element's normalised vectors once,
// into LDS (with the tangents 24 bytes per column), and its four waves then take a row each, with no further barrier.  120 registers
// at three chunks per lane, four waves per SIMD: with a row's chunks interleaved and the next row's on their way it took 256, and 71 us
// instead of 50 at 16 x 1024 x 1152.
// From 5 to 8 chunks per lane there is one instance, at one wave per SIMD: 4 x 1024 x 2048 with tangent 23.9 us, x 2056 45.5, x 4096 72;
// without 12.3 and 15.6.
constexpr int kNormWaves = 4;  // (2 | 4 | 8: 16 x 1024 x 1152 118 | 50 | 52 us, 1 x 256 x 1152 8.3 | 6.4 | 7.2)
template <typename T, bool TAN, bool GATE, int NCH>
__global__ __launch_bounds__(64 * kNormWaves, NCH <= 3 ? 4 : NCH == 4 ? 3 : 1) void gate_adaln_q8_kernel(GateAdalnQ8Args g) {
  constexpr int VEC = Chunk<T>::VEC, NV = GATE ? 3 : 2, PL = VEC / 4;
  extern __shared__ __attribute__((aligned(16))) float4 coef[];  // [vector, tangent of it ...][PL][chunks]: 16 bytes of a chunk per plane
  __shared__ float red[kNormWaves][2 * NV];
  const int b = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int chunks = g.C / VEC, quads = g.C / 4;
  const float invc = 1.0f / (float)g.C;
  const long long base = (long long)b * g.T;
  const T *x = static_cast<const T*>(g.x), *tx = static_cast<const T*>(g.tx), *h = static_cast<const T*>(g.h), *th = static_cast<const T*>(g.th);
  Raw<T> rx[NCH], rh[GATE ? NCH : 1], rt[TAN ? NCH : 1], rth[TAN && GATE ? NCH : 1];
  auto load = [&](unsigned t) {
    const long long at0 = (base + t) * g.C;
#pragma unroll
    for (int j = 0; j < NCH; ++j) {  // chunks past the row's end are read as the first one and take no further part
      const int c = lane + 64 * j;
      const long long at = at0 + (c < chunks ? c * VEC : 0);
      rx[j] = load_raw<T>(x + at);
      if constexpr (GATE) rh[j] = load_raw<T>(h + at);
      if constexpr (TAN) rt[j] = load_raw<T>(tx + at);
      if constexpr (TAN && GATE) rth[j] = load_raw<T>(th + at);
    }
  };
  unsigned t = blockIdx.x * kNormWaves + (unsigned)wave;  // (T < 2^31: a step past the last row stays in range)
  const unsigned T_rows = (unsigned)g.T;
  // Where quad n (four columns) of a vector is kept; this thread's quads are tid + 256 i.  All loads first, the first row's behind
  // them: the prologue is one memory latency and two barriers.
  constexpr int NQ = (NCH * PL + 3) / 4, NT = 64 * kNormWaves;
  auto place = [&](int vec, int n) { return (vec * PL + (PL == 1 ? 0 : n & 1)) * chunks + (PL == 1 ? n : n >> 1); };
  const float* const vs[3] = {g.a, g.b, g.c};
  const float* const tvs[3] = {g.ta, g.tb, g.tc};
  float4 v4[NV][NQ], t4[TAN ? NV : 1][NQ];
#pragma unroll
  for (int k = 0; k < NV; ++k)
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
      const long long at = (long long)b * g.C + 4 * min(tid + NT * i, quads - 1);
      v4[k][i] = *reinterpret_cast<const float4*>(vs[k] + at);
      if constexpr (TAN) t4[k][i] = *reinterpret_cast<const float4*>(tvs[k] + at);
    }
  if (t < T_rows) load(t);
  __builtin_amdgcn_sched_barrier(0);
  float sums[2 * NV];
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    float s = 0.f, st = 0.f;
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
      const float4 v = v4[k][i];
      const bool live = tid + NT * i < quads;  // (quads past the last one were read as the last one)
      s += live ? fmaf(v.x, v.x, fmaf(v.y, v.y, fmaf(v.z, v.z, v.w * v.w))) : 0.f;
      if constexpr (TAN) {
        const float4 u = t4[k][i];
        st += live ? fmaf(v.x, u.x, fmaf(v.y, u.y, fmaf(v.z, u.z, v.w * u.w))) : 0.f;
      }
    }
    sums[2 * k] = wave_sum_dpp(s);
    sums[2 * k + 1] = TAN ? wave_sum_dpp(st) : 0.f;
  }
  if (lane == 0) {
#pragma unroll
    for (int k = 0; k < 2 * NV; ++k) red[wave][k] = sums[k];
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    float s = 0.f, st = 0.f;
#pragma unroll
    for (int w = 0; w < kNormWaves; ++w) {
      s += red[w][2 * k];
      st += red[w][2 * k + 1];
    }
    const float r = 1.0f / sqrtf(s * invc + g.eps), r3m = r * r * r * (st * invc);
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
      const int n = tid + NT * i;
      if (n >= quads) break;
      const float4 v = v4[k][i];
      coef[place(TAN ? 2 * k : k, n)] = make_float4(v.x * r, v.y * r, v.z * r, v.w * r);
      if constexpr (TAN) {
        const float4 u = t4[k][i];
        coef[place(2 * k + 1, n)] = make_float4(u.x * r - v.x * r3m, u.y * r - v.y * r3m, u.z * r - v.z * r3m, u.w * r - v.w * r3m);
      }
    }
  }
  __syncthreads();
  auto vector = [&](float (&out)[VEC], int vec, int c) {
#pragma unroll
    for (int p = 0; p < PL; ++p) {
      const float4 v = coef[(vec * PL + p) * chunks + c];
      out[4 * p] = v.x;
      out[4 * p + 1] = v.y;
      out[4 * p + 2] = v.z;
      out[4 * p + 3] = v.w;
    }
  };
  constexpr int A = 0, TA = 1, B = TAN ? 2 : 1, TB = 3, C = TAN ? 4 : 2, TC = 5;
  while (t < T_rows) {
    const long long row = base + t, at0 = row * g.C;
    float v[NCH][VEC], w[TAN ? NCH : 1][VEC];
    float sxx = 0.f, sxt = 0.f;
#pragma unroll
    for (int j = 0; j < NCH; ++j) {
      const int c = lane + 64 * j;
      const bool live = c < chunks;
      widen<T>(v[j], rx[j]);
      if constexpr (TAN) widen<T>(w[j], rt[j]);
      if constexpr (GATE) {
        float hv[VEC], gc[VEC];
        widen<T>(hv, rh[j]);
        vector(gc, C, live ? c : 0);
        if constexpr (TAN) {
          float thv[VEC], tgc[VEC];
          widen<T>(thv, rth[j]);
          vector(tgc, TC, live ? c : 0);
#pragma unroll
          for (int e = 0; e < VEC; ++e) w[j][e] = fmaf(gc[e], thv[e], fmaf(tgc[e], hv[e], w[j][e]));
        }
#pragma unroll
        for (int e = 0; e < VEC; ++e) v[j][e] = fmaf(gc[e], hv[e], v[j][e]);
        if (live) {
          store_row<T>(static_cast<T*>(g.z) + at0 + c * VEC, v[j]);
          if constexpr (TAN) store_row<T>(static_cast<T*>(g.tz) + at0 + c * VEC, w[j]);
        }
      }
      if (live) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          sxx = fmaf(v[j][e], v[j][e], sxx);
          if constexpr (TAN) sxt = fmaf(v[j][e], w[j][e], sxt);
        }
      }
      __builtin_amdgcn_sched_barrier(0);  // one chunk at a time: interleaved chunks cost more registers than they gain
    }
    const float r = 1.0f / sqrtf(wave_sum_dpp(sxx) * invc + g.eps);
    const float r3m = TAN ? r * r * r * (wave_sum_dpp(sxt) * invc) : 0.f;
    unsigned m = 0, tm = 0;
#pragma unroll
    for (int j = 0; j < NCH; ++j) {
      const int c = lane + 64 * j;
      const bool live = c < chunks;
      float ah[VEC], bh[VEC];
      vector(ah, A, live ? c : 0);
      vector(bh, B, live ? c : 0);
      if constexpr (TAN) {
        float tah[VEC], tbh[VEC];
        vector(tah, TA, live ? c : 0);
        vector(tbh, TB, live ? c : 0);
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          const float xh = v[j][e] * r, txh = w[j][e] * r - v[j][e] * r3m;
          w[j][e] = fmaf(txh, ah[e], fmaf(xh, tah[e], tbh[e]));
        }
        tm = live ? mag_of<VEC>(w[j], tm) : tm;
      }
#pragma unroll
      for (int e = 0; e < VEC; ++e) v[j][e] = fmaf(v[j][e] * r, ah[e], bh[e]);
      m = live ? mag_of<VEC>(v[j], m) : m;
      __builtin_amdgcn_sched_barrier(0);
    }
    const Scale sc = scale_of(wave_max_dpp(m)), tsc = TAN ? scale_of(wave_max_dpp(tm)) : Scale{};
    if (lane == 0) {
      g.s[row] = sc.s;
      if constexpr (TAN) g.ts[row] = tsc.s;
    }
#pragma unroll
    for (int j = 0; j < NCH; ++j) {
      const int c = lane + 64 * j;
      if (c < chunks) {
        store_q8<VEC>(g.q + at0 + c * VEC, v[j], sc);
        if constexpr (TAN) store_q8<VEC>(g.tq + at0 + c * VEC, w[j], tsc);
      }
    }
    t += gridDim.x * kNormWaves;
    if (t < T_rows) load(t);
  }
}

template <typename T, bool GELU, bool TAN>
hipError_t launch_rows(const RowsQ8Args& a, hipStream_t st) {
  const int chunks = a.C / Chunk<T>::VEC, NW = chunks <= 256 ? 1 : chunks <= 1024 ? 4 : 16, NCH = (chunks + 64 * NW - 1) / (64 * NW);
  constexpr long long kMaxX = 1ll << 20;  // (a dimension of a launch is limited to 2^32 - 1 threads)
  const long long wgs = NW == 1 ? (a.R + 3ll) / 4 : a.R;
  const dim3 grid((unsigned)std::min(wgs, kMaxX), !GELU && a.tx != nullptr ? 2 : 1, (unsigned)((wgs + kMaxX - 1) / kMaxX)), block(NW == 1 ? 256 : 64 * NW);
#define TVM_ROWS(N, W) \
  if (NCH == N && NW == W) hipLaunchKernelGGL((rows_q8_kernel<T, GELU, TAN, N, W>), grid, block, 0, st, a);
  TVM_ROWS(1, 1) TVM_ROWS(2, 1) TVM_ROWS(3, 1) TVM_ROWS(4, 1)
  TVM_ROWS(2, 4) TVM_ROWS(3, 4) TVM_ROWS(4, 4)
  TVM_ROWS(2, 16) TVM_ROWS(3, 16) TVM_ROWS(4, 16)
#undef TVM_ROWS
  return hipGetLastError();
}

template <typename T, bool TAN, bool GATE>
hipError_t launch_norm(const GateAdalnQ8Args& a, hipStream_t st) {
  const int chunks = a.C / Chunk<T>::VEC, NCH = (chunks + 63) / 64;
  // about 1024 workgroups in all, and every one of a batch element's the same number of rows per wave where T allows
  const int groups = (int)((a.T + (long long)kNormWaves - 1) / kNormWaves), cap = std::max(1, 1024 / a.B), passes = (groups + cap - 1) / cap;
  const dim3 grid((unsigned)((groups + passes - 1) / passes), (unsigned)a.B), block(64 * kNormWaves);
  const size_t lds = (size_t)a.C * 4 * (GATE ? 3 : 2) * (TAN ? 2 : 1);
#define TVM_NORM(N) hipLaunchKernelGGL((gate_adaln_q8_kernel<T, TAN, GATE, N>), grid, block, lds, st, a)
  if (NCH <= 1) TVM_NORM(1);
  else if (NCH == 2) TVM_NORM(2);
  else if (NCH == 3) TVM_NORM(3);
  else if (NCH == 4) TVM_NORM(4);
  else TVM_NORM(8);
#undef TVM_NORM
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rowquant(const RowsQ8Args& a, int dtype, hipStream_t st) {
  return dtype == 1 ? launch_rows<bf16, false, false>(a, st) : launch_rows<float, false, false>(a, st);
}

hipError_t launch_gelu_q8(const RowsQ8Args& a, int dtype, hipStream_t st) {
  if (dtype == 1) return a.tx != nullptr ? launch_rows<bf16, true, true>(a, st) : launch_rows<bf16, true, false>(a, st);
  return a.tx != nullptr ? launch_rows<float, true, true>(a, st) : launch_rows<float, true, false>(a, st);
}

hipError_t launch_gate_adaln_q8(const GateAdalnQ8Args& a, int dtype, hipStream_t st) {
  const bool tan = a.tx != nullptr, gate = a.h != nullptr;
  if (dtype == 1) {
    if (tan) return gate ? launch_norm<bf16, true, true>(a, st) : launch_norm<bf16, true, false>(a, st);
    return gate ? launch_norm<bf16, false, true>(a, st) : launch_norm<bf16, false, false>(a, st);
  }
  if (tan) return gate ? launch_norm<float, true, true>(a, st) : launch_norm<float, true, false>(a, st);
  return gate ? launch_norm<float, false, true>(a, st) : launch_norm<float, false, false>(a, st);
}

}  // namespace tvm
