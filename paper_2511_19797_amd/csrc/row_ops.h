// Rows of tokens, 16 bytes per thread: loads, conversions, stores, and sums over a wave (adaln.hip, rows_q8.hip).
#pragma once
#include "tvm_common.h"

namespace tvm {
namespace {

// A thread's share of a row: 16 bytes, VEC = 4 columns of float32 or 8 of bfloat16.  (Tried: 8 bytes of bfloat16 per
// thread, i.e. half the registers and twice the waves: slower, forward and backward; what counts is the number of
// bytes a compute unit has in flight.)
template <typename T>
struct alignas(16) Chunk {
  static constexpr int VEC = 16 / sizeof(T);
  T v[VEC];
};
template <typename T> using Raw = uint4;
// Nothing is done to the bytes on the way in (arithmetic right behind a load makes the compiler wait for it there
// and then): idle threads read a valid address like the others and drop their share of the sums instead.
// (Non-temporal loads, which gain 5 % in the activation kernels, lose here: forward +10 %, gate backward +40 %.)
template <typename T>
__device__ __forceinline__ Raw<T> load_raw(const T* p) {
  return *reinterpret_cast<const Raw<T>*>(p);
}
template <typename T>
__device__ __forceinline__ void widen(float (&out)[Chunk<T>::VEC], const Raw<T>& raw) {
  const Chunk<T> c = __builtin_bit_cast(Chunk<T>, raw);
#pragma unroll
  for (int e = 0; e < Chunk<T>::VEC; ++e) out[e] = (float)c.v[e];
}
// The bytes as a value the compiler knows nothing about: what was widened from them before is not kept in
// registers across this point but widened again (half the registers for bfloat16).
__device__ __forceinline__ void forget(uint4& raw) { asm volatile("" : "+v"(raw.x), "+v"(raw.y), "+v"(raw.z), "+v"(raw.w)); }
template <typename T>
__device__ __forceinline__ void store_row(T* p, const float (&in)[Chunk<T>::VEC]) {
  Chunk<T> c;
#pragma unroll
  for (int e = 0; e < Chunk<T>::VEC; ++e) c.v[e] = (T)in[e];
  *reinterpret_cast<Raw<T>*>(p) = __builtin_bit_cast(Raw<T>, c);
}
// VEC consecutive floats at a 16-byte aligned address (zeros for idle lanes), and back.
template <int VEC>
__device__ __forceinline__ void load_f32(float (&out)[VEC], const float* p, bool live) {
#pragma unroll
  for (int q = 0; q < VEC / 4; ++q) {
    const float4 v = reinterpret_cast<const float4*>(p)[q];
    out[4 * q] = live ? v.x : 0.f;
    out[4 * q + 1] = live ? v.y : 0.f;
    out[4 * q + 2] = live ? v.z : 0.f;
    out[4 * q + 3] = live ? v.w : 0.f;
  }
}
template <int VEC>
__device__ __forceinline__ void store_f32(float* p, const float (&in)[VEC]) {
#pragma unroll
  for (int q = 0; q < VEC / 4; ++q)
    reinterpret_cast<float4*>(p)[q] = make_float4(in[4 * q], in[4 * q + 1], in[4 * q + 2], in[4 * q + 3]);
}

// Sum over the wave with data-parallel-primitive moves only (no LDS traffic): a butterfly inside each row of 16
// lanes, then row 0 into row 1 and row 2 into row 3, rows 0-1 into rows 2-3; lane 63 holds the whole and is read
// into a scalar, so every lane gets the same bits.
template <int CTRL, int ROWS>
__device__ __forceinline__ float dpp_from(float x) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, ROWS, 0xf, false));
}
__device__ __forceinline__ float wave_sum_dpp(float x) {
  x += dpp_from<0xB1, 0xf>(x);   // quad_perm [1,0,3,2]
  x += dpp_from<0x4E, 0xf>(x);   // quad_perm [2,3,0,1]
  x += dpp_from<0x141, 0xf>(x);  // row_half_mirror
  x += dpp_from<0x140, 0xf>(x);  // row_mirror
  x += dpp_from<0x142, 0xa>(x);  // lane 15 of the row before, into rows 1 and 3 (the others add 0)
  x += dpp_from<0x143, 0xc>(x);  // lane 31, into rows 2 and 3
  return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), 63));
}

}  // namespace
}  // namespace tvm
