// Exchanges between the lanes of a wave that need no LDS: inside 16 lanes by DPP,
// between them by the swaps of rows (v_permlane16_swap, v_permlane32_swap).
#pragma once

#include <hip/hip_runtime.h>

namespace dora {

template <int CTRL>
__device__ __forceinline__ float dpp(float x) {
  return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), CTRL, 0xF, 0xF, false));
}

// x of the lane 16 (32) further on or back, and this lane's: in an order that
// both lanes see alike.
__device__ __forceinline__ float2 both16(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return make_float2(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float2 both32(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return make_float2(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

__device__ __forceinline__ float sum16(float x) {
  x += dpp<0xB1>(x);          // quad_perm 1,0,3,2
  x += dpp<0x4E>(x);          // quad_perm 2,3,0,1
  x += dpp<0x141>(x);         // row_half_mirror
  return x + dpp<0x140>(x);   // row_mirror
}
__device__ __forceinline__ float add16(float x) {
  const float2 b = both16(x);
  return b.x + b.y;
}
__device__ __forceinline__ float add32(float x) {
  const float2 b = both32(x);
  return b.x + b.y;
}
__device__ __forceinline__ float max16(float x) {
  const float2 b = both16(x);
  return fmaxf(b.x, b.y);
}
__device__ __forceinline__ float max32(float x) {
  const float2 b = both32(x);
  return fmaxf(b.x, b.y);
}

}  // namespace dora
