// Blocks of 128 values in 8-bit floating point with a power-of-two scale: shared by the quantiser, the product and the
// optimizer with 8-bit states.
#pragma once
#include "common.h"

namespace t5mi {

constexpr int kBlock = 128;

// Exponent of the largest finite value 1.75 * 2^top of a type.
template <int Q> constexpr int fp8_top = Q == T5_E4M3 ? 8 : 15;

// e of the block's scale 2^e: the smallest e >= -127 with amax / 2^e <= 1.75 * 2^TOP, 0 for a block of zeros.  amax_bits: the
// bits of the largest finite |x| (they are ordered as the values are).  A subnormal amax has e = -127 either way.
template <int Q>
__device__ __forceinline__ int block_exponent(uint32_t amax_bits) {
  const int e = (int)(amax_bits >> 23) - 127 - fp8_top<Q> + ((amax_bits & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return amax_bits == 0 ? 0 : max(e, -127);
}
// 2^-e for such an e (-127 <= e <= 120): always a normal number, so that x * 2^-e is exact or below the type's range.
__device__ __forceinline__ float block_inverse(int e) { return __uint_as_float((uint32_t)(127 - e) << 23); }
// 2^(byte - 127)
__device__ __forceinline__ float scale_value(uint32_t byte) {
  return __uint_as_float(byte == 0 ? 0x400000u : byte == 255 ? 0x7FC00000u : byte << 23);
}

// |x| as bits, 0 where x is not finite
__device__ __forceinline__ uint32_t finite_bits(float x) {
  const uint32_t b = __float_as_uint(x) & 0x7FFFFFFFu;
  return b < 0x7F800000u ? b : 0u;
}

// Four codes, rounded to nearest even.  Finite inputs are within the type's range by the choice of the scale.
template <int Q>
__device__ __forceinline__ uint32_t pack_fp8x4(float a, float b, float c, float d) {
  int r = 0;
  if constexpr (Q == T5_E4M3) {
    r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, r, false);
    r = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
  } else {
    r = __builtin_amdgcn_cvt_pk_bf8_f32(a, b, r, false);
    r = __builtin_amdgcn_cvt_pk_bf8_f32(c, d, r, true);
  }
  return (uint32_t)r;
}

// Largest of v over the 16 lanes that hold a block's pieces of 8 (lanes 16 i .. 16 i + 15): exchanges within quads, then
// mirror images within 8 and 16 lanes.
template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, true);
}
__device__ __forceinline__ uint32_t max16(uint32_t v) {
  v = max(v, dpp<0xB1>(v));
  v = max(v, dpp<0x4E>(v));
  v = max(v, dpp<0x141>(v));
  return max(v, dpp<0x140>(v));
}

}  // namespace t5mi
