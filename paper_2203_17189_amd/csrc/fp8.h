// Blocks of 128 values in 8-bit floating point with a power-of-two scale: shared by the quantiser, the product and the
// optimizer with 8-bit states.
#pragma once
#include "common.h"

namespace t5mi {

constexpr int kBlock = 128;

// Whether the quantiser reads its matrix in whole pieces of 16 bytes, and whether it reads the eight elements from column c
// (a multiple of 8) of a row as such: those past the row's end too (and drops them) where another row follows.  Rows of four
// float32 would take in the next row with it, and of a last one more than its columns; longer ones end at most four elements
// into a row of more.
inline bool quant_in_pieces(const void* x, int64_t ld, int size) {
  return ((uintptr_t)x & 15) == 0 && ld * size % 16 == 0 && ld >= 8;
}
__host__ __device__ __forceinline__ bool quant_whole_piece(int c, int cols, bool more) { return c + 8 <= cols || (more && c < cols); }

// Exponent of the largest finite value 1.75 * 2^top of a type.
template <int Q> constexpr int fp8_top = Q == T5_E4M3 ? 8 : 15;

// e of the block's scale 2^e: the smallest e >= -127 with amax / 2^e <= 1.75 * 2^TOP, 0 for a block of zeros.  amax_bits: the
// bits of the largest finite |x| (they are ordered as the values are).  A subnormal amax has e = -127 either way.
template <int Q>
__device__ __forceinline__ int block_exponent(uint32_t amax_bits) {
  const int e = (int)(amax_bits >> 23) - 127 - fp8_top<Q> + ((amax_bits & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return amax_bits == 0 ? 0 : max(e, -127);
}
// 2^(byte - 127)
__device__ __forceinline__ float scale_value(uint32_t byte) {
  return __uint_as_float(byte == 0 ? 0x400000u : byte == 255 ? 0x7FC00000u : byte << 23);
}

// The same as the conversions from codes take it: by its exponent alone, of which 0 is 2^-127 and 255 makes NaN.
__device__ __forceinline__ float scale_operand8(uint32_t byte) { return __uint_as_float(byte << 23); }

// |x| as bits, 0 where x is not finite
__device__ __forceinline__ uint32_t finite_bits(float x) {
  const uint32_t b = __float_as_uint(x) & 0x7FFFFFFFu;
  return b < 0x7F800000u ? b : 0u;
}

// The scale 2^e of a block as the conversions take it (e = byte - 127; its exponent alone counts, 2^-127 has an exponent of 0).
__device__ __forceinline__ float scale_of(int e) { return __uint_as_float(max((uint32_t)(e + 127) << 23, 0x400000u)); }

typedef __attribute__((ext_vector_type(2))) short s16x2;

// Codes of a / scale .. d / scale, rounded to nearest even.  Finite inputs are within the type's range by the choice of the
// scale; infinities become NaN in e4m3 and stay in e5m2, NaN stays.
template <int Q>
__device__ __forceinline__ uint32_t pack_fp8x4(float a, float b, float c, float d, float scale) {
  s16x2 r = {0, 0};
  if constexpr (Q == T5_E4M3) {
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, a, b, scale, false);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, c, d, scale, true);
  } else {
    r = __builtin_amdgcn_cvt_scalef32_pk_bf8_f32(r, a, b, scale, false);
    r = __builtin_amdgcn_cvt_scalef32_pk_bf8_f32(r, c, d, scale, true);
  }
  return __builtin_bit_cast(uint32_t, r);
}
// The same of two pairs of bfloat16.
template <int Q>
__device__ __forceinline__ uint32_t pack_fp8x4(uint32_t ab, uint32_t cd, float scale) {
  s16x2 r = {0, 0};
  const bf16x2 lo = __builtin_bit_cast(bf16x2, ab), hi = __builtin_bit_cast(bf16x2, cd);
  if constexpr (Q == T5_E4M3) {
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, lo, scale, false);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, hi, scale, true);
  } else {
    r = __builtin_amdgcn_cvt_scalef32_pk_bf8_bf16(r, lo, scale, false);
    r = __builtin_amdgcn_cvt_scalef32_pk_bf8_bf16(r, hi, scale, true);
  }
  return __builtin_bit_cast(uint32_t, r);
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
