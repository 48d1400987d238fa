// Rows of E2M1 codes with an E8M0 scale for every 32 elements (BAKLAVA_MXFP4): rounding, and values of codes.
//
// A value is code * 2^(byte - 127); with the scales that rounding gives (2^-125 .. 2^125) every value is a normal bf16 number
// or zero, so codes become bf16 operands of a matrix product without a second rounding, two per instruction.
#ifndef BAKLAVA_MXFP4_H
#define BAKLAVA_MXFP4_H

#include "common.h"

namespace baklava {

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));

// The scale as the conversion instructions take it (they use a float's exponent field; 255 makes everything NaN).
__device__ __forceinline__ float mx_scale(uint32_t byte) { return __uint_as_float(byte << 23); }

// Eight codes (element i in bits 4 i .. 4 i + 3) as four pairs of bf16.
__device__ __forceinline__ uint4 mx_values(uint32_t codes, float scale) {
  return make_uint4(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0)),
                    __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1)),
                    __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2)),
                    __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3)));
}

// The scale byte of 32 elements whose largest magnitude has these bf16 bits (sign cleared): 2^e, e = floor(log2 a) - 2, one
// more where a > 1.75 * 2^floor(log2 a), which leaves magnitudes of up to 7 units to the code of 6 and makes the largest of
// the others 4; 0.112 of N(0, 1) values are lost (2-norm), 0.115 without that step.  bf16 bits order like magnitudes, and
// exponent and mantissa lie next to each other: adding 31 carries into the exponent exactly for mantissas above 1.75 (96).
__device__ __forceinline__ uint32_t mx_scale_byte(uint32_t top) {
  if (top >= 0x7f80u) return 255;  // infinite or NaN
  const int e = (int)((top + 31) >> 7) - 2;  // (subnormals: exponent field 0, below the clamp either way)
  return (uint32_t)min(max(e, 2), 252);
}

// Codes of eight bf16 elements, in the order above.  The instruction divides by the scale, rounds to the nearest code, ties
// to even, and saturates; of a block that is not finite the scale says everything, and codes are 0.
__device__ __forceinline__ uint32_t mx_codes(uint4 x, uint32_t byte) {
  if (byte == 255) return 0;
  const float s = mx_scale(byte);
  uint32_t c = 0;
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2_t, x.x), s, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2_t, x.y), s, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2_t, x.z), s, 2);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2_t, x.w), s, 3);
  return c;
}

// Largest magnitude (bf16 bits) of eight elements, and over the four neighbouring lanes that hold the 32 of a scale.
__device__ __forceinline__ uint32_t mx_top(uint4 x) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t w = i == 0 ? x.x : i == 1 ? x.y : i == 2 ? x.z : x.w;
    m = max(m, max(w & 0x7fffu, w >> 16 & 0x7fffu));
  }
  m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0xb1, 0xf, 0xf, true));  // quad_perm:[1,0,3,2]
  return max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x4e, 0xf, 0xf, true));  // quad_perm:[2,3,0,1]
}

// One row of D bf16 elements, 8 per lane of D / 8 neighbouring lanes (`piece` of them this lane's), rounded into row `row` of
// a plane; value = 1 for V.  All lanes of a quad take part.
template <int D>
__device__ __forceinline__ void mx_store(uint4 x, int piece, void* plane, uint8_t* kv_scale, int64_t row, int value) {
  const uint32_t byte = mx_scale_byte(mx_top(x));
  reinterpret_cast<uint32_t*>(plane)[row * (D / 8) + piece] = mx_codes(x, byte);
  if (piece % 4 == 0) kv_scale[row * (D / 16) + value * (D / 32) + piece / 4] = (uint8_t)byte;
}

// The scales of a row's key and value from those of its 32 elements each lane shares (the bytes of a quad are equal): words of
// D / 32 bytes, in every lane of the row.
template <int D>
__device__ __forceinline__ uint2 mx_row_scales(uint32_t byte_k, uint32_t byte_v, int piece) {
  const int shift = 8 * (piece / 4);
  int k = (int)(byte_k << shift), v = (int)(byte_v << shift);
  if (D == 128) {  // four quads of a row of 16 lanes
    k |= __builtin_amdgcn_update_dpp(0, k, 0x124, 0xf, 0xf, true);  // row_ror:4
    v |= __builtin_amdgcn_update_dpp(0, v, 0x124, 0xf, 0xf, true);
    k |= __builtin_amdgcn_update_dpp(0, k, 0x128, 0xf, 0xf, true);  // row_ror:8
    v |= __builtin_amdgcn_update_dpp(0, v, 0x128, 0xf, 0xf, true);
  } else {  // two of eight
    k |= __builtin_amdgcn_update_dpp(0, k, 0x141, 0xf, 0xf, true);  // row_half_mirror
    v |= __builtin_amdgcn_update_dpp(0, v, 0x141, 0xf, 0xf, true);
  }
  return make_uint2((uint32_t)k, (uint32_t)v);
}

// A row mx_store has written, back.
template <int D>
__device__ __forceinline__ uint4 mx_load(int piece, const void* plane, const uint8_t* kv_scale, int64_t row, int value) {
  return mx_values(reinterpret_cast<const uint32_t*>(plane)[row * (D / 8) + piece],
                   mx_scale(kv_scale[row * (D / 16) + value * (D / 32) + piece / 4]));
}

}  // namespace baklava
#endif
