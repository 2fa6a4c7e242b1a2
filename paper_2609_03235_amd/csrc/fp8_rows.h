// Rows of a cache in 8 bits (gfx950): e4m3 numbers (4 exponent bits with bias 7, 3 of mantissa, the largest 448, no
// infinities) times a power of two per row, an e8m0 code c for 2^(c - 127).
//
// A row's power is the smallest with which its largest finite value is at most 448, and at least 2^kMinRowExp. A power
// of two makes both ways exact but for the one rounding to four bits of mantissa: x / 2^e is exact in fp32, and a
// number times 2^e is exact in bf16, so that the hardware's conversions with a scale, one instruction for two numbers,
// give the value itself. (Two ends apart: fp32 values from 1.9375 * 2^127 on round to 256 times 2^120, past the largest
// number of bf16 and fp32; and of codes 0 to 2, which no store here writes, bf16's subnormals hold multiples of 2^-133
// only.) The rounding of e4m3 is relative (half a step is 2^-4 of the value, down to 2^-6), so a scale other than a
// power of two, or one of fewer columns, would not make it smaller.
#pragma once

#include "mfma_frag.h"

namespace sgdkv {

struct E4m3 {
  uint8_t bits;
};

// Keeps the smallest number of a row, 2^-9 times its power, a normal one in fp32 and bf16.
constexpr int kMinRowExp = -110;

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

// A code of a row, through a buffer.
__device__ __forceinline__ uint32_t ld8(rsrc_t r, uint32_t byte_off) {
  return __builtin_amdgcn_raw_buffer_load_b8(r, (int)byte_off, 0, 0);
}

// The word that the conversions below take a code's power from. Its exponent bits alone count: 0 there is 2^-127, and
// 255 makes every number NaN.
__device__ __forceinline__ float conversion_scale(uint32_t code) { return __uint_as_float(code << 23); }
// A code's power as a factor: for 0 the subnormal 2^-127, for 255 an infinity.
__device__ __forceinline__ float power_of(uint32_t code) { return __uint_as_float(max(code << 23, 0x00400000u)); }

// Numbers 2 * HI and 2 * HI + 1 of a word, times a power of two.
template <int HI>
__device__ __forceinline__ uint32_t e4m3_to_bf16(uint32_t w, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, HI));
}
// Eight numbers (two words) as an operand.
__device__ __forceinline__ Frag<__bf16> widen_piece(uint32_t w0, uint32_t w1, float scale) {
  return {u32x4{e4m3_to_bf16<0>(w0, scale), e4m3_to_bf16<1>(w0, scale), e4m3_to_bf16<0>(w1, scale),
                e4m3_to_bf16<1>(w1, scale)}};
}

// |x| where it counts for the row's power.
__device__ __forceinline__ uint32_t finite_size(float x) {
  const uint32_t b = __float_as_uint(x) & 0x7FFFFFFFu;
  return b < 0x7F800000u ? b : 0u;
}
// The code of a row whose largest size is `size` (bits of a finite fp32 number): 448 is 1.75 * 2^8.
__device__ __forceinline__ int row_code(uint32_t size) {
  const int e = (int)(size >> 23) - 127 - 8 + ((size & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return max(e, kMinRowExp) + 127;
}
// 2^-e for a code.
__device__ __forceinline__ float inverse_power(int code) { return __uint_as_float((uint32_t)(254 - code) << 23); }
// Four values, already divided by the row's power, to nearest even; infinities and NaN become NaN.
__device__ __forceinline__ uint32_t to_e4m3(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}

}  // namespace sgdkv
