// Pages held in 4 bits.
//
// Values are e2m1 codes (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives) times a power of
// two that 32 of them share (its exponent + 127 in a byte, 255: all of them are NaN): 32
// channels of a key, and 32 tokens of a channel of V, which are the runs that the
// products of the attention sum over.  The shared exponent is that of the largest
// magnitude less 2, at least -127; the others are rounded to nearest, ties to even, and
// what lies above 6 becomes 6.
//
// A block holds 32 tokens of one head, K and V together, so that a wave reads
// 4352 bytes in one piece:
//   K codes   [t >> 2 & 3][t >> 4][channel >> 5][t & 3][channel & 31]   nibbles, of token t
//   V codes   [channel][token]                                         nibbles, 16 bytes a channel
//   K scales  [t >> 4][t & 3][channel >> 5][(t >> 2) & 3]   of token t
//   V scales  [channel & 15][channel >> 4]
// The codes of K lie so that 16 lanes of one of the attention's loads read runs of 64 bytes, and
// one pass of a packing wave writes 256 (token by token the loads took 16 bytes each from as many
// places: four nodes of 256 rows over 33 x 256 keys 61.3 us, 59.3 so), the scales so that a lane
// finds those of all its matrix operands side by side (attention_fp4.hip).  Tokens past a page's
// end have codes and scales of zero.
#pragma once

#include "device.h"
#include "internal.h"

namespace sc {

constexpr uint32_t kFp4V = 2048, kFp4KScale = 4096, kFp4VScale = 4224;  // offsets in a block

// The scale byte of a group whose largest magnitude has these bits (of an fp32 number).
__device__ __forceinline__ uint32_t fp4_scale(uint32_t top) {
  const uint32_t e = top >> 23;
  return e == 255u ? 255u : e > 2u ? e - 2u : 0u;
}

// Bits of the larger magnitude of two bf16 values in a word, as of an fp32 number.
__device__ __forceinline__ uint32_t bf16x2_top(uint32_t w) {
  const uint32_t lo = w << 16 & 0x7fffffffu, hi = w & 0x7fff0000u;
  return lo > hi ? lo : hi;
}

__device__ __forceinline__ uint32_t umax(uint32_t a, uint32_t b) { return a > b ? a : b; }

// The larger of the values of four neighbouring lanes.
__device__ __forceinline__ uint32_t quad_max(uint32_t x) {
  x = umax(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0xb1, 0xf, 0xf, true));  // lanes 1 0 3 2
  return umax(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x4e, 0xf, 0xf, true));  // lanes 2 3 0 1
}

// Eight bf16 values as codes.
__device__ __forceinline__ uint32_t fp4_codes(const u32x4& v, uint32_t scale) {
  const float s = __uint_as_float(scale << 23);  // of this only the exponent counts
  const uint32_t w0 = v[0], w1 = v[1], w2 = v[2], w3 = v[3];
  uint32_t c = 0;
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, w0), s, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, w1), s, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, w2), s, 2);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, w3), s, 3);
  return scale == 255u ? 0u : c;
}

// Eight codes as bf16 values (exact: two significant bits; 6 times the largest power
// that bf16 values lead to is finite).
__device__ __forceinline__ u32x4 fp4_values(uint32_t c, uint32_t scale) {
  const float s = __uint_as_float(scale << 23);
  u32x4 v;
  v[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 0));
  v[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 1));
  v[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 2));
  v[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 3));
  return v;
}

}  // namespace sc
