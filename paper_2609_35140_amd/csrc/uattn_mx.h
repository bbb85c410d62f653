// The format of a KV cache held in 8 or 4 bits, and its conversions.
//
// A row of head_dim elements is cut into blocks of 32.  A block has one scale
// 2^e, stored as the byte e + 127, and one code an element:
//   8 bits  sign, 4 exponent bits (bias 7), 3 mantissa bits, at most 448
//   4 bits  sign, 2 exponent bits (bias 1), 1 mantissa bit, at most 6; two to a
//           byte, the even element in the low half
// (the E4M3 and E2M1 elements with E8M0 scales of the OCP microscaling formats).
// With a the largest magnitude of the block and `most` 448 or 6, e is the smallest
// whole number, -100 at least, with a <= most * 2^e -- so no element is clipped --
// and an element's code is the nearest to x * 2^-e, ties to the even code.  A block
// with a >= 2^127 (rounding up could leave bf16's range), an infinity or a NaN gets
// the scale byte 255, which reads as NaN in every element.
//
// Every code times every scale that a write makes (bytes 27 to 246 in 8 bits, 27 to 252
// in 4) is a bf16 number, and the gfx950 conversions below give exactly it (and exactly
// the nearest code): tested for all codes with all of these bytes, and for all bf16
// values.  So reading back rounds nothing, and attention over a cache has the bits of
// attention over those bf16 values.  The floor of e keeps every value a normal number:
// the smallest is 2^-109 in 8 bits and 2^-101 in 4, and half of it and less becomes zero.
#pragma once

#include "uattn_numerics.h"

namespace uattn {

constexpr int kMxBlock = 32;     // elements to a scale
constexpr int kMxLeast = 27;     // scale byte of 2^-100
constexpr int kMxNan = 255;      // scale byte of a block that reads as NaN

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short s16x2 __attribute__((ext_vector_type(2)));

// The scale byte as the fp32 operand of the conversions: its exponent field
// (255: infinity, which they answer with NaN; 0: read as 2^-127).
__device__ __forceinline__ float mx_scale(uint32_t byte) { return __uint_as_float(byte << 23); }
// Byte i of a word of scale bytes, the same way.
template <int i>
__device__ __forceinline__ float mx_scale_of(uint32_t word) {
  constexpr int up = 23 - 8 * i;
  return __uint_as_float((up >= 0 ? word << (up & 31) : word >> (-up & 31)) & 0x7F800000u);
}

// Scale byte of a block from the largest magnitude of its elements as bf16 bits
// without sign: e is the exponent less most's, one more where the mantissa is above
// most's (the sum carries).
template <int Bits>
__device__ __forceinline__ uint32_t mx_scale_byte(uint32_t mag) {
  constexpr uint32_t carry = Bits == 8 ? 0x7F - 0x60 : 0x7F - 0x40;  // 448 = 1.75 * 2^8, 6 = 1.5 * 2^2
  constexpr int down = Bits == 8 ? 8 : 2;
  const int byte = max(static_cast<int>((mag + carry) >> 7) - down, kMxLeast);
  return mag >= 0x7F00u ? kMxNan : byte;
}

// Codes of eight elements: one word (4 bits) or two (8).
template <int Bits>
struct MxWords {
  static constexpr int kCount = Bits / 4;
  uint32_t w[kCount];
};

template <int Bits>
__device__ __forceinline__ bf16x8 mx_decode8(const uint32_t* w, float scale) {
  bf16x2 p[4];
  if constexpr (Bits == 4) {
    p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[0], scale, 0);
    p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[0], scale, 1);
    p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[0], scale, 2);
    p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[0], scale, 3);
  } else {
    p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[0], scale, false);
    p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[0], scale, true);
    p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[1], scale, false);
    p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[1], scale, true);
  }
  return __builtin_bit_cast(bf16x8, p);
}

// (By value: __builtin_bit_cast of a vector's element takes the vector's first one.)
__device__ __forceinline__ bf16x2 mx_pair(uint32_t w) { return __builtin_bit_cast(bf16x2, w); }

template <int Bits>
__device__ __forceinline__ MxWords<Bits> mx_encode8(const u32x4& x, float scale) {
  MxWords<Bits> r;
  if constexpr (Bits == 4) {
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, mx_pair(x[0]), scale, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, mx_pair(x[1]), scale, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, mx_pair(x[2]), scale, 2);
    r.w[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, mx_pair(x[3]), scale, 3);
  } else {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      s16x2 p = {0, 0};
      p = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(p, mx_pair(x[2 * i]), scale, false);
      p = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(p, mx_pair(x[2 * i + 1]), scale, true);
      r.w[i] = __builtin_bit_cast(uint32_t, p);
    }
  }
  return r;
}

// The larger magnitudes of the two halves of a and b, as bits.
__device__ __forceinline__ uint32_t mx_max_mag(uint32_t a, uint32_t b) {
  typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
  const u16x2 r = __builtin_elementwise_max(__builtin_bit_cast(u16x2, a & 0x7FFF7FFFu), __builtin_bit_cast(u16x2, b & 0x7FFF7FFFu));
  return __builtin_bit_cast(uint32_t, r);
}

}  // namespace uattn
