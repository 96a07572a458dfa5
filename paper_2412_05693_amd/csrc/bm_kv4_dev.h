// 4-bit rows on the device (gfx950): e2m1 codes with one power-of-two scale per
// 32 elements (include/bm_kv4.h).  gfx950 converts pairs of codes to and from
// bfloat16 or float32 in one instruction, scale included, rounding to nearest
// even and saturating; a scale of exponent 255 makes both results NaN.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "bm_lanes.h"

namespace bm {
namespace kv4 {

typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;

// Planes of a unit (include/bm_kv4.h): K rows in order; V's words of eight codes with four
// slots side by side; the scales of 64 slots side by side, in the order of a lane's slots.
template <int D>
__device__ __forceinline__ uint32_t k_word(uint32_t slot, uint32_t octet) {
  return slot * (D / 8) + octet;
}
template <int D>
__device__ __forceinline__ uint32_t v_word(uint32_t slot, uint32_t octet) {
  return (slot >> 2) * (D / 2) + octet * 4 + (slot & 3);
}
template <int D>
__device__ __forceinline__ uint32_t k_scale_at(uint32_t slot, uint32_t group) {
  return (slot >> 6) * (2 * D) + group * 64 + (slot & 15) * 4 + ((slot >> 4) & 3);
}
template <int D>
__device__ __forceinline__ uint32_t v_scale_at(uint32_t slot, uint32_t group) {
  return (slot >> 6) * (2 * D) + group * 64 + ((slot >> 2) & 3) * 16 + ((slot >> 4) & 3) * 4 + (slot & 3);
}

// 2^E as a float from its scale byte (255: an infinity, which converts to NaN)
__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }

// the scale in byte b of a word
__device__ __forceinline__ float scale_in(uint32_t word, int b) { return scale_of((word >> (8 * b)) & 0xFFu); }

// Scale byte of a group whose largest element has the float bits `top` (sign
// cleared): the exponent of the smallest power of two with top <= 6 2^E = 1.5
// 2^(E + 2).  Adding one less than the mantissa bits of 1.5 carries into the
// exponent exactly when the mantissa exceeds 1.5.
__device__ __forceinline__ uint32_t scale_byte(uint32_t top) {
  if (top >= 0x7F800000u) return 255u;
  const int e = (int)((top + 0x3FFFFFu) >> 23) - 2;
  return (uint32_t)min(max(e, 8), 252);
}

// Eight consecutive elements per lane, four lanes (a quad) per group: the
// lane's eight codes, and the group's scale byte in every lane.  The maximum
// is taken over the bits as integers, so that an infinity or NaN survives it.
__device__ __forceinline__ uint32_t quantise8(const float (&x)[8], uint32_t* byte) {
  uint32_t top = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(x[e]) & 0x7FFFFFFFu);
  top = max(top, lanes::dpp<0xB1>(top));   // quad_perm [1,0,3,2]
  top = max(top, lanes::dpp<0x4E>(top));   // quad_perm [2,3,0,1]
  const uint32_t b = scale_byte(top);
  const float s = scale_of(min(b, 252u));
  uint32_t c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, x[0], x[1], s, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[2], x[3], s, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[4], x[5], s, 2);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[6], x[7], s, 3);
  *byte = b;
  return c;
}

// eight consecutive elements of a row as floats
template <bool BF16>
__device__ __forceinline__ void load8(const void* p, float (&x)[8]) {
  if constexpr (BF16) {
    const u32x4 w = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
  } else {
    const u32x4 w0 = reinterpret_cast<const u32x4*>(p)[0], w1 = reinterpret_cast<const u32x4*>(p)[1];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[i] = __uint_as_float(w0[i]);
      x[4 + i] = __uint_as_float(w1[i]);
    }
  }
}

// Lane `octet` of D / 8 stores its part of a row that a quad per group has quantised: the
// row of slot `slot` of the unit whose planes begin at slot base0 (V's if `values`).
template <int D>
__device__ __forceinline__ void store_row(void* codes, void* scales, bool values, int64_t base0,
                                          uint32_t slot, uint32_t octet, uint32_t code, uint32_t byte) {
  const uint32_t at = values ? v_word<D>(slot, octet) : k_word<D>(slot, octet);
  (static_cast<uint32_t*>(codes) + base0 * (D / 8))[at] = code;
  if ((octet & 3) == 0) {
    const uint32_t g = octet / 4, s = values ? v_scale_at<D>(slot, g) : k_scale_at<D>(slot, g);
    (static_cast<uint8_t*>(scales) + base0 * (D / 32))[s] = (uint8_t)byte;
  }
}

// the two bfloat16 values of code pair SEL (0..3) of eight codes, as one word
template <int SEL>
__device__ __forceinline__ uint32_t bf16_pair(uint32_t codes, float s) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, SEL));
}

// eight codes as eight bfloat16 values (one 16-byte word)
__device__ __forceinline__ u32x4 bf16x8_of(uint32_t codes, float s) {
  u32x4 r;
  r[0] = bf16_pair<0>(codes, s);
  r[1] = bf16_pair<1>(codes, s);
  r[2] = bf16_pair<2>(codes, s);
  r[3] = bf16_pair<3>(codes, s);
  return r;
}

}  // namespace kv4
}  // namespace bm
