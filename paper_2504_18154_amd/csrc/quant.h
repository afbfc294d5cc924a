// The caches of ecoserve_cache: codes of 8 bits with a scale per (token, head), or the layout's own bf16.
//
// A row of D elements with largest magnitude A is held as codes c of x ~ c 2^e, e the smallest integer >= -126 with A <= M 2^e (M = 127 for int8, 448 for
// e4m3), and the byte e + 127: powers of two, so that coding is one rounding, decoding is none (a code has 4 or 7 bits, bf16 8), and the scales are the
// operands that the conversions of gfx950 take.
#pragma once

#include "common.h"

namespace eco {

constexpr int kNative = ECOSERVE_CACHE_LAYOUT, kInt8 = ECOSERVE_CACHE_INT8, kE4m3 = ECOSERVE_CACHE_E4M3;
constexpr int kScaleBytes = 2 * kBlockSize;  // of a (block, head): 16 of the keys, 16 of the values
constexpr uint32_t kBadScale = 255;         // scale byte of a row that holds a NaN or an infinity (codes 0)

inline bool quant_format_ok(int32_t format) { return format == kNative || format == kInt8 || format == kE4m3; }

}  // namespace eco

#if defined(__HIPCC__)
namespace eco {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

template <int F>
struct Cached {
  static constexpr int kBytes = F == kNative ? 2 : 1;   // of an element
  static constexpr int kUnit = F == kNative ? 8 : 16;   // channels of a 16-byte unit of K
};

// 2^(b - 127) of byte i of a word of scale bytes; 255 gives infinity, whose product with a code of 0 is NaN.
template <int I>
__device__ __forceinline__ float scale_of(uint32_t w) {
  const uint32_t at = I == 3 ? w >> 1 : w << (I == 3 ? 0 : 23 - 8 * I);
  return __uint_as_float(at & 0x7f800000u);
}
__device__ __forceinline__ float scale_of_byte(uint32_t b) { return __uint_as_float(b << 23); }

// Codes 0 .. 3 of a word as fp32.
template <int F, int I>
__device__ __forceinline__ float code_value(uint32_t w) {
  if constexpr (F == kInt8) return (float)(int8_t)(w >> (8 * I));
  else return __builtin_amdgcn_cvt_f32_fp8((int)w, I);
}
// Codes 0 and 1, or 2 and 3, of a word of e4m3 as bf16, exactly, times a power of two.
__device__ __forceinline__ uint32_t two_codes(uint32_t w, float scale, bool upper) {
  return upper ? __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, true))
               : __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, false));
}
// Four codes as bf16, exactly, times a power of two.
template <int F>
__device__ __forceinline__ u32x2 codes_to_bf16(uint32_t w, float scale) {
  if constexpr (F == kE4m3) {
    return u32x2{two_codes(w, scale, false), two_codes(w, scale, true)};
  } else {
    return u32x2{pack_bf16x2(code_value<F, 0>(w) * scale, code_value<F, 1>(w) * scale), pack_bf16x2(code_value<F, 2>(w) * scale, code_value<F, 3>(w) * scale)};
  }
}
template <int F>
__device__ __forceinline__ bf16x8 codes_to_bf16x8(uint32_t a, uint32_t b, float scale) {
  const u32x2 x = codes_to_bf16<F>(a, scale), y = codes_to_bf16<F>(b, scale);
  return __builtin_bit_cast(bf16x8, u32x4{x[0], x[1], y[0], y[1]});
}

// A pair of weights as two bf16 numbers each, 16 bits in all: the first ones, and what they leave.  kOpen: values may be infinite, and the product of an infinity with a part of 0, or a
// sum of infinities of either sign, would be NaN: no part is negative then, and the second one is not 0 (of weights from 2^-66 on).
template <bool kOpen>
__device__ __forceinline__ uint32_t first_parts(float a, float b) {
  return kOpen ? __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u) : pack_bf16x2(a, b);
}
template <bool kOpen>
__device__ __forceinline__ uint32_t second_parts(float a, float b, uint32_t first) {
  const float s = a - __uint_as_float(first << 16), t = b - __uint_as_float(first & 0xffff0000u);
  return kOpen ? pack_bf16x2(__builtin_fmaf(a, 0x1p-60f, s), __builtin_fmaf(b, 0x1p-60f, t)) : pack_bf16x2(s, t);
}

// The scale byte of a row with largest magnitude `most` (NaN and infinity: 255), and the factor 2^-e of its codes.
template <int F>
__device__ __forceinline__ uint32_t scale_byte(float most) {
  if (!(most < INFINITY)) return kBadScale;
  const uint32_t u = __float_as_uint(most);
  // most = f 2^x with f in [1, 2): M = 1.984375 2^6 or 1.75 2^8
  const int top = F == kInt8 ? 6 : 8;
  const uint32_t edge = F == kInt8 ? 0x7e0000u : 0x600000u;
  const int e = (int)(u >> 23) - 127 - top + ((u & 0x7fffffu) > edge ? 1 : 0);
  return (uint32_t)(max(e, -126) + 127);
}
__device__ __forceinline__ float inverse_scale(uint32_t byte) { return ldexpf(1.f, 127 - (int)byte); }

// Four values, times the inverse scale, as codes: one rounding to nearest even each.
template <int F>
__device__ __forceinline__ uint32_t to_codes(float a, float b, float c, float d) {
  if constexpr (F == kE4m3) {
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false), true);
  } else {
    // (1.5 2^23 and a whole number of up to 2^22 have the number in their low bits; the sum is the rounding)
    constexpr float kWhole = 12582912.f;
    const uint32_t x = __float_as_uint(a + kWhole), y = __float_as_uint(b + kWhole), z = __float_as_uint(c + kWhole), w = __float_as_uint(d + kWhole);
    return __builtin_amdgcn_perm(__builtin_amdgcn_perm(w, z, 0x0c0c0400u), __builtin_amdgcn_perm(y, x, 0x0c0c0400u), 0x05040100u);
  }
}

}  // namespace eco
#endif
