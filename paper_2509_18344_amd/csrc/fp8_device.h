// 8-bit rows: a block of 128 values as e4m3 codes and a power of two.
#pragma once

#include "kernels_rows.h"
#include "rope_device.h"

namespace subspec {

// Largest of the 16 lanes of a DPP row, in every lane (no NaN among them).
template <int CTRL>
__device__ __forceinline__ float dpp_max(float v) {
  return fmaxf(v, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xF, 0xF, false)));
}
__device__ __forceinline__ float row_max16(float v) {
  v = dpp_max<0xB1>(v);   // quad_perm [1,0,3,2]
  v = dpp_max<0x4E>(v);   // quad_perm [2,3,0,1]
  v = dpp_max<0x141>(v);  // row_half_mirror
  return dpp_max<0x140>(v);  // row_mirror
}

// The scale byte of a block whose largest finite magnitude is `top`: e + 127 for the smallest whole
// e >= -126 with top <= 448 * 2^e.  448 = 1.75 * 2^8, so e is top's exponent less 8, one more where its
// fraction exceeds 1.75.
__device__ __forceinline__ uint32_t fp8_scale_byte(float top) {
  const uint32_t b = __float_as_uint(top);
  const int s = static_cast<int>((b + 0x1FFFFFu) >> 23) - 8;  // (a fraction past 0x600000 carries into the exponent)
  return static_cast<uint32_t>(max(s, 1));
}

// Eight values as codes, 2^-e exact and its products too: one rounding, to nearest even.  What is not
// finite becomes NaN.
__device__ __forceinline__ uint2 fp8_codes(const float (&x)[8], uint32_t scale_byte) {
  const float r = __uint_as_float((254u - scale_byte) << 23);
  float v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = fabsf(x[i]) < __builtin_inff() ? x[i] * r : __builtin_nanf("");
  int lo = 0, hi = 0;
  lo = __builtin_amdgcn_cvt_pk_fp8_f32(v[0], v[1], lo, false);
  lo = __builtin_amdgcn_cvt_pk_fp8_f32(v[2], v[3], lo, true);
  hi = __builtin_amdgcn_cvt_pk_fp8_f32(v[4], v[5], hi, false);
  hi = __builtin_amdgcn_cvt_pk_fp8_f32(v[6], v[7], hi, true);
  return make_uint2(static_cast<uint32_t>(lo), static_cast<uint32_t>(hi));
}

// A block held by the 16 lanes of a DPP row, eight values each: its scale byte and this lane's codes.
__device__ __forceinline__ uint2 fp8_block(const float (&x)[8], uint32_t* scale_byte) {
  float top = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float m = fabsf(x[i]);
    top = fmaxf(top, m < __builtin_inff() ? m : 0.f);
  }
  *scale_byte = fp8_scale_byte(row_max16(top));
  return fp8_codes(x, *scale_byte);
}

// Eight codes times 2^e (given as a float) as bf16 numbers, which hold them exactly for the scale bytes of
// fp8_plain.
template <bool HI>
__device__ __forceinline__ bf16x2_t fp8_two_bf16(uint32_t w, float scale) {
  return __builtin_bit_cast(bf16x2_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, HI));
}
__device__ __forceinline__ bf16x8_t fp8_as_bf16(uint32_t lo, uint32_t hi, float scale) {
  const bf16x2_t a = fp8_two_bf16<false>(lo, scale), b = fp8_two_bf16<true>(lo, scale), c = fp8_two_bf16<false>(hi, scale),
                 d = fp8_two_bf16<true>(hi, scale);
  return bf16x8_t{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// Whether codes under this scale are normal bf16 numbers and finite: they span 2^-9 .. 448.
__device__ __forceinline__ bool fp8_plain(uint32_t scale_byte) { return scale_byte - 16u < 224u; }
// Whether codes or'ed together are all zeros, of either sign.  A block of zeros has the smallest scale, yet any power
// makes bf16 zeros of them: a row of padding must not send the rows beside it down the way of far scales, whose
// sums round elsewhere and which takes longer (64 rows, 55296 x 5120, one of them zeros: 75.3 us, 68.8 so; 66 without).
__device__ __forceinline__ bool fp8_zeros(uint32_t any) { return (any & 0x7F7F7F7Fu) == 0; }
__device__ __forceinline__ float fp8_power(uint32_t scale_byte) { return __uint_as_float(scale_byte << 23); }

// Where the scale byte of block b of row m lies.
__device__ __forceinline__ size_t fp8_scale_at(int b, int m, int M) {
  return (static_cast<size_t>(b / 4) * M + m) * 4 + b % 4;
}

}  // namespace subspec
