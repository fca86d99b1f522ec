// fp8_device.hpp -- device building blocks of the operators in 8-bit floating point.
//
// The format: 128 consecutive values of a row (the last block of a row may be short), or a tile of 128 x 128 values,
// share a power of two 2^e, the least one with max|x| <= 448 * 2^e and e >= -127; a value is held as x / 2^e rounded to
// e4m3 (half to even), the block's scale as the byte e + 127.  Scaling by a power of two is exact, so a code
// depends on nothing but the value and its block, and the matrix instructions take the byte as it is.  A block
// with an infinity or a NaN has scale byte 255 and NaN codes, and stands for NaN throughout.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "dense_device.hpp"

namespace rdfft {

constexpr int kFp8Block = 128;                 // values that share a scale
constexpr int kFp8Lanes = kFp8Block / kVec;    // lanes that hold them
constexpr uint32_t kFp8NaNs = 0x7f7f7f7fu;

// the maximum over each aligned group of 16 lanes (a DPP row)
__device__ __forceinline__ uint32_t row_max(uint32_t v) {
  v = quad_max(v);
  v = max(v, dpp_u32<0x141>(v));  // row_half_mirror: the other quad of eight lanes
  return max(v, dpp_u32<0x140>(v));  // row_mirror: the other eight
}

// Scale byte from the largest |x|, as bits: with |x| = f * 2^k, 1 <= f < 2, e is k - 8 while f <= 448/256, whose
// fraction is 0x600000; more carries into the exponent field.
__device__ __forceinline__ int fp8_scale_byte(uint32_t amax) {
  const int s = (int)((amax + 0x1fffffu) >> 23) - 8;
  return amax >= 0x7f800000u ? kCkNaN : max(s, 0);
}
// What the conversions take for a scale byte: the float 2^e, of which they look at the exponent alone (so 0 is 2^-127).
__device__ __forceinline__ float fp8_scale(int s) { return __uint_as_float((uint32_t)s << 23); }

// Four codes of x / 2^e, half to even (at most 448, so nothing saturates): of floats, or of two pairs of 16-bit values.
__device__ __forceinline__ uint32_t fp8_word(float a, float b, float c, float d, float scale) {
  typedef short s16x2 __attribute__((ext_vector_type(2)));
  s16x2 r = {0, 0};
  r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, a, b, scale, false);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, c, d, scale, true);
  return __builtin_bit_cast(uint32_t, r);
}
template <class E>
__device__ __forceinline__ uint32_t fp8_word(uint32_t ab, uint32_t cd, float scale) {
  typedef short s16x2 __attribute__((ext_vector_type(2)));
  typedef __bf16 b16x2 __attribute__((ext_vector_type(2)));
  typedef _Float16 h16x2 __attribute__((ext_vector_type(2)));
  s16x2 r = {0, 0};
  if constexpr (E::kId == ElemBF16::kId) {
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, __builtin_bit_cast(b16x2, ab), scale, false);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, __builtin_bit_cast(b16x2, cd), scale, true);
  } else {
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(r, __builtin_bit_cast(h16x2, ab), scale, false);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(r, __builtin_bit_cast(h16x2, cd), scale, true);
  }
  return __builtin_bit_cast(uint32_t, r);
}
// Eight codes; NaN for a block that is not finite.
__device__ __forceinline__ Bytes8 fp8_encode(const float* v, int s) {
  const float scale = fp8_scale(s);
  const Bytes8 r = {{fp8_word(v[0], v[1], v[2], v[3], scale), fp8_word(v[4], v[5], v[6], v[7], scale)}};
  return s == kCkNaN ? Bytes8{{kFp8NaNs, kFp8NaNs}} : r;
}

// Eight values.  Of a value within 1/32 of the type's largest number M the code can stand for the power of two past M: it
// stands for +-M, so what was finite comes back finite (Elem*::kMost, kPast).  2^128 is code 256 of byte 247, which is what
// quantize leaves, and as well 128 of byte 248 and so on.
template <class E>
__device__ __forceinline__ void fp8_decode(const Bytes8& r, int s, float* v) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  const float scale = ck_scale(s);
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)r.w[h], false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)r.w[h], true);
    v[4 * h] = a[0];
    v[4 * h + 1] = a[1];
    v[4 * h + 2] = b[0];
    v[4 * h + 3] = b[1];
  }
#pragma unroll
  for (int i = 0; i < kVec; ++i) {
    const float code = v[i];
    v[i] = code * scale;
    if (E::kId == ElemF16::kId) v[i] = fabsf(v[i]) == 65536.f ? copysignf(E::kMost, v[i]) : v[i];
    else if (s >= 247 && s != kCkNaN)
      v[i] = fabsf(code) == __uint_as_float((uint32_t)(127 + 255 - s) << 23) ? copysignf(E::kMost, code) : v[i];
  }
}

// Eight codes of a row that has n; nothing past its end is written.
__device__ __forceinline__ void write_bytes(uint8_t* row, int64_t i0, int64_t n, const Bytes8& c) {
  write_codes(reinterpret_cast<int8_t*>(row), i0, n, c);
}

// The 8-bit form of eight values a lane, 16 consecutive lanes to a block, i0 a multiple of eight; the values past the
// row's end are zeros.  Rows of codes start at multiples of eight bytes.
__device__ __forceinline__ void write_fp8(uint8_t* codes, uint8_t* scales, int64_t i0, int64_t n, const float* v) {
  const int s = fp8_scale_byte(row_max(max_bits8(v)));
  if (i0 >= n) return;
  write_bytes(codes, i0, n, fp8_encode(v, s));
  if (i0 % kFp8Block == 0) scales[i0 / kFp8Block] = (uint8_t)s;
}

}  // namespace rdfft
