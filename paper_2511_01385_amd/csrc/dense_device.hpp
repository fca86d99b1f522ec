// dense_device.hpp -- device building blocks of the operators around the block-circulant layer:
// rows of any element alignment in groups of eight, wave sums, and the 8-bit checkpoint format.
//
// The 8-bit format: 32 consecutive values of a row (the last block of a row may be short) share
// a power of two 2^e, the least one with max|x| <= 127 * 2^e and e >= -127; a value is held as
// rint(x / 2^e) in int8, the block's scale as the byte e + 127.  Scaling by a power of two is exact, so
// the code of a value depends on nothing but the value and its block, and code * 2^e fits in
// bfloat16.  A block with an infinity or a NaN has scale byte 255 and stands for NaN throughout.
// Code 64 of a block whose largest |x| is within 1 % of the type's largest number would stand for the power of two past
// that number: it stands for the number itself (ck_decode), so what was finite comes back finite.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "fft_device.hpp"

namespace rdfft {

constexpr int kVec = 8;         // values a thread loads and stores together
constexpr int kCkBlock = 32;    // values that share a scale
constexpr int kCkLanes = kCkBlock / kVec;
constexpr int kCkNaN = 255;     // scale byte of a block that is not finite

// 16 and 8 bytes at any element's alignment (the memory instructions take it as it comes)
struct __attribute__((packed, aligned(1))) Bytes16 {
  uint32_t w[4];
};
struct __attribute__((packed, aligned(1))) Bytes8 {
  uint32_t w[2];
};

// Storage types: eight values in memory <-> eight floats.  Raw is what a load leaves in
// registers, so that loads can be issued ahead of the arithmetic.
struct ElemF32 {
  using T = float;
  static constexpr int kId = 0;
  // the largest finite number, the step of a block that reaches it, and 64 such steps, as floats
  static constexpr float kMost = 0x1.fffffep127f, kLastStep = 0x1p122f, kPast = __builtin_inff();
  struct Raw {
    Bytes16 a, b;
  };
  __device__ __forceinline__ static Raw load(const T* p) {
    return {*reinterpret_cast<const Bytes16*>(p), *reinterpret_cast<const Bytes16*>(p + 4)};
  }
  __device__ __forceinline__ static void widen(const Raw& r, float* v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[i] = __uint_as_float(r.a.w[i]);
      v[4 + i] = __uint_as_float(r.b.w[i]);
    }
  }
  __device__ __forceinline__ static void store(T* p, const float* v) {
    Bytes16 a, b;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      a.w[i] = __float_as_uint(v[i]);
      b.w[i] = __float_as_uint(v[4 + i]);
    }
    *reinterpret_cast<Bytes16*>(p) = a;
    *reinterpret_cast<Bytes16*>(p + 4) = b;
  }
  __device__ __forceinline__ static float get(const T* p) { return *p; }
  __device__ __forceinline__ static void put(T* p, float v) { *p = v; }
};

template <int ID, float2 (*WIDEN)(uint32_t), uint32_t (*NARROW)(float2)>
struct Elem16 {
  using T = uint16_t;
  static constexpr int kId = ID;
  static constexpr bool kHalf = ID == 2;
  static constexpr float kMost = kHalf ? 65504.f : 0x1.fep127f, kLastStep = kHalf ? 0x1p10f : 0x1p122f,
                         kPast = kHalf ? 65536.f : __builtin_inff();
  using Raw = Bytes16;
  __device__ __forceinline__ static Raw load(const T* p) { return *reinterpret_cast<const Bytes16*>(p); }
  __device__ __forceinline__ static void widen(const Raw& r, float* v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 f = WIDEN(r.w[i]);
      v[2 * i] = f.x;
      v[2 * i + 1] = f.y;
    }
  }
  // rounds to nearest even
  __device__ __forceinline__ static void store(T* p, const float* v) {
    Bytes16 a;
#pragma unroll
    for (int i = 0; i < 4; ++i) a.w[i] = NARROW(make_float2(v[2 * i], v[2 * i + 1]));
    *reinterpret_cast<Bytes16*>(p) = a;
  }
  __device__ __forceinline__ static float get(const T* p) { return WIDEN(*p).x; }
  __device__ __forceinline__ static void put(T* p, float v) { *p = (uint16_t)NARROW(make_float2(v, 0.f)); }
};
using ElemBF16 = Elem16<1, bf16x2_to_f32, f32_to_bf16x2>;
using ElemF16 = Elem16<2, f16x2_to_f32, f32_to_f16x2>;

// fn(storage type) for a value of rdfft_dtype_t
template <class F>
hipError_t with_elem(int storage, F&& fn) {
  switch (storage) {
    case ElemF32::kId: return fn(ElemF32{});
    case ElemBF16::kId: return fn(ElemBF16{});
    case ElemF16::kId: return fn(ElemF16{});
    default: return hipErrorInvalidValue;
  }
}

// Values i0 ... i0+7 of a row of n of any length, zeros past its end.
template <class E>
__device__ __forceinline__ void read_group(const typename E::T* row, int64_t i0, int64_t n, float* v) {
  if (i0 + kVec <= n) {
    E::widen(E::load(row + i0), v);
  } else {
#pragma unroll
    for (int i = 0; i < kVec; ++i) v[i] = i0 + i < n ? E::get(row + i0 + i) : 0.f;
  }
}
template <class E>
__device__ __forceinline__ void write_group(typename E::T* row, int64_t i0, int64_t n, const float* v) {
  if (i0 + kVec <= n) {
    E::store(row + i0, v);
  } else {
#pragma unroll
    for (int i = 0; i < kVec; ++i)
      if (i0 + i < n) E::put(row + i0 + i, v[i]);
  }
}

// ----------------------------------------------------------------------------------
// cross-lane

template <int CTRL>
__device__ __forceinline__ uint32_t dpp_u32(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true);
}
// the maximum over each aligned group of four lanes
__device__ __forceinline__ uint32_t quad_max(uint32_t v) {
  v = max(v, dpp_u32<0xb1>(v));  // quad_perm 1,0,3,2
  return max(v, dpp_u32<0x4e>(v));  // quad_perm 2,3,0,1
}

// the sum over the wave, in every lane: rows of 16 lanes by shifts, then from row to row
__device__ __forceinline__ float wave_sum(float x) {
  const auto step = [](float v, auto ctrl, auto mask) {
    return v + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), decltype(ctrl)::value,
                                                          decltype(mask)::value, 0xf, false));
  };
  using std::integral_constant;
  x = step(x, integral_constant<int, 0x111>{}, integral_constant<int, 0xf>{});  // row_shr 1
  x = step(x, integral_constant<int, 0x112>{}, integral_constant<int, 0xf>{});
  x = step(x, integral_constant<int, 0x114>{}, integral_constant<int, 0xf>{});
  x = step(x, integral_constant<int, 0x118>{}, integral_constant<int, 0xf>{});
  x = step(x, integral_constant<int, 0x142>{}, integral_constant<int, 0xa>{});  // row_bcast 15
  x = step(x, integral_constant<int, 0x143>{}, integral_constant<int, 0xc>{});  // row_bcast 31
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 63));
}

// ----------------------------------------------------------------------------------
// the 8-bit format

// |v| as bits: ordered as the values are, an infinity above every number and a NaN above that
__device__ __forceinline__ uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }

__device__ __forceinline__ uint32_t max_bits8(const float* v) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < kVec; ++i) m = max(m, abs_bits(v[i]));
  return m;
}

// Scale byte of a block from its largest |x|: with |x| = f * 2^k, 1 <= f < 2, e is k - 6 while
// f <= 127/64, whose fraction is 0x7e0000; more carries into the exponent field.
__device__ __forceinline__ int ck_scale_byte(uint32_t amax) {
  const int s = (int)((amax + 0x1ffffu) >> 23) - 6;
  return amax >= 0x7f800000u ? kCkNaN : max(s, 0);
}
// 2^-e (0 for a block that is not finite: with its values taken as 0, so are its codes)
__device__ __forceinline__ float ck_inverse(int s) { return s == kCkNaN ? 0.f : __uint_as_float((uint32_t)(254 - s) << 23); }
// 2^e, NaN for 255
__device__ __forceinline__ float ck_scale(int s) {
  return __uint_as_float(s == kCkNaN ? 0x7fc00000u : s == 0 ? 0x00400000u : (uint32_t)s << 23);
}

// Eight codes.  1.5 * 2^23 + x * 2^-e rounds to an integer, half to even, whose lowest byte is
// the code: one instruction a value, and byte moves.
__device__ __forceinline__ Bytes8 ck_encode(const float* v, int s) {
  const float inv = ck_inverse(s);
  uint32_t c[kVec];
#pragma unroll
  for (int i = 0; i < kVec; ++i) c[i] = __float_as_uint(fmaf(s == kCkNaN ? 0.f : v[i], inv, 12582912.0f));
  Bytes8 r;
#pragma unroll
  for (int h = 0; h < 2; ++h)
    r.w[h] = (c[4 * h] & 0xff) | (c[4 * h + 1] & 0xff) << 8 | (c[4 * h + 2] & 0xff) << 16 | c[4 * h + 3] << 24;
  return r;
}
// Eight values, of a checkpoint of E's numbers (float32 for what a kernel computed).
template <class E>
__device__ __forceinline__ void ck_decode(const Bytes8& r, float scale, float* v) {
#pragma unroll
  for (int i = 0; i < kVec; ++i) v[i] = (float)(int8_t)(r.w[i / 4] >> (8 * (i % 4))) * scale;
  if (scale == E::kLastStep) {
#pragma unroll
    for (int i = 0; i < kVec; ++i) v[i] = fabsf(v[i]) == E::kPast ? copysignf(E::kMost, v[i]) : v[i];
  }
}

// Eight codes of a row, zeros past its end.
__device__ __forceinline__ Bytes8 tail_codes(const int8_t* row, int64_t i0, int64_t n) {
  Bytes8 r = {{0, 0}};
#pragma unroll
  for (int i = 0; i < kVec; ++i)
    if (i0 + i < n) r.w[i / 4] |= (uint32_t)(uint8_t)row[i0 + i] << (8 * (i % 4));
  return r;
}
__device__ __forceinline__ void write_codes(int8_t* row, int64_t i0, int64_t n, const Bytes8& c) {
  if (i0 + kVec <= n) {
    *reinterpret_cast<Bytes8*>(row + i0) = c;
  } else {
#pragma unroll
    for (int i = 0; i < kVec; ++i)
      if (i0 + i < n) row[i0 + i] = (int8_t)(c.w[i / 4] >> (8 * (i % 4)));
  }
}

// The checkpoint of eight values a lane, four consecutive lanes to a block, i0 a multiple of eight.
__device__ __forceinline__ void write_checkpoint(int8_t* codes, uint8_t* scales, int64_t i0, int64_t n, const float* v) {
  const int s = ck_scale_byte(quad_max(max_bits8(v)));
  if (i0 >= n) return;
  write_codes(codes, i0, n, ck_encode(v, s));
  if (i0 % kCkBlock == 0) scales[i0 / kCkBlock] = (uint8_t)s;
}

}  // namespace rdfft
