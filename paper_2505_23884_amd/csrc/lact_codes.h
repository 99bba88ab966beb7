// A cache in 8 bits: a vector is held as e4m3 numbers c_i (sign, 4 bits of
// exponent, 3 of significand; 0x7f is NaN, there are no infinities) and one
// byte e + 127 for all of them, and stands for c_i 2^e. A power of two costs
// no accuracy, since the numbers are floating themselves, and makes every
// value one of bf16 and of fp32: nothing is rounded when it is read.
#pragma once

#include "lact_attn.h"

namespace lact {
namespace attn {

// Exponents that are written: the least e4m3 number, 2^-9, times 2^-117 is the
// least normal fp32, and the largest, 448, times 2^119 is within bf16.
constexpr int kMinExp = -117, kMaxExp = 119;

__device__ __forceinline__ float scale_of(int byte) { return __uint_as_float((uint32_t)byte << 23); }

// The smallest e with a <= 448 2^e = 1.75 2^(e + 8), within the range, plus
// 127, for a finite a >= 0.
__device__ __forceinline__ int scale_byte(float a) {
  const uint32_t x = __float_as_uint(a);
  const int e = (int)(x >> 23) - 135 + ((x & 0x7fffffu) > 0x600000u);
  return min(max(e, kMinExp), kMaxExp) + 127;
}

// Two of four numbers (the low or the high ones) as what they stand for.
template <bool HI>
__device__ __forceinline__ uint32_t codes_bf16(uint32_t codes, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, HI));
}
template <bool HI>
__device__ __forceinline__ f32x2 codes_fp32(uint32_t codes, float scale) {
  return __builtin_bit_cast(f32x2, __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(codes, scale, HI));
}

// Four of them as T: two words of bf16, or four of fp32, from to[0] on.
template <typename T>
__device__ __forceinline__ void widen(uint32_t codes, float scale, uint32_t* to) {
  if constexpr (sizeof(T) == 2) {
    to[0] = codes_bf16<false>(codes, scale);
    to[1] = codes_bf16<true>(codes, scale);
  } else {
    const f32x2 lo = codes_fp32<false>(codes, scale), hi = codes_fp32<true>(codes, scale);
    to[0] = __float_as_uint(lo[0]);
    to[1] = __float_as_uint(lo[1]);
    to[2] = __float_as_uint(hi[0]);
    to[3] = __float_as_uint(hi[1]);
  }
}

}  // namespace attn
}  // namespace lact
