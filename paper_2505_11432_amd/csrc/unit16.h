// Numbers of [0, 1] in 16 bits, with the range of single precision: sign and top bit of the exponent are 0 up to 1.99, the 16 bits below them are seven of
// the exponent and nine of the significand.  Ten significant bits (a rounding is 2^-10 of a number at most) down to 2^-126.
// (bf16 has eight; fp16 eleven, but from 2^-14 on fewer, from 2^-17 on fewer than bf16, and nothing below 2^-25.)
#pragma once
#include <hip/hip_runtime.h>

namespace moe {

// two of them, rounded to nearest, in three instructions
__device__ __forceinline__ unsigned unit16_pack(float lo, float hi) {
  const unsigned a = (__builtin_bit_cast(unsigned, lo) << 2) + 0x8000u, b = (__builtin_bit_cast(unsigned, hi) << 2) + 0x8000u;
  return __builtin_amdgcn_perm(b, a, 0x07060302u);
}
__device__ __forceinline__ float unit16_low(unsigned two) { return __builtin_bit_cast(float, two << 14 & 0x3fffc000u); }
__device__ __forceinline__ float unit16_high(unsigned two) { return __builtin_bit_cast(float, two >> 2 & 0x3fffc000u); }

}  // namespace moe
