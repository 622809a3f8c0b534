// The 8-bit form of token features (lvx_packed): 32 features of a row share an exponent byte b and are whole numbers q
// of steps of 2^(b - 133), |q| <= 127.
//
// b comes from the largest magnitude of the group, as the bits u of a float32: (u + 2^16) >> 23 is its biased exponent, one more
// where it would round to 128 steps (a mantissa of 127.5 / 64 or more: 0x7f0000).  At least 8, so that the step and what
// it is divided by are ordinary floats (smaller groups have steps of 2^-125 all the same).  255 says that the group
// holds an infinity, a NaN or a magnitude of 2^128 (1 - 2^-8) or more: all of it reads as NaN.
// Multiplying by a power of two is exact, so the one rounding is that to a whole number (half to even), off by at most
// half a step, and the packed values are exact in bf16 and in float32.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace lvx {
namespace packed {

constexpr int GROUP = 32;
__host__ __device__ constexpr int groups(int E) { return (E + GROUP - 1) / GROUP; }

__device__ __forceinline__ unsigned magnitude(float x) { return __float_as_uint(x) & 0x7fffffffu; }
__device__ __forceinline__ unsigned exponent_of(unsigned largest) {
  const unsigned b = (largest + 0x10000u) >> 23;
  return b < 8u ? 8u : b > 255u ? 255u : b;
}
__device__ __forceinline__ float step_of(unsigned b) { return b == 255u ? __builtin_nanf("") : __uint_as_float((b - 6u) << 23); }
__device__ __forceinline__ float inverse_step_of(unsigned b) { return b == 255u ? 0.f : __uint_as_float((260u - b) << 23); }

// x in whole steps (half to even): the sum with 1.5 * 2^23 has no bits below one, and the product is exact.  (What the numbers of a
// group that reads as NaN are says nothing.)
constexpr float ROUNDER = 12582912.f;
__device__ __forceinline__ float steps(float x, float inverse) { return fmaf(x, inverse, ROUNDER); }
__device__ __forceinline__ int8_t whole(float s) { return (int8_t)(__float_as_uint(s) & 0xffu); }
__device__ __forceinline__ float value(float s, float step) { return (s - ROUNDER) * step; }

}  // namespace packed
}  // namespace lvx
