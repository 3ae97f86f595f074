// Rows held in 8 bits: D codes and one exponent byte b per token and head, for the
// values code * 2^(b - 127); b = 255 is NaN.
//
// The scale is a power of two rather than max / 127. Quantising is then exact up to
// the one rounding of each entry (no quotient, so every implementation gets the same
// codes), reading back into bf16 does not round (a code has at most 8 significant
// bits), and a tile for the tensor cores can be formed in bf16 without error. It costs
// whole-number codes up to one of their 7 bits, half of one on average, and e4m3
// nothing.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp8.h>

#include "pair_common.cuh"

namespace pairk {
namespace q8 {

constexpr int kPlain = -1;  // a cache in the type of its queries
constexpr int kI8 = PAIR_CACHE_I8, kE4M3 = PAIR_CACHE_E4M3;

// 2^(b - 127); 2^-127 is below the normal numbers.
__device__ __forceinline__ float scale_of(uint32_t b) {
  return __uint_as_float(b == 255 ? 0x7fc00000u : b ? b << 23 : 0x00400000u);
}

// The four codes of a word.
template <int F>
__device__ __forceinline__ void decode4(uint32_t w, float (&x)[4]) {
  if constexpr (F == kI8) {
    w ^= 0x80808080u;  // code + 128
#pragma unroll
    for (int k = 0; k < 4; ++k)  // 2^23 + (code + 128), by its bits
      x[k] = __uint_as_float(__byte_perm(w, 0x4b000000u, 0x7440 | k)) - 8388736.f;
  } else {
    const __half2 lo(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)w, __NV_E4M3));
    const __half2 hi(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w >> 16), __NV_E4M3));
    const float2 a = __half22float2(lo), b = __half22float2(hi);
    x[0] = a.x, x[1] = a.y, x[2] = b.x, x[3] = b.y;
  }
}
template <int F>
__device__ __forceinline__ float decode1(uint32_t byte) {
  float x[4];
  decode4<F>(byte, x);
  return x[0];
}

__device__ __forceinline__ __nv_bfloat162 as_bf16x2(uint32_t x) {
  return *reinterpret_cast<const __nv_bfloat162 *>(&x);
}
// Whole numbers c over 64 out of the bytes u = c + 128 in the low halves of x's halves: a
// byte u is as a bf16 number u 2^-133 (below 128 a subnormal one, from there on one of
// the least exponent, in the same steps). Times 2^127, less 2.
__device__ __forceinline__ __nv_bfloat162 whole_to_bf16(uint32_t x) {
  return __hfma2(as_bf16x2(x), as_bf16x2(0x7f007f00u), as_bf16x2(0xc000c000u));
}

// The exponent byte of a row whose largest |x| has these bits: the least one with
// which it is below 127.5 or 464, half a step above the largest code. A significand of
// 1 + m with E - 6 gives 64 (1 + m), at most 127 if it is below 127.5; with E - 8 e4m3
// gets 256 (1 + m), at most 448 if it is below 464. What is not below carries into the
// exponent (464 too, which would round to 448: the bytes are the contract, and the same
// comparison does for both formats).
template <int F>
__device__ __forceinline__ uint32_t exponent_of(uint32_t top) {
  constexpr uint32_t carry = F == kI8 ? 0x010000u : 0x180000u;
  constexpr int down = F == kI8 ? 6 : 8;
  return top >= 0x7f800000u ? 255u : (uint32_t)max(0, (int)((top + carry) >> 23) - down);
}

// Codes of four entries, times `inv` = 2^(127 - b): exact up to the one rounding, to
// nearest even.
template <int F>
__device__ __forceinline__ uint32_t encode4(const float (&x)[4], float inv) {
  if constexpr (F == kI8) {
    uint32_t u[4];
#pragma unroll
    for (int k = 0; k < 4; ++k)  // the addition rounds, and leaves the code in the low byte
      u[k] = __float_as_uint(x[k] * inv + 12582912.f);
    return __byte_perm(__byte_perm(u[0], u[1], 0x0040), __byte_perm(u[2], u[3], 0x0040), 0x5410);
  } else {
    const __nv_fp8x2_storage_t lo = __nv_cvt_float2_to_fp8x2(
        make_float2(x[0] * inv, x[1] * inv), __NV_SATFINITE, __NV_E4M3);
    const __nv_fp8x2_storage_t hi = __nv_cvt_float2_to_fp8x2(
        make_float2(x[2] * inv, x[3] * inv), __NV_SATFINITE, __NV_E4M3);
    return (uint32_t)lo | (uint32_t)hi << 16;
  }
}

}  // namespace q8
}  // namespace pairk
