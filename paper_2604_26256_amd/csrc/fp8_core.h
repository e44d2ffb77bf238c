// Conversions between fp32, bf16 bits and OCP E4M3FN codes, shared by the append
// kernels.  Included by HIP sources only.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace dora {

__device__ __forceinline__ float bf16_bits_to_f32(uint16_t b) {
  return __uint_as_float((uint32_t)b << 16);
}

// Value of an E4M3FN code, exact in fp32.
__device__ __forceinline__ float e4m3_to_f32(uint32_t c) {
  const uint32_t sign = (c & 0x80u) << 24;
  const uint32_t e = (c >> 3) & 0xFu, m = c & 0x7u;
  if (e == 0xFu && m == 0x7u) return __uint_as_float(sign | 0x7FC00000u);
  if (e == 0) {  // subnormal (or zero): m * 2^-9
    const float v = (float)m * 0x1p-9f;
    return sign ? -v : v;
  }
  return __uint_as_float(sign | ((e + 120u) << 23) | (m << 20));
}

// Nearest E4M3FN code of x, ties to the even mantissa, saturating to +-448.
// Works on the fp32 bit pattern: the 20 mantissa bits below the kept 3 decide
// the rounding, and a carry out of the mantissa moves into the exponent.
__device__ __forceinline__ uint32_t f32_to_e4m3(float x) {
  const uint32_t u = __float_as_uint(x);
  const uint32_t sign = (u >> 24) & 0x80u;
  const uint32_t a = u & 0x7FFFFFFFu;
  if (a > 0x7F800000u) return sign | 0x7Fu;                 // NaN
  if (a >= 0x43E00000u) return sign | 0x7Eu;                // >= 448 (inf included)
  if (a < 0x3C800000u) {                                    // below 2^-6: steps of 2^-9
    const float m = __builtin_rintf(__uint_as_float(a) * 512.0f);  // exact scaling, RNE
    return sign | (uint32_t)m;                              // 8 -> 0x08 = 2^-6
  }
  const uint32_t keep = (a >> 20) & 0x7u, rest = a & 0xFFFFFu;
  uint32_t code = ((((a >> 23) - 120u) << 3) | keep);
  if (rest > 0x80000u || (rest == 0x80000u && (keep & 1u))) code += 1u;
  return sign | code;
}

}  // namespace dora
