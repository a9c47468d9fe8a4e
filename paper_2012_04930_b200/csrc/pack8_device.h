// The 8-bit format of activation checkpoints, as kernels read and write it.  32 consecutive columns of a row share a step
// 2^(e - 127), e a byte; a value is q * step with q in [-127, 127].  e is the smallest byte from 1 on for which the largest
// magnitude of the 32 rounds to at most 127 steps, so every value is off by at most half a step.  (e ends at 248: what would
// round to 128 steps of 2^121, the last 0.4 % below infinity, is kept as 127 of them.)  A step is a power of two:
// x / step and q * step are exact, and q * step is a bf16 number, which the tensor cores take without a split.  A block with
// a value that is not finite has e = 255 and q = 0: 0 * 2^128 (the infinity) restores as NaN.
#pragma once
#include <cuda_runtime.h>

#include <cstdint>

namespace gcnsa {
namespace {

constexpr int kPackBlock = 32;

// bits: the largest of the block's magnitudes as fp32 words with the sign cleared (as integers these order like the values,
// infinity and NaN last)
__device__ __forceinline__ uint32_t pack8_exponent(uint32_t bits) {
  if (bits >= 0x7f800000u) return 255;
  // 2^(exponent - 133) puts the value at 64 to 128 steps; from 127.5 on (mantissa 1.9921875, 0x10000 below the next exponent) it
  // would round to 128
  return (uint32_t)min(max((int)((bits + 0x10000u) >> 23) - 6, 1), 248);
}
// the larger of two magnitudes as such a word; a NaN stays one
__device__ __forceinline__ float pack8_larger(float a, float b) {
  float m;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(m) : "f"(fabsf(a)), "f"(fabsf(b)));
  return m;
}
__device__ __forceinline__ uint32_t pack8_magnitude(const float (&x)[4]) {
  return __float_as_uint(pack8_larger(pack8_larger(x[0], x[1]), pack8_larger(x[2], x[3])));
}
__device__ __forceinline__ float pack8_step(uint32_t e) { return __uint_as_float(e << 23); }
// Four values as bytes: rint(x / step) is the low byte of x / step + 1.5 2^23 (x / step is exact and below 128; ties to even); zeros
// where the block is not finite.
__device__ __forceinline__ uint32_t pack8_bytes(const float (&x)[4], uint32_t e) {
  const float inv = __uint_as_float((254 - e) << 23);
  float s[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) s[k] = fmaf(x[k], inv, 12582912.f);
  if (e >= 248)
#pragma unroll
    for (int k = 0; k < 4; ++k) s[k] = e == 255 ? 0.f : fminf(fmaxf(s[k], 12582912.f - 127.f), 12582912.f + 127.f);
  return __byte_perm(__byte_perm(__float_as_uint(s[0]), __float_as_uint(s[1]), 0x0040),
                     __byte_perm(__float_as_uint(s[2]), __float_as_uint(s[3]), 0x0040), 0x5410);
}
// four packed bytes as floats: 2^23 + (q + 128) has q + 128 as its low byte
__device__ __forceinline__ void pack8_open(uint32_t q4, float (&v)[4]) {
  q4 ^= 0x80808080u;
  v[0] = __uint_as_float(__byte_perm(q4, 0x4B000000u, 0x7540)) - 8388736.f;
  v[1] = __uint_as_float(__byte_perm(q4, 0x4B000000u, 0x7541)) - 8388736.f;
  v[2] = __uint_as_float(__byte_perm(q4, 0x4B000000u, 0x7542)) - 8388736.f;
  v[3] = __uint_as_float(__byte_perm(q4, 0x4B000000u, 0x7543)) - 8388736.f;
}

}  // namespace
}  // namespace gcnsa
