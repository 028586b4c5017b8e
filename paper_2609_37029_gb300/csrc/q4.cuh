// Keys and values held in 4 bits: the format's arithmetic (definition: lsp_kv_cache
// in include/lsp.h).
//
// A word holds eight codes c + 8 (c = -7..7); with shift 4 k and mask 0x000F000F it
// gives the pair of elements 2 k and 2 k + 1 in two 16-bit halves.  A code in the
// low bits of the bfloat16 128.0 makes 128 + (c + 8), exactly; minus 136 that is c,
// times the scale (five significant bits) a number of eight: no step rounds.
#pragma once

#include "common.cuh"

namespace lsp {

constexpr int kQ4Group = 32;
constexpr uint32_t kQ4Zero = 0x88888888u;        // eight codes of 0

__device__ __forceinline__ uint32_t bf2_bits(__nv_bfloat162 x) { return *reinterpret_cast<uint32_t*>(&x); }
__device__ __forceinline__ __nv_bfloat162 bits_bf2(uint32_t x) { return *reinterpret_cast<__nv_bfloat162*>(&x); }

// Two elements (codes in the low 4 bits of each half of w) times two scales, as a pair of bfloat16.
__device__ __forceinline__ uint32_t q4_pair(uint32_t w, uint32_t scales) {
  uint32_t x;
  asm("lop3.b32 %0, %1, 0x000F000F, 0x43004300, 0xEA;" : "=r"(x) : "r"(w));      // (w & mask) | 128.0
  return bf2_bits(__hmul2(__hsub2(bits_bf2(x), bits_bf2(0x43084308u)), bits_bf2(scales)));
}

// The scale of a group from the greatest |x| of its values (as bits, so that what is
// not finite counts as greater than what is): the least number of five significant
// bits with 7 s >= a.  a / 7 correctly rounded and cut to five bits is that number,
// or the one before it; 7 s is exact.
__device__ __forceinline__ float q4_scale(uint32_t a_bits) {
  if (a_bits >= 0x7F800000u) return __uint_as_float(0x7FC00000u);
  const float a = __uint_as_float(a_bits);
  const uint32_t bits = __float_as_uint(__fdiv_rn(a, 7.0f)) & ~0x7FFFFu;
  const float low = __uint_as_float(bits);
  return 7.0f * low < a ? __uint_as_float(bits + 0x80000u) : low;
}

// Eight codes of a group.  The product with the reciprocal names a whole number that
// is the nearest or next to it; what is left over is exact (r s has eight bits, and
// the difference no more than x's) and says which, ties to the even one.
__device__ __forceinline__ uint32_t q4_codes(const float* x, float s) {
  if (!(s > 0.0f)) return kQ4Zero;                // an empty group, or one that is NaN
  const float up = s < 1.1754944e-30f ? 18446744073709551616.0f : 1.0f;          // (2^64: reciprocals stay finite)
  s *= up;
  const float inv = 1.0f / s, half = 0.5f * s;
  uint32_t w = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float y = x[e] * up, r = rintf(y * inv), rest = fmaf(-r, s, y);
    int c = (int)r;
    if (rest > half || (rest == half && (c & 1))) ++c;
    else if (rest < -half || (rest == -half && (c & 1))) --c;
    w |= (uint32_t)(c + 8) << (16 * (e & 1) + 4 * (e >> 1));
  }
  return w;
}

}  // namespace lsp
