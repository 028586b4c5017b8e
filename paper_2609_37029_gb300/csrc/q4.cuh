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

template <bool kX>
struct BoolTag {
  static constexpr bool value = kX;
};

// Shared memory by its 32-bit addresses: through a pointer whose origin the compiler cannot see, every access is a
// generic one with 64-bit arithmetic.
__device__ __forceinline__ uint32_t ld_shared(uint32_t at) {
  uint32_t x;
  asm volatile("ld.shared.u32 %0, [%1];" : "=r"(x) : "r"(at) : "memory");
  return x;
}
__device__ __forceinline__ void ld_shared2(uint32_t at, uint32_t& x, uint32_t& y) {
  asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(x), "=r"(y) : "r"(at) : "memory");
}
__device__ __forceinline__ uint32_t ld_shared_u16(uint32_t at) {
  uint32_t x;
  asm volatile("ld.shared.u16 %0, [%1];" : "=r"(x) : "r"(at) : "memory");
  return x;
}
__device__ __forceinline__ void st_shared4(uint32_t at, uint32_t x, uint32_t y, uint32_t z, uint32_t w) {
  asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(x), "r"(y), "r"(z), "r"(w) : "memory");
}
__device__ __forceinline__ uint4 ld_shared4(uint32_t at) {
  uint4 x;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(x.x), "=r"(x.y), "=r"(x.z), "=r"(x.w) : "r"(at) : "memory");
  return x;
}

// A run of a block's codes or scales into shared memory (addresses and bytes multiples of 16).
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst),
               "l"(src), "r"(bytes), "r"(bar)
               : "memory");
}

constexpr uint32_t kQ4Zero = 0x88888888u;        // eight codes of 0

__device__ __forceinline__ uint32_t bf2_bits(__nv_bfloat162 x) { return *reinterpret_cast<uint32_t*>(&x); }
__device__ __forceinline__ __nv_bfloat162 bits_bf2(uint32_t x) { return *reinterpret_cast<__nv_bfloat162*>(&x); }

// a + b and a b + c: two fp32 operations an instruction
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 d;
  asm("{\n .reg .b64 x, y;\n mov.b64 x, {%2, %3};\n mov.b64 y, {%4, %5};\n add.rn.f32x2 x, x, y;\n mov.b64 {%0, %1}, x;\n}"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 d;
  asm("{\n .reg .b64 x, y, z;\n mov.b64 x, {%2, %3};\n mov.b64 y, {%4, %5};\n mov.b64 z, {%6, %7};\n"
      " fma.rn.f32x2 x, x, y, z;\n mov.b64 {%0, %1}, x;\n}"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return d;
}

// What unpacking takes besides, in registers: a loop that has them as immediate
// operands moves them there for every pair.
struct Q4Consts {
  uint32_t mask, one, minus;
  __device__ __forceinline__ Q4Consts() {
    asm volatile("mov.b32 %0, 0x000F000F;" : "=r"(mask));
    asm volatile("mov.b32 %0, 0x43004300;" : "=r"(one));         // 128.0
    asm volatile("mov.b32 %0, 0xC308C308;" : "=r"(minus));       // -136.0
  }
};

// Two elements (codes in the low 4 bits of each half of w) times two scales, as a pair of bfloat16.
__device__ __forceinline__ uint32_t q4_pair(const Q4Consts& k, uint32_t w, uint32_t scales) {
  uint32_t x;
  asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(x) : "r"(w), "r"(k.mask), "r"(k.one));      // (w & mask) | 128.0
  return bf2_bits(__hmul2(__hadd2(bits_bf2(x), bits_bf2(k.minus)), bits_bf2(scales)));
}

// Eighths of a word's four pairs, for products that have a factor for the 8 anyway.  A
// code in the upper four bits of 2.0's mantissa makes 2 + (c + 8) / 8, and of that times
// s less 3 s is c s / 8: one fused step, because 3 s (seven significant bits) is a
// bfloat16 number too, and so is the result.  (What c s is beyond bfloat16's largest
// number stays finite.)
struct Q4Eighths {
  uint32_t mask, two;
  __device__ __forceinline__ Q4Eighths() {
    asm volatile("mov.b32 %0, 0x00780078;" : "=r"(mask));
    asm volatile("mov.b32 %0, 0x40004000;" : "=r"(two));
  }
};
__device__ __forceinline__ void q4_eighths(const Q4Eighths& k, uint32_t w, uint32_t scales, uint32_t (&x)[4]) {
  const __nv_bfloat162 minus = __hmul2(bits_bf2(scales), bits_bf2(0xC040C040u));         // -3 s
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t y;
    asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(y) : "r"(i == 0 ? w << 3 : w >> (4 * i - 3)), "r"(k.mask), "r"(k.two));
    x[i] = bf2_bits(__hfma2(bits_bf2(y), bits_bf2(scales), minus));
  }
}

// The scale of a group from the greatest |x| of its values (as bits, so that what is
// not finite counts as greater than what is): the least number of five significant
// bits with 7 s >= a.  A quotient that is never below a / 7 and hardly above it, cut
// to five bits, is that number or the one before it; 7 s is exact and tells.
__device__ __forceinline__ float q4_scale(uint32_t a_bits) {
  if (a_bits >= 0x7F800000u) return __uint_as_float(0x7FC00000u);
  const float a = __uint_as_float(a_bits);
  const uint32_t bits = __float_as_uint(__fmul_ru(a, 0.14285715f)) & ~0x7FFFFu;  // (the next number above 1/7)
  return 7.0f * __uint_as_float(bits) < a ? __uint_as_float(bits + 0x80000u) : __uint_as_float(bits);
}

// Eight codes of a group, by x / s and a sum whose last place is the whole number:
// 1.5 2^23 + 8 + c, so that codes are the low bits (rounded to nearest, ties to even;
// the 8 moves no tie).  What the quotient may not do is reach a tie, or leave one:
//   f32   it is the correctly rounded one: the reciprocal and one step of the exact
//         remainder (Markstein 1990).  Ties n + 1/2 are fp32 numbers, and an x next
//         to s (n + 1/2) lies at least half a last place of the quotient from it.
//   bf16  (x of eight significant bits) a quotient is a tie, or at least 2^-4 / (2 31)
//         > 2^-10 from one; rounded to multiples of 2^-13 first, it stays what it is.
template <bool kShort>                           // x of eight significant bits
__device__ __forceinline__ uint32_t q4_codes(float* x, float s) {
  if (!(s >= 1e-30f)) {
    if (!(s > 0.0f)) return kQ4Zero;             // an empty group, or one that is NaN
    s *= 18446744073709551616.0f;                // (times 2^64: reciprocals stay finite)
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] *= 18446744073709551616.0f;
  }
  float inv;
  if constexpr (kShort)
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(s));      // (2^-23 of it: what is off by that is rounded away)
  else
    inv = __frcp_rn(s);
  uint32_t w = 0;
  const float2 inv2 = make_float2(inv, inv);
#pragma unroll
  for (int e = 0; e < 8; e += 2) {
    const float2 x2 = make_float2(x[e], x[e + 1]);
    float2 y;
    if constexpr (kShort) {
      y = add2(fma2(x2, inv2, make_float2(1536.0f, 1536.0f)), make_float2(12582920.0f - 1536.0f, 12582920.0f - 1536.0f));
    } else {
      const float2 q = make_float2(x2.x * inv, x2.y * inv);
      y = add2(fma2(fma2(make_float2(-q.x, -q.y), make_float2(s, s), x2), inv2, q), make_float2(12582920.0f, 12582920.0f));
    }
    w += __float_as_uint(y.x) << (2 * e);
    w += __float_as_uint(y.y) << (2 * e + 16);
  }
  return w - 0x4B400000u * 0x11111111u;          // (the upper bits of the eight numbers)
}

}  // namespace lsp
