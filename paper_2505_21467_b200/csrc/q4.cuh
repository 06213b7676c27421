// The 4-bit rows of dlm_kv_cache_q4: groups of 32 consecutive values with one scale byte each.
//
//   value = (n - 8) * s,   n in 1 .. 15 (4 bits),   s = (1 + m / 8) * 2^(e - 20) from the byte eeeeemmm
//
// s has 4 significant bits and n - 8 has 3, so a value has 7 and is exact in bf16 (8): what the tensor cores multiply is the
// cache's value itself.  The byte has no sign and no special values, so its bf16 pattern is a shift and an add.  s is amax / 7
// rounded to nearest: the largest value is then at most 7.44 s, which rounds to 7, and no value is off by more than s / 2.
//
// Eight consecutive values are a 32-bit word with value j in bits 4 (j / 2) .. + 3 of its lower half (j even) or upper half (j
// odd), so that a shift and one three-input logic operation lift a pair of neighbours into the mantissas of two bf16: 128 + n
// is 0x4300 | n, and one fused multiply-add with c = -136 s leaves (n - 8) s.  136 s = 17 * (8 + m) * 2^.. has 8 significant
// bits, so c and the result are exact.  1.4 instructions a value.
#pragma once

#include <cuda_bf16.h>
#include <stdint.h>

#include "sm100_ptx.cuh"

namespace q4 {

constexpr int kGroup = 32;
constexpr uint32_t kScaleExponent = (127u - 20u) << 7;   // of byte 0, as bf16 bits
constexpr uint32_t kLargestBits = 0x46D2;                // bf16 of 7 * 3840, the largest value that the format holds

__device__ __forceinline__ uint32_t scale_bf16(uint32_t byte) { return (byte << 4) + kScaleExponent; }

struct Scale {
  __nv_bfloat162 s, c;   // the scale and -136 times it, twice each
};
__device__ __forceinline__ Scale make_scale(uint32_t byte) {
  const uint32_t b = scale_bf16(byte) * 0x00010001u;
  Scale r;
  r.s = *reinterpret_cast<const __nv_bfloat162*>(&b);
  r.c = __hmul2(r.s, __floats2bfloat162_rn(-136.f, -136.f));
  return r;
}

// The eight values of a word as four bf16 pairs.
__device__ __forceinline__ void decode8(uint32_t word, const Scale& sc, uint32_t (&out)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t p = ((word >> (4 * i)) & 0x000F000Fu) | 0x43004300u;
    const __nv_bfloat162 v = __hfma2(*reinterpret_cast<const __nv_bfloat162*>(&p), sc.s, sc.c);
    out[i] = *reinterpret_cast<const uint32_t*>(&v);
  }
}

// Eight values of a row per lane, a group of 32 per four neighbouring lanes (all lanes of the warp take part): the lane's word and the
// group's scale byte.  Quotients are taken with a reciprocal and one correction step: a quotient that lies exactly between two
// integers has few bits, the correction makes it exact and it goes to the even one; any other is at least 2^-12 of its size away from such a
// border.  The same holds for amax / 7 and the borders of the scale's 4 significant bits.
__device__ __forceinline__ uint32_t encode8(uint4 raw, uint32_t& byte) {
  uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
  uint32_t am = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) am = __vmaxu2(am, w[i] & 0x7FFF7FFFu);
  uint32_t a = max(am & 0xFFFFu, am >> 16);
  if (a > kLargestBits) {   // NaN, infinities and what is too large
    a = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
      for (int h = 0; h < 32; h += 16) {
        const uint32_t v = (w[i] >> h) & 0x7FFFu;
        const uint32_t to = v > 0x7F80u ? 0u : min(v, kLargestBits);
        w[i] = (w[i] & ~(0x7FFFu << h)) | (to << h);
        a = max(a, to);
      }
    }
  }
  a = max(a, __shfl_xor_sync(0xffffffffu, a, 1));
  a = max(a, __shfl_xor_sync(0xffffffffu, a, 2));
  const float amax = __uint_as_float(a << 16);
  const float t0 = amax * (1.f / 7.f), t = fmaf(fmaf(-7.f, t0, amax), 1.f / 7.f, t0);
  const uint32_t tb = __float_as_uint(t);
  const int e = (int)((tb + 0x7FFFFu + ((tb >> 20) & 1u)) >> 20) - (int)((127u - 20u) << 3);
  byte = (uint32_t)min(max(e, 0), 255);
  const float s = __uint_as_float(scale_bf16(byte) << 16), inv = __fdividef(1.f, s);
  const uint64_t inv2 = sm100::pack2(inv, inv), minus_s2 = sm100::pack2(-s, -s), magic2 = sm100::pack2(12582920.f, 12582920.f);
  uint32_t n[2][4];   // 1.5 * 2^23 + 8 + quotient as a float: its last bits are the rounded quotient + 8
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint64_t x = sm100::pack2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xFFFF0000u));
    const uint64_t y = sm100::mul2(x, inv2), z = sm100::fma2(sm100::fma2(minus_s2, y, x), inv2, y);
    float lo, hi;
    sm100::unpack2(sm100::add2(z, magic2), lo, hi);
    n[0][i] = __float_as_uint(lo);
    n[1][i] = __float_as_uint(hi);
  }
  // (what is above those bits stays above bit 16 of the sums)
  const uint32_t even = n[0][0] + (n[0][1] << 4) + (n[0][2] << 8) + (n[0][3] << 12), odd = n[1][0] + (n[1][1] << 4) + (n[1][2] << 8) + (n[1][3] << 12);
  return __byte_perm(even, odd, 0x5410);
}

}  // namespace q4
