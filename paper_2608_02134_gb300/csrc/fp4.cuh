// Rows held in 4 bits.  A row is cut into blocks of 16 channels; a block has a scale s and a
// value is c s with c one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 and a sign (e2m1).  s is the upper
// byte but for the sign of a half: 5 bits of exponent, 3 of mantissa, so s as half is the byte
// shifted left by 7, and c s, with at most 6 bits of mantissa, is exact in half and in bf16.
// A byte above 0xf8 is a NaN: a block with a value that is not finite stands for 16 NaN.
//
// A head's part of a page holds the codes of its slots, d / 2 bytes each (the even channel in
// the low half of a byte), and then their scales, d / 16 bytes each.
#pragma once

#include <cuda_fp16.h>

#include "cache.cuh"

namespace gmc {

constexpr uint32_t FP4_MAX_SCALE = 0xe0;  // 8192: 6 s stays below the largest half
constexpr uint32_t FP4_NAN_SCALE = 0xf9;

// Bytes of one head's part of a page (a multiple of 4).
inline long long fp4_part(int ps, int d) { return (long long)ps * (d / 2 + d / 16); }

// Byte offset of a row's scales from the start of its page and head.
__device__ __forceinline__ long long fp4_scale_at(const KV& c, int slot) {
  return (long long)c.ps * (c.d / 2) + (long long)slot * (c.d / 16);
}

// Two scales as halves, the first one's in the low half of a word.
__device__ __forceinline__ uint32_t fp4_scales(uint32_t s0, uint32_t s1) {
  return (s0 << 7) | (s1 << 23);
}
__device__ __forceinline__ uint32_t fp4_scale2(uint32_t s) { return s * 0x00800080u; }

__device__ __forceinline__ uint32_t hmul2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}

// The four bytes of a word as four pairs of halves.
__device__ __forceinline__ void fp4_halves(uint32_t w, uint32_t* h) {
  asm("{\n\t.reg .b8 a, b, c, d;\n\t"
      "mov.b32 {a, b, c, d}, %4;\n\t"
      "cvt.rn.f16x2.e2m1x2 %0, a;\n\t"
      "cvt.rn.f16x2.e2m1x2 %1, b;\n\t"
      "cvt.rn.f16x2.e2m1x2 %2, c;\n\t"
      "cvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
      : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3])
      : "r"(w));
}
// Eight codes as eight bf16.
__device__ __forceinline__ uint4 fp4_bf16(uint32_t w, uint32_t scale2) {
  uint32_t h[4];
  fp4_halves(w, h);
  uint32_t r[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    h[i] = hmul2(h[i], scale2);
    const float2 v = __half22float2(*reinterpret_cast<const __half2*>(&h[i]));
    const __nv_bfloat162 b = __floats2bfloat162_rn(v.x, v.y);  // exact
    r[i] = *reinterpret_cast<const uint32_t*>(&b);
  }
  return make_uint4(r[0], r[1], r[2], r[3]);
}

// Eight floats as codes: the nearest, ties to the even code, 6 at most.
__device__ __forceinline__ uint32_t fp4_codes(const float* y) {
  uint32_t r;
  asm("{\n\t.reg .b8 a, b, c, d;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
      "mov.b32 %0, {a, b, c, d};\n\t}"
      : "=r"(r)
      : "f"(y[0]), "f"(y[1]), "f"(y[2]), "f"(y[3]), "f"(y[4]), "f"(y[5]), "f"(y[6]), "f"(y[7]));
  return r;
}

// 32 bytes at once: whole sectors.
__device__ __forceinline__ void store32(void* p, const uint4& lo, const uint4& hi) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(lo.x),
               "r"(lo.y), "r"(lo.z), "r"(lo.w), "r"(hi.x), "r"(hi.y), "r"(hi.z), "r"(hi.w)
               : "memory");
}

// A block's codes and scale from its bf16 values.
//   s = max |x| / 6 rounded to 3 bits behind the point, ties to even, 2^-17 at least where any
//   x is not 0, 8192 at most; code = x / s rounded.
// Both are exact for bf16 values: a quotient of an 8-bit and a 4-bit mantissa that is no tie is
// 2^-10 of itself or more away from one, and products with 1 / 6 and 1 / s as sums of two floats
// leave ties ties (1 / s alone is off by 2^-24, which misses them).
__device__ __forceinline__ uint32_t max_u16x2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("max.u16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
// The largest of eight magnitudes, as an integer: a NaN is larger than infinity.
__device__ __forceinline__ uint32_t fp4_top(const uint4& v) {
  constexpr uint32_t M = 0x7fff7fffu;
  const uint32_t t = max_u16x2(max_u16x2(v.x & M, v.y & M), max_u16x2(v.z & M, v.w & M));
  return max(t & 0xffffu, t >> 16);
}
struct Fp4Scale {
  uint32_t byte;
  float hi, lo;  // 1 / s
  // top: the block's largest magnitude, the bits of a bf16
  __device__ __forceinline__ explicit Fp4Scale(uint32_t top) {
    hi = lo = 0.f;
    byte = FP4_NAN_SCALE;
    if (top >= 0x7f80u) return;
    const float x = __uint_as_float(top << 16);
    constexpr float S = 0.166666671633720397949f, R = -4.967053879312289e-09f;  // S + R = 1 / 6
    const float t = fmaf(x, S, x * R);
    if (t >= 6.103515625e-05f) {  // 2^-14: a normal half
      const uint32_t b = __float_as_uint(t);
      byte = min(((b + 0x7ffffu + ((b >> 20) & 1u)) >> 20) - (112u << 3), FP4_MAX_SCALE);
    } else {
      byte = max((uint32_t)__float2int_rn(t * 131072.f), top != 0u ? 1u : 0u);
      if (byte == 0u) return;
    }
    const float s = __half2float(__ushort_as_half((unsigned short)(byte << 7)));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(hi) : "f"(s));
    lo = fmaf(-s, hi, 1.f) * hi;
  }
  __device__ __forceinline__ uint32_t codes(const uint4& v) const {
    if (byte == FP4_NAN_SCALE) return 0u;
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    float y[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const f32x2 x = pair(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
      const float2 z = unpair(fma2(x, pair(hi, hi), mul2(x, pair(lo, lo))));
      y[2 * i] = z.x;
      y[2 * i + 1] = z.y;
    }
    return fp4_codes(y);
  }
};
__device__ __forceinline__ uint2 fp4_block(const uint4& v0, const uint4& v1, uint32_t* scale) {
  const Fp4Scale s(max(fp4_top(v0), fp4_top(v1)));
  *scale = s.byte;
  return make_uint2(s.codes(v0), s.codes(v1));
}

// Weights become halves.  They are 2^(x - m) of logits x, m a base FP4_UP below the maximum that
// it was taken from, so that maximum's weight is 2^7 and a half loses 2^-32 of it at most where a
// weight is small: a sum over N keys behind one that outweighs them N 2^-32 (taken against the
// maximum itself N 2^-25, 0.3 % at 100,000 keys).  Above, halves reach to 2^16: m follows the
// running maximum only once that lies FP4_ROOM above it.  Maxima are rounded up (of large logits
// one rounding is more than that room), so no weight is beyond it.
constexpr float FP4_UP = 7.f, FP4_ROOM = FP4_UP + 8.f;

__device__ __forceinline__ void unpack_bf16(const uint4& v, float* x) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}

}  // namespace gmc
