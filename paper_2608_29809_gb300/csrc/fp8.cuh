// Eight-bit values: e4m3 codes with a power-of-two scale byte (see
// rc_fp8 / rc_kv8 in include/regioncache.h).
#pragma once
#include <cuda_fp16.h>
#include <stdint.h>

#include "common.cuh"

namespace rc {

// The scale byte of a block whose largest magnitude has the f32 bits `a`
// (sign cleared): the least e >= -127 with a <= 448 2^e = 1.75 2^(e + 8), plus
// 127.  Magnitudes compare like their bits, NaN above infinity, so an integer
// maximum over a block keeps non-finite values.
__device__ __forceinline__ int scale_byte(uint32_t a) {
  if (a >= 0x7f800000u) return 255;
  const int e = int(a >> 23) - 8 + ((a & 0x7fffffu) > 0x600000u ? 1 : 0);
  return e < 0 ? 0 : e;
}
// 2^(127 - b) in f32, NaN for 255.  (scale_byte gives at most 247, but a pool may
// come with a scale of 254, whose inverse is a subnormal.)
__device__ __forceinline__ float scale_inverse(int b) {
  return __uint_as_float(b == 255 ? 0x7fffffffu : b == 254 ? 0x400000u : uint32_t(254 - b) << 23);
}
// 2^(b - 127) in f32, NaN for 255.
__device__ __forceinline__ float scale_value(int b) {
  return __uint_as_float(b == 255 ? 0x7fffffffu : b == 0 ? 0x400000u : uint32_t(b) << 23);
}
// A part of a softmax row (sum l of weights 2^(s - m), products with the values)
// is kept as l 2^-e, m + e and products 2^-e: with this e the sum lies in [2^-8,
// 2^-7), so that up to 96 parts' products add up without passing the largest
// value.  Products take their value scale after 2^-e: only a result that f32
// cannot hold overflows.
__device__ __forceinline__ int part_exponent(float l) {
  return l > 0.f ? min(int(__float_as_uint(l) >> 23) - 127 + 8, 126) : 0;
}
// Two values as e4m3 codes (nearest, ties to even; `lo` in the low byte).
__device__ __forceinline__ uint32_t e4m3x2(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
// Two values times inv as codes (one packed product).
__device__ __forceinline__ uint32_t e4m3x2(float lo, float hi, uint64_t inv) {
  uint64_t v;
  asm("{\n\t.reg .b64 t;\n\tmov.b64 t, {%1, %2};\n\tmul.rn.f32x2 %0, t, %3;\n\t}"
      : "=l"(v)
      : "f"(lo), "f"(hi), "l"(inv));
  float a, b;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v));
  return e4m3x2(a, b);
}
__device__ __forceinline__ uint64_t both(float v) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %1};" : "=l"(r) : "f"(v));
  return r;
}
// Two codes as f16 (exact).
__device__ __forceinline__ uint32_t e4m3x2_f16x2(uint32_t codes) {
  uint32_t r;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"(uint16_t(codes)));
  return r;
}
// Four codes as f16: the lower and the upper two.
__device__ __forceinline__ void e4m3x4_f16(uint32_t w, uint32_t& lo, uint32_t& hi) {
  asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\t"
      "cvt.rn.f16x2.e4m3x2 %0, l;\n\tcvt.rn.f16x2.e4m3x2 %1, h;\n\t}"
      : "=r"(lo), "=r"(hi)
      : "r"(w));
}
__device__ __forceinline__ float2 e4m3x2_f32(uint32_t codes) {
  const uint32_t h = e4m3x2_f16x2(codes);
  return __half22float2(*reinterpret_cast<const __half2*>(&h));
}

// Eight consecutive source values as f32 bits' magnitudes' maximum and as
// eight codes: of bf16 (one 16-byte load) or f32 (two).
template <class T>
struct Eight;
template <>
struct Eight<__nv_bfloat16> {
  uint4 u;
  __device__ __forceinline__ void load(const __nv_bfloat16* p) {
    u = *reinterpret_cast<const uint4*>(p);
  }
  // values [0, n) of an unaligned or ragged run; the rest are zero
  __device__ __forceinline__ void load_some(const __nv_bfloat16* p, int n) {
    const uint16_t* s = reinterpret_cast<const uint16_t*>(p);
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      w[i] = (2 * i < n ? uint32_t(s[2 * i]) : 0u) |
             (2 * i + 1 < n ? uint32_t(s[2 * i + 1]) << 16 : 0u);
    u = make_uint4(w[0], w[1], w[2], w[3]);
  }
  __device__ __forceinline__ void zero() { u = make_uint4(0, 0, 0, 0); }
  __device__ __forceinline__ uint32_t top() const {  // f32 bits of the largest magnitude
    const uint32_t m = __vmaxu2(__vmaxu2(u.x & 0x7fff7fffu, u.y & 0x7fff7fffu),
                                __vmaxu2(u.z & 0x7fff7fffu, u.w & 0x7fff7fffu));
    const uint32_t a = m << 16, b = m & 0xffff0000u;
    return a > b ? a : b;
  }
  static __device__ __forceinline__ uint32_t four(uint32_t a, uint32_t b, uint64_t inv) {
    return __byte_perm(
        e4m3x2(__uint_as_float(a << 16), __uint_as_float(a & 0xffff0000u), inv),
        e4m3x2(__uint_as_float(b << 16), __uint_as_float(b & 0xffff0000u), inv), 0x5410);
  }
  __device__ __forceinline__ uint2 codes(float inv) const {
    return make_uint2(four(u.x, u.y, both(inv)), four(u.z, u.w, both(inv)));
  }
};
template <>
struct Eight<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float* p) {
    a = *reinterpret_cast<const float4*>(p);
    b = *reinterpret_cast<const float4*>(p + 4);
  }
  __device__ __forceinline__ void load_some(const float* p, int n) {
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < n ? p[i] : 0.f;
    a = make_float4(v[0], v[1], v[2], v[3]);
    b = make_float4(v[4], v[5], v[6], v[7]);
  }
  __device__ __forceinline__ void zero() { a = b = make_float4(0.f, 0.f, 0.f, 0.f); }
  static __device__ __forceinline__ uint32_t mag(float v) { return __float_as_uint(v) & 0x7fffffffu; }
  __device__ __forceinline__ uint32_t top() const {
    return max(max(max(mag(a.x), mag(a.y)), max(mag(a.z), mag(a.w))),
               max(max(mag(b.x), mag(b.y)), max(mag(b.z), mag(b.w))));
  }
  __device__ __forceinline__ uint2 codes(float inv) const {
    const uint64_t i = both(inv);
    return make_uint2(__byte_perm(e4m3x2(a.x, a.y, i), e4m3x2(a.z, a.w, i), 0x5410),
                      __byte_perm(e4m3x2(b.x, b.y, i), e4m3x2(b.z, b.w, i), 0x5410));
  }
};

}  // namespace rc
