// Activations of the experts' products.
#pragma once
#include "../../include/regioncache.h"
#include "common.cuh"

namespace rc {

// What a product's results are written as.
enum ExpertsOut { OUT_BF16, OUT_F32, OUT_CODES };

// a b + c, cut to 0 .. 1.
__device__ __forceinline__ float fma_sat(float a, float b, float c) {
  float r;
  asm("fma.rn.sat.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
// v / (1 + 2^e) of four values with one reciprocal, of the product of the
// denominators: the special-function unit, a power and a reciprocal each, is what
// the epilogue waits for.  e is cut to 31 (also that of a NaN, which so leaves the other
// three as they are), so that the product stays finite; a little more than 2^-31 is taken
// off the quotients, so that those that were cut are 0 for v of any size, and the others
// are off by no more than that.  Power and reciprocal are good to a few steps of f32.
__device__ __forceinline__ void over_one_plus(float2& v, float2& w, float2 e, float2 f) {
  const float2 a = f2_add(make_float2(ex2_ftz(fminf(e.x, 31.f)), ex2_ftz(fminf(e.y, 31.f))),
                          f2_of(1.f));
  const float2 b = f2_add(make_float2(ex2_ftz(fminf(f.x, 31.f)), ex2_ftz(fminf(f.y, 31.f))),
                          f2_of(1.f));
  const float2 c = f2_mul(a, b);  // (v.x's and w.x's denominators, v.y's and w.y's)
  const float2 r = f2_mul(f2_of(rcp_ftz(c.x * c.y)), make_float2(c.y, c.x));
  constexpr float LESS = -0x1.002p-31f;
  v = f2_mul(v, make_float2(fma_sat(r.x, b.x, LESS), fma_sat(r.y, b.y, LESS)));
  w = f2_mul(w, make_float2(fma_sat(r.x, a.x, LESS), fma_sat(r.y, a.y, LESS)));
}
// GELU by its sigmoid: (1 + tanh a) / 2 = 1 / (1 + exp(-2 a)).
__device__ __forceinline__ float2 gelu_power(float2 v) {
  const float k = -2.f * 0.7978845608028654f * 1.4426950408889634f;  // sqrt(2 / pi), log2 e
  return f2_mul(v, f2_fma(f2_mul(v, v), f2_of(0.044715f * k), f2_of(k)));
}
__device__ __forceinline__ float2 silu_power(float2 v) {
  return f2_mul(v, f2_of(-1.4426950408889634f));
}
__device__ __forceinline__ float act_of(int act, float v) {
  float2 a = f2_of(v), b = f2_of(0.f);
  if (act == RC_ACT_GELU) over_one_plus(a, b, gelu_power(a), b);
  if (act == RC_ACT_SILU) over_one_plus(a, b, silu_power(a), b);
  return a.x;
}

}  // namespace rc
