// Activations of the experts' products.
#pragma once
#include "../../include/regioncache.h"
#include "common.cuh"

namespace rc {

// What a product's results are written as.
enum ExpertsOut { OUT_BF16, OUT_F32, OUT_CODES };

// The least of three, or NaN where one is.
__device__ __forceinline__ float min_nan(float a, float b, float c) {
  float r;
  asm("min.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
// v / (1 + 2^e).  Power and reciprocal are good to a few steps of f32, so results of any
// size are as good as e, of which a rounding may lose 2^-24 of itself.
__device__ __forceinline__ float over_one_plus(float v, float e) {
  return v * rcp_ftz(1.f + ex2_ftz(e));
}
// The same of four values, no e above 31, with one reciprocal, of the product of the
// denominators: the special-function unit, a power and a reciprocal each, is what
// the epilogue waits for.
__device__ __forceinline__ void over_one_plus(float2& v, float2& w, float2 e, float2 f) {
  const float2 a = f2_add(make_float2(ex2_ftz(e.x), ex2_ftz(e.y)), f2_of(1.f));
  const float2 b = f2_add(make_float2(ex2_ftz(f.x), ex2_ftz(f.y)), f2_of(1.f));
  const float2 c = f2_mul(a, b);  // (v.x's and w.x's denominators, v.y's and w.y's)
  const float2 r = f2_mul(f2_of(rcp_ftz(c.x * c.y)), make_float2(c.y, c.x));
  v = f2_mul(v, f2_mul(r, b));
  w = f2_mul(w, f2_mul(r, a));
}
// GELU by its sigmoid: (1 + tanh a) / 2 = 1 / (1 + exp(-2 a)).
__device__ __forceinline__ float2 gelu_power(float2 v) {
  const float k = -2.f * 0.7978845608028654f * 1.4426950408889634f;  // sqrt(2 / pi), log2 e
  return f2_mul(v, f2_fma(f2_mul(v, v), f2_of(0.044715f * k), f2_of(k)));
}
__device__ __forceinline__ float2 silu_power(float2 v) {
  return f2_mul(v, f2_of(-1.4426950408889634f));
}
template <bool GELU>
__device__ __forceinline__ float2 power(float2 v) {
  return GELU ? gelu_power(v) : silu_power(v);
}
__device__ __forceinline__ float act_of(int act, float v) {
  if (act == RC_ACT_GELU) return over_one_plus(v, gelu_power(f2_of(v)).x);
  if (act == RC_ACT_SILU) return over_one_plus(v, silu_power(f2_of(v)).x);
  return v;
}
// N values, in fours; where one is so far below zero that its e is above 31, or is no
// number, which would take the other three with it, they go one by one.  (Asked for each
// four: the gated 4128 x 2 rows of 16 experts to codes 63.4 us; now 63.0.)
template <int N, bool GELU>
__device__ __forceinline__ void activate(float* v) {
  float least = v[0];
#pragma unroll
  for (int j = 1; j < N; j += 2) least = min_nan(least, v[j], v[j + 1 < N ? j + 1 : j]);
  if (least >= (GELU ? -5.6f : -21.4f)) {
#pragma unroll
    for (int j = 0; j < N; j += 4) {
      float2 a = make_float2(v[j], v[j + 1]), b = make_float2(v[j + 2], v[j + 3]);
      over_one_plus(a, b, power<GELU>(a), power<GELU>(b));
      v[j] = a.x, v[j + 1] = a.y, v[j + 2] = b.x, v[j + 3] = b.y;
    }
  } else {
#pragma unroll
    for (int j = 0; j < N; j += 2) {
      const float2 e = power<GELU>(make_float2(v[j], v[j + 1]));
      v[j] = over_one_plus(v[j], e.x), v[j + 1] = over_one_plus(v[j + 1], e.y);
    }
  }
}

}  // namespace rc
