// Rotary positions (rc_rotary_plan, rc_rotary_apply).
#include <math.h>

#include "../../include/regioncache.h"
#include "block.h"
#include "common.cuh"

namespace rc {

namespace {

// cos and sin of a place within the turn (a fraction of 2^64).  The nearest
// quarter turn comes off in integers, so nothing is lost; on what is left, at
// most an eighth of a turn, the Taylor series up to the 10th (cos) and 9th
// degree (sin): the next terms are below 2^-32 and 2^-28 of the result.
__device__ __forceinline__ float2 cos_sin(uint64_t place) {
  const uint32_t quarter = uint32_t((place + (uint64_t(1) << 61)) >> 62) & 3u;
  const long long rest = (long long)(place - (uint64_t(quarter) << 62));
  const float t = float(rest) * (6.283185307179586f * 5.421010862427522e-20f);  // 2 pi 2^-64
  const float s = t * t;
  float c = fmaf(s, -1.f / 3628800.f, 1.f / 40320.f);
  c = fmaf(c, s, -1.f / 720.f);
  c = fmaf(c, s, 1.f / 24.f);
  c = fmaf(c, s, -0.5f);
  c = fmaf(c, s, 1.f);
  float n = fmaf(s, 1.f / 362880.f, -1.f / 5040.f);
  n = fmaf(n, s, 1.f / 120.f);
  n = fmaf(n, s, -1.f / 6.f);
  n = fmaf(n * s, t, t);
  const float a = quarter & 1 ? n : c, b = quarter & 1 ? c : n;
  return make_float2(quarter == 1 || quarter == 2 ? -a : a, quarter >= 2 ? -b : b);
}

template <class T, int W>
struct alignas(sizeof(T) * W) Some {
  T v[W];
};
__device__ __forceinline__ float value(float v) { return v; }
__device__ __forceinline__ float value(bf16 v) { return bf2f(v); }
__device__ __forceinline__ void put(float& to, float v) { to = v; }
__device__ __forceinline__ void put(bf16& to, float v) { to = f2bf(v); }

// A CTA turns `per` rows: the cosines and sines of their pairs (the same for all
// heads) go to shared memory, then a thread takes the same unit of one head after
// another.  In a head, units 0 .. pair_units - 1 are turned: with HALF W channels
// and the W that are rot / 2 further, with PAIRS W neighbours (W = 1: a pair); the
// others are W channels that are only copied.  Bound by memory,
// and by a CTA's start, whose first loads wait for the cosines: 16384 rows of 32 x 72, pairs,
// two axes, 31.0 us where 151 MB take 22, 4096 CTAs, 1216 at once (a unit of eight bytes
// found by two divisions: 33; the next unit loaded before this one is turned: 36).
template <class T, int W, bool HALF>
__global__ void __launch_bounds__(256)
rotary_kernel(const __grid_constant__ RotaryArgs a) {
  extern __shared__ float2 turns[];
  pdl_wait();
  pdl_trigger();
  const int half = a.plan.rot / 2;
  const int rows = a.count ? live_count(a.count, a.rows, blockIdx.x == 0 && threadIdx.x == 0
                                                             ? a.err : nullptr) : a.rows;
  const long long row0 = (long long)blockIdx.x * a.per;
  const int here = int(min((long long)a.per, rows - row0));
  if (here <= 0) return;
  for (int i = threadIdx.x; i < here * half; i += blockDim.x) {
    const int r = i / half, p = i - r * half;
    const int axis = (p >= a.plan.pairs[0]) + (p >= a.plan.pairs[0] + a.plan.pairs[1]);
    const long long at = a.positions
                             ? (long long)a.positions[(row0 + r) * a.plan.axes + axis]
                             : row0 + r;
    const float2 cs = cos_sin(uint64_t(at) * a.plan.turns[p]);
    turns[i] = make_float2(a.plan.amplitude * cs.x,
                           a.inverse ? -a.plan.amplitude * cs.y : a.plan.amplitude * cs.y);
  }
  __syncthreads();

  constexpr bool PAIR = !HALF && W > 1;  // (pairs within a unit)
  constexpr int OF = PAIR ? W / 2 : W;   // pairs of a unit
  using Unit = Some<T, W>;
  const int pair_units = half / OF, rest = a.y == a.x ? 0 : (a.head_dim - a.plan.rot) / W;
  const int units = pair_units + rest, first = a.plan.first, apart = HALF ? half : 1;
  const int at_once = max(1, int(blockDim.x) / units);  // heads
  const int slot = int(threadIdx.x) / units;
  const int step_r = at_once / a.heads, step_h = at_once - step_r * a.heads;
  if (slot >= at_once) return;
  // (more units than threads: several for each)
  for (int u = int(threadIdx.x) % units; u < units; u += blockDim.x) {
    const bool copied = u >= pair_units;
    int c = copied ? (u - pair_units) * W : first + u * (PAIR || HALF ? W : 2);
    if (copied && c >= first) c += a.plan.rot;
    int r = slot / a.heads, h = slot - r * a.heads;
    const T* x = static_cast<const T*>(a.x) + row0 * a.ldx + c;
    T* y = static_cast<T*>(a.y) + row0 * a.ldy + c;
    while (r < here) {
      const T* from = x + (long long)r * a.ldx + (long long)h * a.head_dim;
      T* to = y + (long long)r * a.ldy + (long long)h * a.head_dim;
      const float2* cs = turns + r * half + u * OF;
      Unit p = *reinterpret_cast<const Unit*>(from);
      if (copied) {
        *reinterpret_cast<Unit*>(to) = p;
      } else if (PAIR) {
#pragma unroll
        for (int k = 0; k + 1 < W; k += 2) {
          const float va = value(p.v[k]), vb = value(p.v[k + 1]);
          put(p.v[k], va * cs[k / 2].x - vb * cs[k / 2].y);
          put(p.v[k + 1], vb * cs[k / 2].x + va * cs[k / 2].y);
        }
        *reinterpret_cast<Unit*>(to) = p;
      } else {
        Unit q = *reinterpret_cast<const Unit*>(from + apart);
#pragma unroll
        for (int k = 0; k < W; ++k) {
          const float va = value(p.v[k]), vb = value(q.v[k]);
          put(p.v[k], va * cs[k].x - vb * cs[k].y);
          put(q.v[k], vb * cs[k].x + va * cs[k].y);
        }
        *reinterpret_cast<Unit*>(to) = p;
        *reinterpret_cast<Unit*>(to + apart) = q;
      }
      r += step_r, h += step_h;
      if (h >= a.heads) h -= a.heads, ++r;
    }
  }
}

template <class T, int W>
cudaError_t go(RotaryArgs a, cudaStream_t st) {
  const int half = a.plan.rot / 2;
  const int units = half / (a.plan.layout != RC_ROTARY_HALF && W > 1 ? W / 2 : W);
  // rows of a CTA: four units for each thread, but a CTA for each half of an SM first
  const long long most = (a.rows + 303LL) / 304, want = 1 + 1023LL / ((long long)a.heads * units);
  a.per = int(want < most ? want : most);
  if (a.per > 16) a.per = 16;
  const size_t smem = size_t(a.per) * half * sizeof(float2);
  const dim3 grid(unsigned((a.rows + (long long)a.per - 1) / a.per));
  count_launches(1);
  if (a.plan.layout == RC_ROTARY_HALF)
    return launch_k(rotary_kernel<T, W, true>, grid, dim3(256), smem, st, a);
  return launch_k(rotary_kernel<T, W, false>, grid, dim3(256), smem, st, a);
}

template <class T>
cudaError_t widest(const RotaryArgs& a, cudaStream_t st) {
  // channels a thread moves at once: what divides every offset in a row, up to 16 B
  uintptr_t all = (reinterpret_cast<uintptr_t>(a.x) | reinterpret_cast<uintptr_t>(a.y)) / sizeof(T);
  all |= uintptr_t(a.ldx) | uintptr_t(a.ldy) | uintptr_t(a.head_dim) | uintptr_t(a.plan.first) |
         uintptr_t(a.plan.layout == RC_ROTARY_HALF ? a.plan.rot / 2 : a.plan.rot);
  if (sizeof(T) == 2 && all % 8 == 0) return go<T, 8>(a, st);
  if (all % 4 == 0) return go<T, 4>(a, st);
  if (all % 2 == 0) return go<T, 2>(a, st);
  return go<T, 1>(a, st);
}

}  // namespace

cudaError_t launch_rotary(const RotaryArgs& a, cudaStream_t st) {
  return a.f32 ? widest<float>(a, st) : widest<bf16>(a, st);
}

}  // namespace rc
