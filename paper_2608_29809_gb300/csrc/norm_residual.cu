// The row work between two products (rc_norm_residual): the weighted sum of
// expert rows, norm, gate and residual of a block's output, and the norm and
// modulation before the next block, in one pass.
#include "../../include/regioncache.h"
#include "block.h"
#include "common.cuh"
#include "fp8.cuh"

namespace rc {

namespace {

// A row is dealt in vectors of eight columns: thread t of the row's TPR holds
// vectors t, t + TPR ..  (NV at most), from the first load to the last store, so
// x and h are read once; the sums of a norm go through the registers that hold
// the row (its variance is that of the differences from the mean, two passes
// there).  Sixteen neighbouring threads hold the 128 columns of a scale.
__device__ __forceinline__ void unpack(const Eight<bf16>& e, float* v) {
  const uint32_t w[4] = {e.u.x, e.u.y, e.u.z, e.u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(w[i] << 16);
    v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void unpack(const Eight<float>& e, float* v) {
  v[0] = e.a.x, v[1] = e.a.y, v[2] = e.a.z, v[3] = e.a.w;
  v[4] = e.b.x, v[5] = e.b.y, v[6] = e.b.z, v[7] = e.b.w;
}
template <class T>
__device__ __forceinline__ void load(Eight<T>& e, const T* p, int n, bool wide) {
  if (wide && n >= 8) e.load(p);
  else if (n > 0) e.load_some(p, n);
  else e.zero();
}
// Eight (n) of a vector of f32 parameters, `rest` where there are none.
__device__ __forceinline__ void parameters(const float* p, int c, int n, float rest, float* v) {
  if (p && n >= 8 && (reinterpret_cast<uintptr_t>(p) & 15) == 0) {
    const float4 a = __ldg(reinterpret_cast<const float4*>(p + c));
    const float4 b = __ldg(reinterpret_cast<const float4*>(p + c) + 1);
    v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w;
    v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = p && k < n ? __ldg(p + c + k) : rest;
  }
}
__device__ __forceinline__ void store(bf16* p, const float* v, int n, bool wide) {
  if (wide && n >= 8) {
    *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]),
                                              pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (k < n) p[k] = f2bf(v[k]);
  }
}
__device__ __forceinline__ void store(float* p, const float* v, int n, bool wide) {
  if (wide && n >= 8) {
    reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (k < n) p[k] = v[k];
  }
}

// Sum over the row's threads; `slots` of the CTA's warps (TPR > 32), used in
// turn so that one barrier a sum is enough.
template <int TPR>
__device__ __forceinline__ float row_sum(float v, float (*slots)[16], int& turn) {
  v = warp_sum(v);
  if (TPR == 32) return v;
  const int warp = threadIdx.x >> 5;
  if ((threadIdx.x & 31) == 0) slots[turn][warp] = v;
  __syncthreads();
  v = 0.f;
#pragma unroll
  for (int w = 0; w < TPR / 32; ++w) v += slots[turn][w];
  turn ^= 1;
  return v;
}

template <int TPR, int NV>
__device__ __forceinline__ void normalise(const NormOf& o, float (*v)[8], int t, int cols,
                                          float (*slots)[16], int& turn) {
  if (o.kind == RC_NORM_NONE) return;
  float mean = 0.f, sum = 0.f;
  if (o.kind == RC_NORM_LAYER) {
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int k = 0; k < 8; ++k) sum += v[i][k];
    mean = row_sum<TPR>(sum, slots, turn) / float(cols);
    sum = 0.f;
  }
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int n = cols - (t + i * TPR) * 8;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      v[i][k] = k < n ? v[i][k] - mean : 0.f;
      sum = fmaf(v[i][k], v[i][k], sum);
    }
  }
  const float r = 1.f / sqrtf(row_sum<TPR>(sum, slots, turn) / float(cols) + o.eps);
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = (t + i * TPR) * 8, n = cols - c;
    if (n <= 0) continue;
    float w[8], b[8];
    parameters(o.weight, c, n, 1.f, w);
    parameters(o.bias, c, n, 0.f, b);
#pragma unroll
    for (int k = 0; k < 8; ++k) v[i][k] = fmaf(v[i][k] * r, w[k], b[k]);
  }
}

// The item that owns `row`, -1 for none, by the whole warp: the last offset that is
// not above the row, a thirty-second of the list at a time.
__device__ __forceinline__ int item_of(const int* offsets, int n_items, int rows, int row) {
  const int lane = threadIdx.x & 31;
  int lo = 0, len = n_items;
  while (len > 1) {
    const int step = (len - 1) / 32 + 1;
    const long long at = (long long)lane * step;
    const bool under = at < len && offsets[lo + int(at)] <= row;
    const int last = 31 - __clz(int(__ballot_sync(0xffffffffu, under)));
    if (last < 0) return -1;
    lo += last * step;
    len = min(step, len - last * step);
  }
  const int first = offsets[lo], end = offsets[lo + 1];
  return first >= 0 && first <= row && row < end && end <= rows ? lo : -1;
}

template <class TX, class TH, int TPR, int NV>
__global__ void __launch_bounds__(TPR == 32 ? 128 : TPR)
norm_residual_kernel(const __grid_constant__ ResidualArgs a) {
  __shared__ float slots[2][16];
  pdl_wait();
  pdl_trigger();
  constexpr int ROWS = TPR == 32 ? 4 : 1;
  const int t = TPR == 32 ? threadIdx.x & 31 : threadIdx.x;
  if (a.row_offsets && blockIdx.x == 0)
    for (int i = threadIdx.x; i < a.n_items; i += blockDim.x)
      if (a.row_offsets[i] < 0 || a.row_offsets[i] > a.row_offsets[i + 1] ||
          a.row_offsets[i + 1] > a.rows)
        atomicOr(a.err, DEVERR_COUNT);
  const long long row = (long long)blockIdx.x * ROWS + (TPR == 32 ? threadIdx.x >> 5 : 0);
  if (row >= a.rows) return;

  const auto wide = [](const void* p, long long ld, int size) {
    return ((reinterpret_cast<uintptr_t>(p) | uintptr_t(ld * size)) & 15) == 0;
  };
  const TX* x = static_cast<const TX*>(a.x);
  const TH* h = static_cast<const TH*>(a.h);
  const bool wide_x = wide(x, a.ldx, sizeof(TX)), wide_h = wide(h, a.ldh, sizeof(TH));
  float v[NV][8], r[NV][8];
  {
    Eight<TX> ex[NV];
    Eight<TH> eh[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (t + i * TPR) * 8;
      load(ex[i], x + row * a.ldx + c, x ? a.cols - c : 0, wide_x);
      load(eh[i], h + row * a.ldh + c, h && a.top_k == 0 ? a.cols - c : 0, wide_h);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) unpack(ex[i], v[i]), unpack(eh[i], r[i]);
  }
  const int item = a.row_offsets ? item_of(a.row_offsets, a.n_items, a.rows, int(row)) : 0;
  if (item < 0) return;  // (the row's threads alike)
  const long long mod = (long long)item * a.ld_mod;

  for (int j = 0; h && j < a.top_k; ++j) {
    const int place = a.places[row * a.top_k + j];
    if (place < 0) continue;
    if (place >= a.h_rows) {
      if (t == 0) atomicOr(a.err, DEVERR_INDEX);
      continue;
    }
    const float w = a.weights[row * a.top_k + j];
    Eight<TH> eh[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (t + i * TPR) * 8;
      load(eh[i], h + (long long)place * a.ldh + c, a.cols - c, wide_h);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      float u[8];
      unpack(eh[i], u);
#pragma unroll
      for (int k = 0; k < 8; ++k) r[i][k] = fmaf(w, u[k], r[i][k]);
    }
  }

  int turn = 0;
  if (h) {
    normalise<TPR, NV>(a.post, r, t, a.cols, slots, turn);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (t + i * TPR) * 8, n = a.cols - c;
      if (n <= 0) continue;
      float g[8];
      parameters(a.gate ? a.gate + mod : nullptr, c, n, 1.f, g);
#pragma unroll
      for (int k = 0; k < 8; ++k)
        v[i][k] = k < n ? fmaf(a.residual_scale, v[i][k], g[k] * r[i][k]) : 0.f;
    }
  } else {
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int k = 0; k < 8; ++k) v[i][k] *= a.residual_scale;
  }
  if (a.x_out) {
    TX* out = static_cast<TX*>(a.x_out);
    const bool wide_out = wide(out, a.ldx_out, sizeof(TX));
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (t + i * TPR) * 8;
      if (c < a.cols) store(out + row * a.ldx_out + c, v[i], a.cols - c, wide_out);
    }
  }
  if (!a.y && !a.y8.codes) return;

  normalise<TPR, NV>(a.pre, v, t, a.cols, slots, turn);
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = (t + i * TPR) * 8, n = a.cols - c;
    if (n > 0) {
      float s[8], b[8];
      parameters(a.scale ? a.scale + mod : nullptr, c, n, 0.f, s);
      parameters(a.shift ? a.shift + mod : nullptr, c, n, 0.f, b);
#pragma unroll
      for (int k = 0; k < 8; ++k) v[i][k] = k < n ? fmaf(v[i][k], 1.f + s[k], b[k]) : 0.f;
    }
    if (a.y8.codes) {
      Eight<float> e;
      e.a = make_float4(v[i][0], v[i][1], v[i][2], v[i][3]);
      e.b = make_float4(v[i][4], v[i][5], v[i][6], v[i][7]);
      if (n <= 0) e.zero();
      uint32_t top = e.top();
#pragma unroll
      for (int o = 8; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
      const int b = scale_byte(top);
      const uint2 q = e.codes(scale_inverse(b));
      uint8_t* dst = a.y8.codes + row * a.y8.ld + c;
      if (n >= 8) {
        *reinterpret_cast<uint2*>(dst) = q;
      } else {
        for (int k = 0; k < n; ++k) dst[k] = uint8_t((k < 4 ? q.x : q.y) >> (8 * (k & 3)));
      }
      if (n > 0 && (t & 15) == 0) a.y8.scales[(long long)(c / 128) * a.y8.lds + row] = uint8_t(b);
    } else if (n > 0) {
      if (a.y_f32) {
        float* y = static_cast<float*>(a.y);
        store(y + row * a.ldy + c, v[i], n, wide(y, a.ldy, 4));
      } else {
        bf16* y = static_cast<bf16*>(a.y);
        store(y + row * a.ldy + c, v[i], n, wide(y, a.ldy, 2));
      }
    }
  }
}

template <class TX, class TH>
cudaError_t go(const ResidualArgs& a, cudaStream_t st) {
  count_launches(1);
  const auto one = [&](void (*kernel)(ResidualArgs), int threads, int rows) {
    return launch_k(kernel, dim3(unsigned((a.rows + (long long)rows - 1) / rows)), dim3(threads),
                    0, st, a);
  };
  if (a.cols <= 1280 && a.rows > 1024) return one(norm_residual_kernel<TX, TH, 32, 5>, 128, 4);
  if (a.cols <= 2048) return one(norm_residual_kernel<TX, TH, 128, 2>, 128, 1);
  if (a.cols <= 5120) return one(norm_residual_kernel<TX, TH, 128, 5>, 128, 1);
  return one(norm_residual_kernel<TX, TH, 512, 4>, 512, 1);
}

}  // namespace

cudaError_t launch_norm_residual(const ResidualArgs& a, cudaStream_t st) {
  if (a.x_f32) return a.h_f32 ? go<float, float>(a, st) : go<float, bf16>(a, st);
  return a.h_f32 ? go<bf16, float>(a, st) : go<bf16, bf16>(a, st);
}

}  // namespace rc
