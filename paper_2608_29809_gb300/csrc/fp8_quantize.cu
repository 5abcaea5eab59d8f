// Quantised matrices (rc_fp8): the quantiser.
#include "common.cuh"
#include "fp8.cuh"
#include "kernels.h"

namespace rc {

namespace {

constexpr int GROUP = 128;  // columns of a scale

// ------------------------------------------------------------- quantiser
// One scale per row and 128 columns: half a warp takes the 128 values of a
// group (16 lanes of eight values), finds their largest magnitude by four
// shuffles and writes its 128 codes; one pass over x.
template <class T, bool WIDE>
__global__ void __launch_bounds__(256)
quant_rows_kernel(const T* __restrict__ x, int ldx, int rows, int cols, int groups,
                  uint8_t* __restrict__ codes, int ld, uint8_t* __restrict__ scales, int lds) {
  pdl_wait();
  pdl_trigger();
  const int half = (blockIdx.x * 256 + threadIdx.x) >> 4, halves = gridDim.x * 16;
  const int sub = threadIdx.x & 15;
  const long long units = (long long)rows * groups;
  const long long rounds = (units + halves - 1) / halves;
  for (long long it = 0; it < rounds; ++it) {  // (every lane takes part in the shuffles)
    const long long u = it * halves + half;
    const int r = int(u / groups), g = int(u - (long long)r * groups);
    const int c = g * GROUP + sub * 8;
    const int n = u < units ? cols - c : 0;
    Eight<T> v;
    if (WIDE && n >= 8) v.load(x + (long long)r * ldx + c);
    else if (n > 0) v.load_some(x + (long long)r * ldx + c, n);
    else v.zero();
    uint32_t top = v.top();
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
    const int b = scale_byte(top);
    const uint2 q = v.codes(scale_inverse(b));
    uint8_t* dst = codes + (long long)r * ld + c;
    if (n >= 8) {
      *reinterpret_cast<uint2*>(dst) = q;
    } else {
      for (int i = 0; i < n; ++i) dst[i] = uint8_t((i < 4 ? q.x : q.y) >> (8 * (i & 3)));
    }
    if (sub == 0 && u < units) scales[(long long)g * lds + r] = uint8_t(b);
  }
}

// One scale per 128 x 128 values: a CTA holds the block in registers (16
// lanes a row, 16 rows at a time).
template <class T, bool WIDE>
__global__ void __launch_bounds__(256)
quant_blocks_kernel(const T* __restrict__ x, int ldx, int rows, int cols,
                    uint8_t* __restrict__ codes, int ld, uint8_t* __restrict__ scales, int lds) {
  pdl_wait();
  pdl_trigger();
  __shared__ uint32_t tops[8];
  const int sub = threadIdx.x & 15, row0 = threadIdx.x >> 4;
  const int g = blockIdx.y, rb = blockIdx.x;
  const int c = g * GROUP + sub * 8, n = cols - c;
  Eight<T> v[8];
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int r = rb * 128 + i * 16 + row0;
    if (r >= rows || n <= 0) v[i].zero();
    else if (WIDE && n >= 8) v[i].load(x + (long long)r * ldx + c);
    else v[i].load_some(x + (long long)r * ldx + c, n);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, v[i].top());
  top = __reduce_max_sync(0xffffffffu, top);
  if ((threadIdx.x & 31) == 0) tops[threadIdx.x >> 5] = top;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, tops[i]);
  const int b = scale_byte(top);
  const float inv = scale_inverse(b);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int r = rb * 128 + i * 16 + row0;
    if (r >= rows) continue;
    const uint2 q = v[i].codes(inv);
    uint8_t* dst = codes + (long long)r * ld + c;
    if (n >= 8) {
      *reinterpret_cast<uint2*>(dst) = q;
    } else {
      for (int j = 0; j < n; ++j) dst[j] = uint8_t((j < 4 ? q.x : q.y) >> (8 * (j & 3)));
    }
  }
  if (threadIdx.x == 0) scales[(long long)g * lds + rb] = uint8_t(b);
}

template <class T, bool WIDE>
cudaError_t quantize(const T* x, int ldx, const Fp8Mat& out, cudaStream_t st) {
  const int groups = (out.cols + GROUP - 1) / GROUP;
  count_launches(1);
  if (out.group == 1) {
    const long long units = (long long)out.rows * groups;
    const long long ctas = (units + 15) / 16;
    return launch_k(quant_rows_kernel<T, WIDE>, dim3(unsigned(ctas < 152 * 8 ? ctas : 152 * 8)),
                    dim3(256), 0, st, x, ldx, out.rows, out.cols, groups, out.codes, out.ld,
                    out.scales, out.lds);
  }
  return launch_k(quant_blocks_kernel<T, WIDE>,
                  dim3(unsigned((out.rows + 127LL) / 128), unsigned(groups)), dim3(256), 0, st, x,
                  ldx, out.rows, out.cols, out.codes, out.ld, out.scales, out.lds);
}

}  // namespace

cudaError_t launch_fp8_quantize(const void* x, int ldx, bool f32, const Fp8Mat& out,
                                cudaStream_t st) {
  const size_t row = size_t(ldx) * (f32 ? 4 : 2);
  const bool wide = ((reinterpret_cast<uintptr_t>(x) | (out.rows > 1 ? row : 0)) & 15u) == 0;
  if (f32) {
    const float* p = static_cast<const float*>(x);
    return wide ? quantize<float, true>(p, ldx, out, st) : quantize<float, false>(p, ldx, out, st);
  }
  const bf16* p = static_cast<const bf16*>(x);
  return wide ? quantize<bf16, true>(p, ldx, out, st) : quantize<bf16, false>(p, ldx, out, st);
}

}  // namespace rc
