// Quantised matrices (rc_fp8): the quantiser.
#include "common.cuh"
#include "eight_bit.h"
#include "fp8.cuh"

namespace rc {

namespace {

constexpr int GROUP = 128;  // columns of a scale

// ------------------------------------------------------------- quantiser
// One scale per row and 128 columns.  A warp takes four groups of its row, two
// at a time: the 16 lanes of a group hold eight values each, find the largest
// magnitude by four shuffles and write the codes; one pass over x, all its loads
// under way at once.  The scales of a CTA's eight rows leave together.
// (With the groups of all rows dealt one by one, and their scales written byte
// by byte: 4096 x 4608 bf16 15.5 us; now 10.4, 5.5 TB/s.  Eight groups a warp: 10.9,
// and 14.8 against 12.8 at 16384 x 1152, where more of its lanes have nothing.)
constexpr int ROWS = 8, GROUPS = 4;  // of a CTA
template <class T, bool WIDE>
__global__ void __launch_bounds__(32 * ROWS)
quant_rows_kernel(const T* __restrict__ x, int ldx, int rows, int cols, int groups,
                  uint8_t* __restrict__ codes, int ld, uint8_t* __restrict__ scales, int lds) {
  pdl_wait();
  pdl_trigger();
  __shared__ uint8_t s_scale[GROUPS][ROWS];
  const int warp = threadIdx.x >> 5, half = (threadIdx.x >> 4) & 1, sub = threadIdx.x & 15;
  const long long r0 = (long long)blockIdx.x * ROWS, r = r0 + warp;
  const int g0 = blockIdx.y * GROUPS;
  Eight<T> v[GROUPS / 2];
  int n[GROUPS / 2];
#pragma unroll
  for (int i = 0; i < GROUPS / 2; ++i) {
    const int c = (g0 + 2 * i + half) * GROUP + sub * 8;
    n[i] = r < rows ? cols - c : 0;
    if (WIDE && n[i] >= 8) v[i].load(x + r * ldx + c);
    else if (n[i] > 0) v[i].load_some(x + r * ldx + c, n[i]);
    else v[i].zero();
  }
#pragma unroll
  for (int i = 0; i < GROUPS / 2; ++i) {
    uint32_t top = v[i].top();
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
    const int b = scale_byte(top);
    const uint2 q = v[i].codes(scale_inverse(b));
    uint8_t* dst = codes + r * ld + (g0 + 2 * i + half) * GROUP + sub * 8;
    if (n[i] >= 8) {
      *reinterpret_cast<uint2*>(dst) = q;
    } else {
      for (int k = 0; k < n[i]; ++k) dst[k] = uint8_t((k < 4 ? q.x : q.y) >> (8 * (k & 3)));
    }
    if (sub == 0) s_scale[2 * i + half][warp] = uint8_t(b);
  }
  __syncthreads();
  const int k = threadIdx.x % ROWS, g = threadIdx.x / ROWS;
  if (g < GROUPS && g0 + g < groups && r0 + k < rows)
    scales[(long long)(g0 + g) * lds + r0 + k] = s_scale[g][k];
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
  if (out.group == 1)
    return launch_k(quant_rows_kernel<T, WIDE>,
                    dim3(unsigned((out.rows + (long long)ROWS - 1) / ROWS),
                         unsigned((groups + GROUPS - 1) / GROUPS)),
                    dim3(32 * ROWS), 0, st, x, ldx, out.rows, out.cols, groups, out.codes, out.ld,
                    out.scales, out.lds);
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
