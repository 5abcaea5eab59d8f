// How the epilogue warps of the eight-bit products write 32 x 32 chunks of an
// accumulator (lane = row, v = its columns), by way of the warp's own shared
// memory.
#pragma once
#include "common.cuh"
#include "tc_eight_bit.cuh"
#include "tma_host.h"

namespace rc {
namespace tc {

// The instruction descriptor of kind::mxf8f6f4 without its sizes: e4m3 x e4m3
// into f32, both K-major, power-of-two scale bytes; N >> 3 at bit 17, M >> 7 at
// bit 27, the byte of each scale word that the MMA takes at bits 4 (W) and 29 (x).
constexpr uint32_t IDESC_E4M3 = 1u << 23;
constexpr int CHUNK_STAGING = 32 * 128;  // bytes of a warp's chunk at most

// In the layout of a box of 32 columns with a swizzle as wide as its rows
// (which also keeps the row-per-lane writes free of bank conflicts), then by TMA;
// what lies outside y is not written.
template <class T>
__device__ __forceinline__ void store_chunk(const CUtensorMap* map, uint8_t* stg, int lane,
                                            const float* v, int r0, int c0) {
  const uint32_t s0 = saddr(stg);
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(
                       s0 + lane * 128 + 16 * (j ^ (lane & 7))),
                   "f"(v[4 * j]), "f"(v[4 * j + 1]), "f"(v[4 * j + 2]), "f"(v[4 * j + 3])
                   : "memory");
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(
                       s0 + lane * 64 + 16 * (j ^ ((lane >> 1) & 3))),
                   "r"(pack_bf16x2(v[8 * j], v[8 * j + 1])),
                   "r"(pack_bf16x2(v[8 * j + 2], v[8 * j + 3])),
                   "r"(pack_bf16x2(v[8 * j + 4], v[8 * j + 5])),
                   "r"(pack_bf16x2(v[8 * j + 6], v[8 * j + 7]))
                   : "memory");
  }
  fence_proxy_async_smem();
  __syncwarp();
  if (lane == 0) tma_store_2d(map, s0, c0, r0);
}
// Any alignment, the first `rows` rows and `cols` columns at y: neighbouring lanes
// write neighbouring columns.
template <class T>
__device__ __forceinline__ void write_chunk(T* y, int ldy, int rows, int cols, uint8_t* stg,
                                            int lane, const float* v) {
  float* s = reinterpret_cast<float*>(stg);
#pragma unroll
  for (int j = 0; j < 32; ++j) s[lane * 32 + (j ^ lane)] = v[j];
  __syncwarp();
  if (lane < cols) {
    y += lane;
    for (int row = 0; row < min(32, rows); ++row, y += ldy) *y = T(s[row * 32 + (lane ^ row)]);
  }
  __syncwarp();  // the staging area is rewritten by the next chunk
}

// y [rows][n] in boxes of 32 x 32 whose rows are swizzled over their own width.
template <class T>
cudaError_t tma_map_chunks(T* y, int rows, int n, int ld, CUtensorMap* out) {
  auto fn = tma_encode_fn();
  if (!fn) return cudaErrorNotSupported;
  constexpr bool F32 = sizeof(T) == 4;
  const cuuint64_t dims[2] = {cuuint64_t(n), cuuint64_t(rows)};
  const cuuint64_t strides[1] = {cuuint64_t(ld) * sizeof(T)};
  const cuuint32_t box[2] = {32, 32}, es[2] = {1, 1};
  const CUresult r =
      fn(out, F32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, y, dims,
         strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
         F32 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
         CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

}  // namespace tc
}  // namespace rc
