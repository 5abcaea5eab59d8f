// Attention over the paged eight-bit cache (rc_kv8).
#include "common.cuh"
#include "fp8.cuh"
#include "kernels.h"

namespace rc {

namespace {

// A warp takes one (query row, head): each lane the scores of its own keys,
// online softmax per lane, joined at the end.
template <int DH>
__global__ void __launch_bounds__(128)
attn_row_kernel(const __grid_constant__ Kv8Pool pool, const __grid_constant__ Kv8AttnArgs a) {
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31;
  const int head = blockIdx.y, req = blockIdx.z, i = blockIdx.x * 4 + (threadIdx.x >> 5);
  const int q0 = a.offsets[req], nq = a.offsets[req + 1] - q0, len = a.lengths[req];
  if (q0 < 0 || nq < 0 || nq > a.max_q || q0 > a.q_rows - nq || len < 0 ||
      len > (long long)a.ld_table * KV8_BLOCK) {
    if (lane == 0) atomicOr(a.err, DEVERR_COUNT);
    return;
  }
  if (i >= nq) return;
  const int kvh = head / (a.heads / pool.heads);
  const bf16* q = a.q + (long long)(q0 + i) * a.ldq + head * DH;
  const int seen = a.causal ? max(0, len - nq + i + 1) : len;
  const float scale = rsqrtf(float(DH));
  float m = -3.0e38f, l = 0.f, o[DH];
#pragma unroll
  for (int c = 0; c < DH; ++c) o[c] = 0.f;
  for (int t = lane; t < seen; t += 32) {
    const int page = a.table[(long long)req * a.ld_table + t / KV8_BLOCK];
    if (page < 0 || page >= pool.blocks) {
      atomicOr(a.err, DEVERR_INDEX);
      continue;
    }
    const long long at = (long long)page * pool.heads + kvh;
    const uint8_t* k = pool.code[0] + (at * KV8_BLOCK + t % KV8_BLOCK) * DH;
    const uint8_t* v = pool.code[1] + (at * KV8_BLOCK + t % KV8_BLOCK) * DH;
    float s = 0.f;
    for (int c = 0; c < DH; c += 2) {
      const float2 x = e4m3x2_f32(*reinterpret_cast<const uint16_t*>(k + c));
      s += x.x * bf2f(q[c]) + x.y * bf2f(q[c + 1]);
    }
    s *= scale_value(pool.scale[0][at]) * scale;
    const float m2 = s > m ? s : m, f = expf(m - m2), p = expf(s - m2);
    const float pv = p * scale_value(pool.scale[1][at]);
    l = l * f + p;
#pragma unroll
    for (int c = 0; c < DH; c += 2) {
      const float2 x = e4m3x2_f32(*reinterpret_cast<const uint16_t*>(v + c));
      o[c] = o[c] * f + pv * x.x;
      o[c + 1] = o[c + 1] * f + pv * x.y;
    }
    m = m2;
  }
  float mm = m;
#pragma unroll
  for (int w = 16; w > 0; w >>= 1) mm = fmaxf(mm, __shfl_xor_sync(0xffffffffu, mm, w));
  const float f = expf(m - mm);
  l = warp_sum(l * f);
  bf16* out = a.o + (long long)(q0 + i) * a.ldo + head * DH;
#pragma unroll
  for (int c = 0; c < DH; ++c) {
    const float s = warp_sum(o[c] * f);
    if (lane == 0) out[c] = f2bf(l == 0.f ? 0.f : s / l);
  }
}

template <int DH>
cudaError_t attention(const Kv8Pool& pool, const Kv8AttnArgs& a, cudaStream_t st) {
  count_launches(1);
  return launch_k(attn_row_kernel<DH>,
                  dim3(unsigned((a.max_q + 3) / 4), unsigned(a.heads), unsigned(a.n)), dim3(128),
                  0, st, pool, a);
}

}  // namespace

cudaError_t launch_kv8_attention(const Kv8Pool& pool, const Kv8AttnArgs& a, cudaStream_t st) {
  if ((long long)a.max_q * (a.heads / pool.heads) <= 64) return launch_kv8_few(pool, a, st);
  switch (pool.dh) {
    case 64: return attention<64>(pool, a, st);
    case 72: return attention<72>(pool, a, st);
    default: return attention<128>(pool, a, st);
  }
}

}  // namespace rc
