// Attention of few query rows over the paged eight-bit cache (rc_kv8): what
// bounds it is the cache's bytes, read once for each sixteen rows of a key head.
//
// A unit is sixteen rows (query, head of the key head's group) of one request
// and key head.  A cluster of up to eight CTAs shares the unit's keys, four
// warps a CTA; a warp takes every fourth half block of its CTA's (32 tokens: a
// contiguous run of keys and one of values), which bulk copies bring ahead of
// it into a ring of its own.  Codes become f16 exactly in registers and go
// through mma.sync with the rows as M = 16 (the tensor memory path has no use
// for a sixteenth of its rows).  Keys and channels are taken in an order that
// makes each lane's fragment a contiguous piece of a row: a sum's order is
// free.  Running maximum and sum per row in f32; a block's key scale joins the
// row's power of two in the exponent of one factor, its value scale multiplies
// the block's products as they are added in f32.  Warps' and CTAs' parts are
// added in their order, through shared memory and the cluster's.
#include <math.h>

#include "common.cuh"
#include "fp8.cuh"
#include "kernels.h"
#include "tc_common.cuh"

namespace rc {

namespace {

using namespace rc::tc;

constexpr int WARPS = 4, ROWS = 16, HALF = 32;  // HALF: tokens of a ring stage

template <int DH>
struct FCfg {
  static constexpr int PART = HALF * DH;       // bytes of a stage's keys
  static constexpr int STAGE = 2 * PART;
  static constexpr int STAGES = DH == 128 ? 3 : 5;
  static constexpr int RING = WARPS * STAGES * STAGE;
  static constexpr int KS = (DH + 15) / 16;    // MMA steps of 16 channels
  static constexpr int NB = DH / 8;            // blocks of 8 channels of the result
  static constexpr int PSTRIDE = DH + 4;       // floats of a partial row: channels, max, sum
  static constexpr int PARTS = WARPS * ROWS * PSTRIDE * 4;  // goes over the ring
  static_assert(PARTS <= RING, "the parts fit the ring");
  static constexpr size_t SMEM = size_t(RING) + WARPS * STAGES * 8 + 16;
};

__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes,
                                          uint32_t bar) {
  asm volatile(
      "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::
          "r"(dst), "l"(src), "r"(bytes), "r"(bar)
      : "memory");
}
__device__ __forceinline__ void mma_f16(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
      "{%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ uint2 lds64(uint32_t a) {
  uint2 v;
  asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a));
  return v;
}
__device__ __forceinline__ uint32_t lds32(uint32_t a) {
  uint32_t v;
  asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(a));
  return v;
}
__device__ __forceinline__ uint32_t lds8(uint32_t a) {
  uint32_t v;
  asm volatile("ld.shared.u8 %0, [%1];" : "=r"(v) : "r"(a));
  return v;
}
__device__ __forceinline__ float lds_cluster(uint32_t a) {
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(a));
  return v;
}

template <int DH>
__global__ void __launch_bounds__(WARPS * 32, 2)
few_rows_kernel(const __grid_constant__ Kv8Pool pool, const __grid_constant__ Kv8AttnArgs a,
                int parts) {
  using C = FCfg<DH>;
  extern __shared__ __align__(128) uint8_t smem[];
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + C::RING);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(bars + WARPS * C::STAGES);
  const int warp = warp_index(), lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const uint32_t ring = saddr(smem) + warp * (C::STAGES * C::STAGE);
  const uint32_t bar0 = saddr(bars) + 8 * warp * C::STAGES;
  if (threadIdx.x == 0) {
    for (int i = 0; i < WARPS * C::STAGES; ++i) mbar_init(saddr(bars) + 8 * i, 1);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncthreads();
  pdl_wait();
  pdl_trigger();
  const int part = parts > 1 ? int(cluster_ctarank()) : 0;
  const int group = a.heads / pool.heads;
  const int head = blockIdx.y % pool.heads, chunk = blockIdx.y / pool.heads, req = blockIdx.z;
  const int q0 = a.offsets[req], nq = a.offsets[req + 1] - q0, len = a.lengths[req];
  // (the same for every CTA of a cluster)
  if (q0 < 0 || nq < 0 || nq > a.max_q || q0 > a.q_rows - nq || len < 0 ||
      len > (long long)a.ld_table * KV8_BLOCK) {
    if (threadIdx.x == 0) atomicOr(a.err, DEVERR_COUNT);
    return;
  }
  const int rows = nq * group, row0 = chunk * ROWS;
  if (row0 >= rows) return;

  // ---- queries: two rows a lane, in the channel order of the key fragments
  // (step s < 4 of a 64-channel part: channels 16 t + 4 s ..; the last 8 of 72:
  // 4 t .. for t < 2), each row divided by the power of two of its largest
  // magnitude so that it fits f16 (what falls below f16's range there is below
  // 2^-24 of it)
  uint32_t qf[C::KS][4];
  int qe[2], seen[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int row = row0 + g + 8 * h;
    const bool in = row < rows;
    const int i = in ? row / group : 0;
    seen[h] = !in ? 0 : a.causal ? max(0, len - nq + i + 1) : len;
    const bf16* q = a.q + (long long)(q0 + i) * a.ldq + (head * group + row - i * group) * DH;
    uint2 raw[C::KS];
    uint32_t top = 0;
#pragma unroll
    for (int s = 0; s < C::KS; ++s) {
      const int c = DH == 72 && s == 4 ? 64 + 4 * t : (s >> 2) * 64 + 16 * t + 4 * (s & 3);
      raw[s] = make_uint2(0, 0);
      if (in && c < DH) raw[s] = *reinterpret_cast<const uint2*>(q + c);
      const uint32_t m = __vmaxu2(raw[s].x & 0x7fff7fffu, raw[s].y & 0x7fff7fffu);
      top = max(top, max(m << 16, m & 0xffff0000u));
    }
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
    qe[h] = min(int(top >> 23), 240);
    const float f = __uint_as_float(uint32_t(254 - qe[h]) << 23);
#pragma unroll
    for (int s = 0; s < C::KS; ++s) {
      const float2 lo = unpack_bf16x2(raw[s].x), hi = unpack_bf16x2(raw[s].y);
      qf[s][h] = pack_f16(lo.x * f, lo.y * f);
      qf[s][2 + h] = pack_f16(hi.x * f, hi.y * f);
    }
  }

  // ---- this warp's half blocks: first + 4 i for i < mine
  const int halves = (len + HALF - 1) / HALF;
  const int h0 = int((long long)part * halves / parts);
  const int h1 = int((long long)(part + 1) * halves / parts);
  const int first = h0 + warp, mine = first < h1 ? (h1 - first + WARPS - 1) / WARPS : 0;
  const int* table = a.table + (long long)req * a.ld_table;
  // lane l holds block and scale bytes of half blocks l of the current 32 and
  // of the next 32
  int page[2], sk[2], sv[2];
  const auto look_up = [&](int from, int b) {
    page[b] = -1;
    sk[b] = sv[b] = 0;
    if (from + lane < mine) {
      const int p = table[(first + (from + lane) * WARPS) / (KV8_BLOCK / HALF)];
      if (p < 0 || p >= pool.blocks) {
        atomicOr(a.err, DEVERR_INDEX);
      } else {
        page[b] = p;
        sk[b] = pool.scale[0][(long long)p * pool.heads + head];
        sv[b] = pool.scale[1][(long long)p * pool.heads + head];
      }
    }
  };
  look_up(0, 0);
  look_up(32, 1);
  // (i is at most one batch of 32 ahead of the current one)
  const auto issue = [&](int i, int base) {
    if (i >= mine) return;
    const int p0 = __shfl_sync(0xffffffffu, page[0], i & 31);
    const int p1 = __shfl_sync(0xffffffffu, page[1], i & 31);
    const int p = i - base < 32 ? p0 : p1;
    if (p < 0 || lane != 0) return;
    const int h = (first + i * WARPS) % (KV8_BLOCK / HALF), st = i % C::STAGES;
    const long long at = (((long long)p * pool.heads + head) * KV8_BLOCK + h * HALF) * DH;
    mbar_expect_tx(bar0 + 8 * st, C::STAGE);
    bulk_load(ring + st * C::STAGE, pool.code[0] + at, C::PART, bar0 + 8 * st);
    bulk_load(ring + st * C::STAGE + C::PART, pool.code[1] + at, C::PART, bar0 + 8 * st);
  };
  for (int i = 0; i < C::STAGES; ++i) issue(i, 0);

  float o[C::NB][4], m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
#pragma unroll
  for (int n = 0; n < C::NB; ++n)
#pragma unroll
    for (int j = 0; j < 4; ++j) o[n][j] = 0.f;
  const float unit = 1.4426950408889634f * rsqrtf(float(DH));  // scores in base 2
  uint32_t phases = 0;  // a bit for each stage
  bool ok = true;

  for (int i = 0, base = 0; i < mine; ++i) {
    if (i - base == 32) {
      base += 32;
      page[0] = page[1];
      sk[0] = sk[1];
      sv[0] = sv[1];
      look_up(base + 32, 1);
    }
    const int src = i - base, st = i % C::STAGES;
    const int p = __shfl_sync(0xffffffffu, page[0], src);
    const int bk = __shfl_sync(0xffffffffu, sk[0], src);
    const int bv = __shfl_sync(0xffffffffu, sv[0], src);
    const int key0 = (first + i * WARPS) * HALF;
    if (p >= 0) {
      if (!mbar_sleep_warp(bar0 + 8 * st, (phases >> st) & 1, abort_flag)) { ok = false; break; }
      phases ^= 1u << st;
      const uint32_t ks = ring + st * C::STAGE, vs = ks + C::PART;
      // ---- scores of 32 keys: place n of 8-key block j is key
      // 16 (j / 2) + 8 (j % 2) + n / 2 + 4 (n % 2), so that a lane's weights
      // belong to keys t, t + 4, t + 8, t + 12 of each sixteen
      float s[4][4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        s[j][0] = s[j][1] = s[j][2] = s[j][3] = 0.f;
        const uint32_t row = ks + (8 * j + (g >> 1) + 4 * (g & 1)) * DH;
        uint32_t w[(C::KS + 3) & ~3];
#pragma unroll
        for (int b = 0; b < DH / 64; ++b) {
          const uint2 x = lds64(row + 64 * b + 16 * t), y = lds64(row + 64 * b + 16 * t + 8);
          w[4 * b] = x.x;
          w[4 * b + 1] = x.y;
          w[4 * b + 2] = y.x;
          w[4 * b + 3] = y.y;
        }
        if (DH == 72) w[4] = t < 2 ? lds32(row + 64 + 4 * t) : 0u;
#pragma unroll
        for (int k = 0; k < C::KS; ++k)
          mma_f16(s[j], qf[k], e4m3x2_f16x2(w[k] & 0xffffu), e4m3x2_f16x2(w[k] >> 16));
      }
      // ---- softmax of the two rows
      float corr[2];
      bool any[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        // 2^(row's exponent + block's) log2(e) / sqrt(DH)
        const int e = qe[h] + bk - 127;
        const float f = bk == 255 ? __uint_as_float(0x7fffffffu)
                        : e < 1   ? 0.f
                                  : unit * __uint_as_float(uint32_t(min(e, 254)) << 23);
        any[h] = seen[h] > key0;
        float top = -INFINITY;
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            float& x = s[j][2 * h + c];
            x = key0 + 8 * j + t + 4 * c < seen[h] ? x * f : -INFINITY;
            top = fmaxf(top, x);
          }
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
        const float next = fmaxf(m[h], top), ref = next == -INFINITY ? 0.f : next;
        corr[h] = ex2_ftz(m[h] - ref);
        m[h] = next;
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            float& x = s[j][2 * h + c];
            x = ex2_ftz(x - ref);
            sum += x;
          }
        l[h] = l[h] * corr[h] + sum;  // (this lane's keys; the lanes' sums meet at the end)
      }
      // ---- values: weights of sixteen keys as A fragments (f16: half a step
      // is 2^-11 of a weight), eight channels at a time as B
      uint32_t pf[2][4];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        pf[u][0] = pack_f16(s[2 * u][0], s[2 * u][1]);
        pf[u][1] = pack_f16(s[2 * u][2], s[2 * u][3]);
        pf[u][2] = pack_f16(s[2 * u + 1][0], s[2 * u + 1][1]);
        pf[u][3] = pack_f16(s[2 * u + 1][2], s[2 * u + 1][3]);
      }
      const float value = scale_value(bv);
      const int left = len - key0;  // (tokens behind the last may hold NaN codes)
      const auto add = [&](int n, const float* x) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            float& y = o[n][2 * h + c];
            y = y * corr[h] + (any[h] ? value * x[2 * h + c] : 0.f);
          }
      };
#pragma unroll
      for (int b = 0; b < DH / 64; ++b) {
#pragma unroll
        for (int w = 0; w < 2; ++w) {
          float x[4][4];
#pragma unroll
          for (int n = 0; n < 4; ++n) x[n][0] = x[n][1] = x[n][2] = x[n][3] = 0.f;
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            uint32_t v[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const int key = 16 * u + t + 4 * k;
              v[k] = lds32(vs + key * DH + 64 * b + 8 * g + 4 * w);
              if (key >= left) v[k] = 0;
            }
            const uint32_t a01 = __byte_perm(v[0], v[1], 0x5140), b01 = __byte_perm(v[0], v[1], 0x7362);
            const uint32_t a23 = __byte_perm(v[2], v[3], 0x5140), b23 = __byte_perm(v[2], v[3], 0x7362);
            mma_f16(x[0], pf[u], e4m3x2_f16x2(a01 & 0xffffu), e4m3x2_f16x2(a23 & 0xffffu));
            mma_f16(x[1], pf[u], e4m3x2_f16x2(a01 >> 16), e4m3x2_f16x2(a23 >> 16));
            mma_f16(x[2], pf[u], e4m3x2_f16x2(b01 & 0xffffu), e4m3x2_f16x2(b23 & 0xffffu));
            mma_f16(x[3], pf[u], e4m3x2_f16x2(b01 >> 16), e4m3x2_f16x2(b23 >> 16));
          }
#pragma unroll
          for (int n = 0; n < 4; ++n) add(8 * b + 4 * w + n, x[n]);
        }
      }
      if (DH == 72) {
        float x[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          uint32_t v[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const int key = 16 * u + t + 4 * k;
            v[k] = lds8(vs + key * DH + 64 + g);
            if (key >= left) v[k] = 0;
          }
          mma_f16(x, pf[u], e4m3x2_f16x2(v[0] | v[1] << 8), e4m3x2_f16x2(v[2] | v[3] << 8));
        }
        add(C::NB - 1, x);
      }
      __syncwarp();  // the stage has been read
    }
    issue(i + C::STAGES, base);
  }
  if (!ok) {
    *abort_flag = 1;
    atomicOr(a.err, DEVERR_TIMEOUT);
  }

  // ---- the warps' parts, over the ring: per row its channels, maximum, sum
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    l[h] += __shfl_xor_sync(0xffffffffu, l[h], 1);
    l[h] += __shfl_xor_sync(0xffffffffu, l[h], 2);
  }
  __syncthreads();
  float* mine_at = reinterpret_cast<float*>(smem) + warp * ROWS * C::PSTRIDE;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    float* r = mine_at + (g + 8 * h) * C::PSTRIDE;
#pragma unroll
    for (int n = 0; n < C::NB; ++n)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const int place = 2 * t + c;  // the result's column of its 8-channel block
        const int ch = DH == 72 && n == 8 ? 64 + place : (n >> 3) * 64 + 8 * place + (n & 7);
        r[ch] = o[n][2 * h + c];
      }
    if (t == 0) {
      r[DH] = m[h];
      r[DH + 1] = l[h];
    }
  }
  __syncthreads();
  const auto join = [&](int row, int ch, int n, auto at, float& top, float& sum) {
    // n parts of a row's channel: their common maximum, sum and products
    top = -INFINITY;
    for (int p = 0; p < n; ++p) top = fmaxf(top, at(p, row, DH));
    const float ref = top == -INFINITY ? 0.f : top;
    float x = 0.f;
    sum = 0.f;
    for (int p = 0; p < n; ++p) {
      const float f = ex2_ftz(at(p, row, DH) - ref);
      x += f * at(p, row, ch);
      sum += f * at(p, row, DH + 1);
    }
    return x;
  };
  const int live = min(ROWS, rows - row0);
  const auto write = [&](int row, int ch, float x, float sum) {
    const int i = (row0 + row) / group, h = head * group + row0 + row - i * group;
    a.o[(long long)(q0 + i) * a.ldo + h * DH + ch] = f2bf(sum == 0.f ? 0.f : x / sum);
  };
  const float* warps = reinterpret_cast<const float*>(smem);
  const auto of_warp = [&](int p, int row, int c) {
    return warps[(p * ROWS + row) * C::PSTRIDE + c];
  };
  if (parts == 1) {
    for (int e = threadIdx.x; e < live * DH; e += WARPS * 32) {
      float top, sum;
      const float x = join(e / DH, e % DH, WARPS, of_warp, top, sum);
      write(e / DH, e % DH, x, sum);
    }
    return;
  }
  // the CTA's part, behind the warps'
  float* cta = reinterpret_cast<float*>(smem) + WARPS * ROWS * C::PSTRIDE;
  static_assert(C::PARTS + ROWS * C::PSTRIDE * 4 <= C::RING, "the CTA's part fits the ring");
  for (int e = threadIdx.x; e < live * DH; e += WARPS * 32) {
    float top, sum;
    const int row = e / DH, ch = e % DH;
    cta[row * C::PSTRIDE + ch] = join(row, ch, WARPS, of_warp, top, sum);
    if (ch == 0) {
      cta[row * C::PSTRIDE + DH] = top;
      cta[row * C::PSTRIDE + DH + 1] = sum;
    }
  }
  cluster_sync();
  const uint32_t base = saddr(cta);
  const auto of_cta = [&](int p, int row, int c) {
    return lds_cluster(mapa_shared(base + 4 * (row * C::PSTRIDE + c), uint32_t(p)));
  };
  for (int e = part * WARPS * 32 + threadIdx.x; e < live * DH; e += parts * WARPS * 32) {
    float top, sum;
    const float x = join(e / DH, e % DH, parts, of_cta, top, sum);
    write(e / DH, e % DH, x, sum);
  }
  cluster_sync();  // (no CTA leaves while its part may be read)
}

constexpr int SMS = 152;

template <int DH>
cudaError_t few(const Kv8Pool& pool, const Kv8AttnArgs& a, cudaStream_t st) {
  using C = FCfg<DH>;
  RC_TRY(cudaFuncSetAttribute(few_rows_kernel<DH>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                              int(C::SMEM)));
  const int group = a.heads / pool.heads;
  const long long chunks = ((long long)a.max_q * group + ROWS - 1) / ROWS;
  const long long units = chunks * pool.heads * a.n;
  // Enough CTAs for two an SM, several times over where lengths may differ,
  // and no fewer than four half blocks a warp
  long long parts = (2 * SMS * (a.n > 1 ? 4 : 1)) / units;
  const long long most = (long long)a.ld_table * (KV8_BLOCK / HALF) / (4 * WARPS);
  if (parts > most) parts = most;
  if (parts > 8) parts = 8;
  if (parts < 1) parts = 1;
  if (chunks * pool.heads > 65535) return cudaErrorInvalidConfiguration;
  const dim3 grid(unsigned(parts), unsigned(chunks * pool.heads), unsigned(a.n));
  count_launches(1);
  return launch_k_cluster(few_rows_kernel<DH>, grid, dim3(WARPS * 32), C::SMEM, int(parts), st,
                          pool, a, int(parts));
}

}  // namespace

cudaError_t launch_kv8_few(const Kv8Pool& pool, const Kv8AttnArgs& a, cudaStream_t st) {
  switch (pool.dh) {
    case 64: return few<64>(pool, a, st);
    case 72: return few<72>(pool, a, st);
    default: return few<128>(pool, a, st);
  }
}

}  // namespace rc
