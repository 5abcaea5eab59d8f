// Attention of few query rows over the paged eight-bit cache (rc_kv8): what
// bounds it is the cache's bytes, read once for each eight or sixteen rows of a
// key head.
//
// A unit is up to 8 NR rows (query, head of the key head's group) of one
// request and key head.  A cluster of CTAs shares the unit's keys, six warps a CTA
// and two CTAs an SM (or twelve and one, where units are few); a warp takes its
// turn of the half blocks (32 tokens: a contiguous run of keys and one of
// values), which bulk copies bring ahead of it into a ring of its own.  Codes
// become f16 exactly in registers and are the A operand of mma.sync (16 keys,
// then 16 channels), the rows N = 8: with rows as M = 16 the same work took
// twice the MMAs and half as many more instructions.  Keys and channels are taken in an order that makes each
// lane's fragment a contiguous piece of a row: a sum's order is free.
//   S^T = K Q^T    maximum and sum of a row over the eight lanes that hold it
//   O^T += V^T P^T  P as B by transposing 8 x 8 tiles in registers
// As in the kernel for many rows, a block's key scale joins the factor of its
// scores and its value scale the exponent of its weights, both relative to
// references that are raised (and O rescaled) only when the weights would
// leave 2^11.  Weights are f16, taken 2^4 up: to 2^15, and exact to 2^-9 of
// themselves down to 2^-20 of that reference.  So that they stay there, a block
// whose value scale lies more than 2^4 below its reference is multiplied apart and
// added in f32: a weight is off by at most 2^-9 of itself or 2^-25 of its row's
// largest.  Causal rows keep
// the value reference of the last block that they see: later ones may have far
// larger values, or none (scale 255: NaN weights for the rows that see the block,
// and its value codes are left out).
// 48 requests of 500 to 12000 tokens, a row each, 32 heads over 8 of 128: 615 MB
// in 101 us, 6.1 TB/s (a copy runs at 6.8).  Sixteen rows of 128 channels want more
// than the 168 registers that two CTAs an SM leave a thread (72 bytes spilled).
#include <math.h>

#include "common.cuh"
#include "eight_bit.h"
#include "fp8.cuh"
#include "per_device.h"
#include "tc_eight_bit.cuh"

namespace rc {

namespace {

using namespace rc::tc;

constexpr int HALF = 32;  // tokens of a ring stage
constexpr int MAX_PARTS = 8;
constexpr int WARPS_OF_TWO = 6;  // of a CTA, two an SM (twice as many of one alone)
constexpr float NO_REF = -1e30f;
// how far scores and value scales may pass their references, and fall below
constexpr float RAISE = 8.f, RAISE_VALUE = 3.f, APART = -4.f;
// weights' exponent beside that
constexpr float WEIGHT_UP = 4.f, PRODUCT_DOWN = 1.f / 16.f;
static_assert(RAISE + RAISE_VALUE + WEIGHT_UP <= 15.f, "f16");

template <int DH, int NR, int W>
struct FCfg {
  static constexpr int ROWS = 8 * NR;
  static constexpr int WARPS = W;
  static constexpr int PART = HALF * DH;       // bytes of a stage's keys
  static constexpr int STAGE = 2 * PART;
  static constexpr int STAGES = DH == 128 ? 2 : DH == 72 ? 3 : 4;
  static constexpr int RING = WARPS * STAGES * STAGE;
  static constexpr int KS = (DH + 15) / 16;    // MMA steps of 16 channels
  static constexpr int MB = (DH + 15) / 16;    // blocks of 16 channels of the result
  static constexpr int PSTRIDE = DH + 4;       // floats of a partial row: channels, max, sum
  static_assert((WARPS * 32 + 1) * 4 <= ROWS * PSTRIDE * 4, "the lengths fit a row's parts");
  static_assert(WARPS * ROWS * PSTRIDE * 4 <= RING, "the warps' parts fit the ring");
  // a row's parts of the cluster's CTAs, in its owner
  static_assert(WARPS * MAX_PARTS <= 96, "part_exponent");
  static constexpr int JOIN = (ROWS + MAX_PARTS) * PSTRIDE * 4;
  static constexpr size_t SMEM = size_t(RING) + JOIN + WARPS * STAGES * 8 + 16;
};

__device__ __forceinline__ void mma_f16(float* c, uint32_t a0, uint32_t a1, uint32_t a2,
                                        uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
      "{%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transposed(uint32_t a) {  // of an 8 x 8 tile of f16
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(a));
  return r;
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
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
__device__ __forceinline__ uint4 lds128(uint32_t a) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
               : "r"(a));
  return v;
}
__device__ __forceinline__ void sts32(uint32_t a, uint32_t v) {
  asm volatile("st.shared.u32 [%0], %1;" ::"r"(a), "r"(v) : "memory");
}
__device__ __forceinline__ void cluster_arrive() {
  asm volatile("barrier.cluster.arrive.release;" ::: "memory");
}
__device__ __forceinline__ void cluster_wait() {
  asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
}

// O^T += V^T P^T of a half block: acc[mb][r] are 16 channels x 8 rows, pf the
// weights of its two 16-key steps; `left` tokens of it are the request's (those
// behind may hold NaN codes).
template <int DH, int NR>
__device__ __forceinline__ void add_values(float (*acc)[NR][4], const uint32_t (*pf)[NR][2],
                                           uint32_t vs, int g, int t, int left) {
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const uint32_t row = vs + (16 * u + t) * DH;
#pragma unroll
    for (int b = 0; b < DH / 64; ++b) {
      uint2 v[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        v[k] = lds64(row + 4 * k * DH + 64 * b + 8 * g);
        if (left < HALF && 16 * u + t + 4 * k >= left) v[k] = make_uint2(0, 0);
      }
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        const uint32_t k0 = w ? v[0].y : v[0].x, k1 = w ? v[1].y : v[1].x;
        const uint32_t k2 = w ? v[2].y : v[2].x, k3 = w ? v[3].y : v[3].x;
#pragma unroll
        for (int p = 0; p < 2; ++p) {
          // the channels 4 w + 2 p and the next of this lane's eight
          const uint32_t sel = p ? 0x7362 : 0x5140;
          uint32_t a0, a1, a2, a3;
          e4m3x4_f16(__byte_perm(k0, k1, sel), a0, a1);
          e4m3x4_f16(__byte_perm(k2, k3, sel), a2, a3);
#pragma unroll
          for (int r = 0; r < NR; ++r)
            mma_f16(acc[4 * b + 2 * w + p][r], a0, a1, a2, a3, pf[u][r][0], pf[u][r][1]);
        }
      }
    }
    if (DH == 72) {
      uint32_t v[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        v[k] = lds8(row + 4 * k * DH + 64 + g);
        if (left < HALF && 16 * u + t + 4 * k >= left) v[k] = 0;
      }
      uint32_t a0, a2;
      e4m3x4_f16(v[0] | v[1] << 8 | v[2] << 16 | v[3] << 24, a0, a2);
#pragma unroll
      for (int r = 0; r < NR; ++r)
        mma_f16(acc[4][r], a0, 0u, a2, 0u, pf[u][r][0], pf[u][r][1]);
    }
  }
}

template <int DH, int NR, int W>
__global__ void __launch_bounds__(W * 32, 2 * WARPS_OF_TWO / W)
few_rows_kernel(const __grid_constant__ Kv8Pool pool, const __grid_constant__ Kv8AttnArgs a,
                int parts, int longest_first) {
  using C = FCfg<DH, NR, W>;
  constexpr int WARPS = C::WARPS;
  extern __shared__ __align__(128) uint8_t smem[];
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + C::RING + C::JOIN);
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
  const int head = blockIdx.y % pool.heads, chunk = blockIdx.y / pool.heads;
  int req = blockIdx.z;
  if (longest_first) {
    // The request of this rank among the lengths (in steps of a half block; the
    // lower number first): a thread ranks each.  No two keys are the same, and
    // places behind the last request hold zeros.
    const uint32_t keys = saddr(smem) + C::RING;
    volatile int* found = reinterpret_cast<volatile int*>(smem + C::RING + WARPS * 32 * 4);
    const int halves = int(threadIdx.x) < a.n ? max(a.lengths[threadIdx.x], 0) / HALF : 0;
    const uint32_t key = uint32_t(min(halves, (1 << 24) - 1)) << 8 | (255 - threadIdx.x);
    sts32(keys + 4 * threadIdx.x, int(threadIdx.x) < a.n ? key : 0u);
    __syncthreads();
    int rank = 0;
#pragma unroll 4
    for (int r = 0; r < a.n; r += 4) {
      const uint4 k = lds128(keys + 4 * r);
      rank += (k.x > key) + (k.y > key) + (k.z > key) + (k.w > key);
    }
    if (int(threadIdx.x) < a.n && rank == int(blockIdx.z)) *found = int(threadIdx.x);
    __syncthreads();
    req = __shfl_sync(0xffffffffu, *found, 0);
  }
  // This warp's half blocks are first + stride i: the table's first entries are
  // asked for beside the request's sizes (an entry that it has no use for is not
  // looked at).
  const int first = part * WARPS + warp, stride = parts * WARPS;
  const int* table = a.table + (long long)req * a.ld_table;
  const auto place = [&](int i) { return (first + i * stride) / (KV8_BLOCK / HALF); };
  const int entry = place(lane) < a.ld_table ? table[place(lane)] : -1;
  const int q0 = a.offsets[req], nq = a.offsets[req + 1] - q0, len = a.lengths[req];
  // (the same for every CTA of a cluster)
  if (q0 < 0 || nq < 0 || nq > a.max_q || q0 > a.q_rows - nq || len < 0 ||
      len > (long long)a.ld_table * KV8_BLOCK) {
    if (threadIdx.x == 0) atomicOr(a.err, DEVERR_COUNT);
    return;
  }
  const int rows = nq * group, row0 = chunk * C::ROWS;  // (below 2^31: the entry point's check)
  if (row0 >= rows || rows > a.most_rows) return;
  if (parts > 1) cluster_arrive();  // (waited for before anything is put into a peer)

  // ---- lane l holds place and scales (-1: none) of half blocks l of the current
  // 32 and of the next 32; the next ones' scales are still on their way
  const int halves = (len + HALF - 1) / HALF;
  const int mine = first < halves ? (halves - first + stride - 1) / stride : 0;
  int page[2], scales, scale_k, scale_v;
  const auto look_up = [&](int b, bool in, int p) {
    page[b] = -1;
    if (!in) return;
    if (p < 0 || p >= pool.blocks) {
      atomicOr(a.err, DEVERR_INDEX);
    } else {
      page[b] = p;
      scale_k = pool.scale[0][(long long)p * pool.heads + head];
      scale_v = pool.scale[1][(long long)p * pool.heads + head];
    }
  };
  const auto looked_up = [&](int b) { return page[b] < 0 ? -1 : scale_v << 8 | scale_k; };
  look_up(0, lane < mine, entry);
  // (i is at most one batch of 32 ahead of the current one)
  const auto issue = [&](int i, int base) {
    if (i >= mine) return;
    const int p0 = __shfl_sync(0xffffffffu, page[0], i & 31);
    const int p1 = __shfl_sync(0xffffffffu, page[1], i & 31);
    const int p = i - base < 32 ? p0 : p1;
    if (p < 0 || lane != 0) return;
    const int h = (first + i * stride) % (KV8_BLOCK / HALF), st = i % C::STAGES;
    const long long at = (((long long)p * pool.heads + head) * KV8_BLOCK + h * HALF) * DH;
    mbar_expect_tx(bar0 + 8 * st, C::STAGE);
    bulk_load(ring + st * C::STAGE, pool.code[0] + at, C::PART, bar0 + 8 * st);
    bulk_load(ring + st * C::STAGE + C::PART, pool.code[1] + at, C::PART, bar0 + 8 * st);
  };
  page[1] = -1;
  for (int i = 0; i < C::STAGES; ++i) issue(i, 0);
  scales = looked_up(0);
  look_up(1, 32 + lane < mine, 32 + lane < mine ? table[place(32 + lane)] : -1);

  // ---- queries as B fragments, row 8 r + g, in the channel order of the keys
  // (step s < 4 of a 64-channel part: channels 16 t + 4 s ..; the last 8 of 72:
  // 4 t .. for t < 2), each row divided by the power of two of its largest
  // magnitude so that it fits f16 (what falls below f16's range there is below
  // 2^-24 of it).  Softmax works on rows 8 r + 2 t + c: their factors come from
  // the lanes that hold them.
  uint32_t qf[C::KS][NR][2];
  float own[NR][2];
  int seen[NR][2], least = len;
#pragma unroll
  for (int r = 0; r < NR; ++r) {
    const int row = row0 + 8 * r + g;
    const bool in = row < rows;
    const int i = in ? row / group : 0;
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
    const int e = min(int(top >> 23), 240);
    const float f = __uint_as_float(uint32_t(254 - e) << 23);
#pragma unroll
    for (int s = 0; s < C::KS; ++s) {
      const float2 lo = unpack_bf16x2(raw[s].x), hi = unpack_bf16x2(raw[s].y);
      qf[s][r][0] = pack_f16(lo.x * f, lo.y * f);
      qf[s][r][1] = pack_f16(hi.x * f, hi.y * f);
    }
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const int er = __shfl_sync(0xffffffffu, e, 4 * (2 * t + c));
      own[r][c] = 1.4426950408889634f * rsqrtf(float(DH)) * scale_value(er);  // in base 2
      const int mr = row0 + 8 * r + 2 * t + c;
      // (rows past the unit's last see what it sees)
      seen[r][c] = a.causal ? max(0, len - nq + min(mr, rows - 1) / group + 1) : len;
      least = min(least, seen[r][c]);
    }
  }
  least = __reduce_min_sync(0xffffffffu, least);

  // (the rows that see a block have seen all before it, so they share `ref`)
  float o[C::MB][NR][4], m[NR][2], l[NR][2], ref = NO_REF, own_ref[NR][2];
#pragma unroll
  for (int r = 0; r < NR; ++r) {
#pragma unroll
    for (int b = 0; b < C::MB; ++b)
#pragma unroll
      for (int j = 0; j < 4; ++j) o[b][r][j] = 0.f;
    m[r][0] = m[r][1] = -INFINITY;
    l[r][0] = l[r][1] = 0.f;
    own_ref[r][0] = own_ref[r][1] = NO_REF;
  }
  uint32_t phases = 0;  // a bit for each stage
  bool ok = true;

  int st = 0;
#pragma unroll 1
  for (int i = 0, base = 0; i < mine; ++i) {
    if (i - base == 32) {
      base += 32;
      page[0] = page[1];
      scales = looked_up(1);
      const int next = base + 32 + lane;
      look_up(1, next < mine, next < mine ? table[place(next)] : -1);
    }
    const int both = __shfl_sync(0xffffffffu, scales, i - base);
    if (both >= 0) {
      const int kb = both & 255, vb = both >> 8;
      const float kf = scale_value(max(kb, vb) == 255 ? 255 : kb);
      const float bv = vb == 255 ? ref : float(vb);
      const int key0 = (first + i * stride) * HALF;
      if (!mbar_sleep_warp(bar0 + 8 * st, (phases >> st) & 1, abort_flag)) { ok = false; break; }
      phases ^= 1u << st;
      const uint32_t ks = ring + st * C::STAGE;
      // ---- scores of 32 keys, 16 an MMA: its row n is key n / 2 + 4 (n % 2)
      // (+ 8 for n >= 8), so that a lane's weights, transposed, belong to keys
      // t, t + 4, t + 8, t + 12 of each sixteen
      float s[2][NR][4];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
#pragma unroll
        for (int r = 0; r < NR; ++r) s[u][r][0] = s[u][r][1] = s[u][r][2] = s[u][r][3] = 0.f;
        const uint32_t row = ks + (16 * u + (g >> 1) + 4 * (g & 1)) * DH;
        uint32_t w[2][(C::KS + 3) & ~3];
#pragma unroll
        for (int k = 0; k < 2; ++k) {  // keys of rows g and g + 8
#pragma unroll
          for (int b = 0; b < DH / 64; ++b) {
            const uint2 x = lds64(row + 8 * k * DH + 64 * b + 16 * t);
            const uint2 y = lds64(row + 8 * k * DH + 64 * b + 16 * t + 8);
            w[k][4 * b] = x.x;
            w[k][4 * b + 1] = x.y;
            w[k][4 * b + 2] = y.x;
            w[k][4 * b + 3] = y.y;
          }
          if (DH == 72) w[k][4] = t < 2 ? lds32(row + 8 * k * DH + 64 + 4 * t) : 0u;
        }
#pragma unroll
        for (int k = 0; k < C::KS; ++k) {
          uint32_t a0, a1, a2, a3;
          e4m3x4_f16(w[0][k], a0, a2);
          e4m3x4_f16(w[1][k], a1, a3);
#pragma unroll
          for (int r = 0; r < NR; ++r)
            mma_f16(s[u][r], a0, a1, a2, a3, qf[k][r][0], qf[k][r][1]);
        }
      }
      // ---- in base 2, hidden ones -infinity; this lane's largest of each row.
      // Place [u][r][2 j + c] is key 16 u + 8 j + g / 2 + 4 (g % 2), row 2 t + c
      const bool whole = least - key0 >= HALF;
      float top[NR][2];
#pragma unroll
      for (int r = 0; r < NR; ++r)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          float f = own[r][c] * kf;
          f = f > 3e38f ? 3e38f : f;  // (an infinite factor would make NaN of a score of 0)
          top[r][c] = -INFINITY;
#pragma unroll
          for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              float& x = s[u][r][2 * j + c];
              x *= f;
              if (!whole &&
                  key0 + 16 * u + 8 * j + (g >> 1) + 4 * (g & 1) >= seen[r][c]) x = -INFINITY;
              top[r][c] = fmaxf(top[r][c], x);
            }
        }
      // ---- references: raised where a row's scores, or the values, pass them
      bool raise = bv > ref + RAISE_VALUE;
#pragma unroll
      for (int r = 0; r < NR; ++r)
#pragma unroll
        for (int c = 0; c < 2; ++c) raise |= top[r][c] > m[r][c] + RAISE;
      if (__any_sync(0xffffffffu, raise)) {
        const float to = bv > ref + RAISE_VALUE ? bv : ref;
        const float values = ref > NO_REF ? ex2_ftz(ref - to) : 1.f;
        ref = to;
#pragma unroll
        for (int r = 0; r < NR; ++r)
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            float x = top[r][c];  // of the eight lanes that hold the row
            x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 4));
            x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 8));
            x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 16));
            x = fmaxf(x, m[r][c]);
            float corr = x == -INFINITY ? 1.f : ex2_ftz(m[r][c] - x);
            m[r][c] = x;
            l[r][c] *= corr;
            if (seen[r][c] > key0) {
              corr *= values;
              own_ref[r][c] = ref;
            }
#pragma unroll
            for (int b = 0; b < C::MB; ++b) {
              o[b][r][c] *= corr;
              o[b][r][2 + c] *= corr;
            }
          }
      }
      // ---- weights: f16 (half a step is 2^-11 of a weight), transposed to B
      const float d = bv - ref;
      const bool apart = d < APART;
      const float dv = (apart ? 0.f : d) + WEIGHT_UP, back = ex2_ftz(-dv);
      uint32_t pf[2][NR][2];
#pragma unroll
      for (int r = 0; r < NR; ++r) {
        float sum[2] = {0.f, 0.f};
        const float m0 = m[r][0] == -INFINITY ? 0.f : m[r][0] - dv;
        const float m1 = m[r][1] == -INFINITY ? 0.f : m[r][1] - dv;
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const float x = ex2_ftz(s[u][r][2 * j] - m0), y = ex2_ftz(s[u][r][2 * j + 1] - m1);
            sum[0] += x;
            sum[1] += y;
            pf[u][r][j] = transposed(pack_f16(x, y));
          }
        // (this lane's keys; the lanes' sums meet at the end)
        l[r][0] += sum[0] * back;
        l[r][1] += sum[1] * back;
      }
      // ---- values
      const int left = len - key0;
      if (vb == 255) {
        // (0 times a NaN code would reach the rows that do not see it)
      } else if (!apart) {
        add_values<DH, NR>(o, pf, ks + C::PART, g, t, left);
      } else {
        float x[C::MB][NR][4];
        const float f = ex2_ftz(fmaxf(d, -126.f));
#pragma unroll
        for (int b = 0; b < C::MB; ++b)
#pragma unroll
          for (int r = 0; r < NR; ++r)
#pragma unroll
            for (int j = 0; j < 4; ++j) x[b][r][j] = 0.f;
        add_values<DH, NR>(x, pf, ks + C::PART, g, t, left);
#pragma unroll
        for (int b = 0; b < C::MB; ++b)
#pragma unroll
          for (int r = 0; r < NR; ++r)
#pragma unroll
            for (int j = 0; j < 4; ++j) o[b][r][j] += f * x[b][r][j];
      }
      __syncwarp();  // the stage has been read
    }
    issue(i + C::STAGES, base);
    if (++st == C::STAGES) st = 0;
  }
  if (!ok) {
    *abort_flag = 1;
    atomicOr(a.err, DEVERR_TIMEOUT);
  }

  // ---- the warps' parts (part_exponent), over the ring: per row its channels,
  // maximum, sum
#pragma unroll
  for (int r = 0; r < NR; ++r)
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
      for (int x = 4; x < 32; x *= 2) l[r][c] += __shfl_xor_sync(0xffffffffu, l[r][c], x);
  __syncthreads();
  float* mine_at = reinterpret_cast<float*>(smem) + warp * C::ROWS * C::PSTRIDE;
#pragma unroll
  for (int r = 0; r < NR; ++r)
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      float* row = mine_at + (8 * r + 2 * t + c) * C::PSTRIDE;
      const float unit = own_ref[r][c] > NO_REF ? scale_value(int(own_ref[r][c])) : 0.f;
      const int e = part_exponent(l[r][c]);
      const float down = __uint_as_float(uint32_t(127 - e) << 23);
      const float o_down = down * PRODUCT_DOWN;
#pragma unroll
      for (int b = 0; b < C::MB; ++b) {
        if (DH == 72 && b == 4) {
          row[64 + g] = o[b][r][c] * o_down * unit;
        } else {  // channels 8 g + 2 (b % 4) and the next of a 64-channel part
          const int ch = 64 * (b >> 2) + 8 * g + 2 * (b & 3);
          row[ch] = o[b][r][c] * o_down * unit;
          row[ch + 1] = o[b][r][2 + c] * o_down * unit;
        }
      }
      if (g == 0) {
        row[DH] = m[r][c] + float(e);
        row[DH + 1] = l[r][c] * down;
      }
    }
  __syncthreads();
  // n parts of a row's channel, `far` floats apart: their common maximum, sum
  // and products
  const auto join = [&](const float* at, int n, int far, int ch, float& top, float& sum) {
    top = -INFINITY;
    for (int p = 0; p < n; ++p) top = fmaxf(top, at[p * far + DH]);
    const float base = top == -INFINITY ? 0.f : top;
    float x = 0.f;
    sum = 0.f;
    for (int p = 0; p < n; ++p) {
      const float f = ex2_ftz(at[p * far + DH] - base);
      x += f * at[p * far + ch];
      sum += f * at[p * far + DH + 1];
    }
    return x;
  };
  const int live = min(C::ROWS, rows - row0);
  const auto write = [&](int row, int ch, float x, float sum) {
    const int i = (row0 + row) / group, h = head * group + row0 + row - i * group;
    a.o[(long long)(q0 + i) * a.ldo + h * DH + ch] = f2bf(sum == 0.f ? 0.f : x / sum);
  };
  const float* warps = reinterpret_cast<const float*>(smem);
  // row r's owner in the cluster is CTA r mod parts, which keeps its parts at
  // [r / parts][part]
  const uint32_t joined = saddr(smem) + C::RING;
  if (parts > 1) cluster_wait();  // (every CTA of the cluster has begun)
  for (int e = threadIdx.x; e < live * DH; e += WARPS * 32) {
    float top, sum;
    const int row = e / DH, ch = e - row * DH;
    const float x = join(warps + row * C::PSTRIDE, WARPS, C::ROWS * C::PSTRIDE, ch, top, sum);
    if (parts == 1) {
      write(row, ch, x, sum);
      continue;
    }
    const uint32_t at = mapa_shared(
        joined + 4 * ((row / parts * parts + part) * C::PSTRIDE), uint32_t(row % parts));
    asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(at + 4 * ch), "f"(x) : "memory");
    if (ch == 0)
      asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(at + 4 * DH), "f"(top),
                   "f"(sum)
                   : "memory");
  }
  if (parts == 1) return;
  cluster_sync();
  const float* parts_at = reinterpret_cast<const float*>(smem + C::RING);
  const int rows_here = live > part ? (live - part + parts - 1) / parts : 0;
  for (int e = threadIdx.x; e < rows_here * DH; e += WARPS * 32) {
    float top, sum;
    const int k = e / DH, ch = e - k * DH;
    const float x = join(parts_at + k * parts * C::PSTRIDE, parts, C::PSTRIDE, ch, top, sum);
    write(k * parts + part, ch, x, sum);
  }
}

constexpr int SMS = 152;

template <int DH, int NR, int W>
cudaError_t launch(const Kv8Pool& pool, const Kv8AttnArgs& a, long long chunks, long long parts,
                   bool longest_first, cudaStream_t st) {
  using C = FCfg<DH, NR, W>;
  RC_TRY(cudaFuncSetAttribute(few_rows_kernel<DH, NR, W>,
                              cudaFuncAttributeMaxDynamicSharedMemorySize, int(C::SMEM)));
  const dim3 grid(unsigned(parts), unsigned(chunks * pool.heads), unsigned(a.n));
  count_launches(1);
  return launch_k_cluster(few_rows_kernel<DH, NR, W>, grid, dim3(W * 32), C::SMEM, int(parts), st,
                          pool, a, int(parts), longest_first ? 1 : 0);
}

// How many clusters of `parts` CTAs of W warps the current device holds at once
// (found out at the first call; -1 where that fails).
template <int DH, int NR, int W>
int clusters_at_once(int parts) {
  static PerDevice<MAX_PARTS + 1> known;
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess) {
    cudaGetLastError();
    return -1;
  }
  return known.get(dev, parts, [&] {
    using C = FCfg<DH, NR, W>;
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = unsigned(parts);
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(unsigned(parts));
    cfg.blockDim = dim3(W * 32);
    cfg.dynamicSmemBytes = C::SMEM;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    int n = -1;
    if (cudaFuncSetAttribute(few_rows_kernel<DH, NR, W>,
                             cudaFuncAttributeMaxDynamicSharedMemorySize,
                             int(C::SMEM)) != cudaSuccess ||
        cudaOccupancyMaxActiveClusters(&n, few_rows_kernel<DH, NR, W>, &cfg) != cudaSuccess) {
      cudaGetLastError();
      return -1;
    }
    return n;
  });
}

template <int DH, int NR>
cudaError_t few(const Kv8Pool& pool, const Kv8AttnArgs& a, cudaStream_t st) {
  constexpr int WARPS = WARPS_OF_TWO, ROWS = FCfg<DH, NR, WARPS>::ROWS;
  const int group = a.heads / pool.heads;
  const long long most_rows = (long long)a.max_q * group;
  const long long chunks =
      ((most_rows < a.most_rows ? most_rows : a.most_rows) + ROWS - 1) / ROWS;
  const long long units = chunks * pool.heads * a.n;
  // CTAs for two an SM at once.  Of requests that may differ, half as long as the
  // longest on average, the longest is done within the others' time when there
  // are about 600 CTAs, as long as a warp keeps 16 half blocks, beside which a
  // CTA's 5 us of start and end count little (16 heads of 72: 8 requests of 4096
  // tokens, one part 23.5 us, two 19.2, three 26.1; 16: one 29.3, two 36.3, but of
  // 500 to 9000 tokens one 54.7, two 35.9, three 41.6; 64 of 100 to 8000: one 96,
  // two 116.  48 of 500 to 12000, 8 key heads of 128: one 117, two 101, three 113).
  // The longest length is what the table holds: 8 requests of 500 tokens take 6.6
  // us with a table of that width and 14.7 with one of 16384 tokens.
  const long long halves = (long long)a.ld_table * (KV8_BLOCK / HALF);
  long long parts = 2 * SMS / units, more = halves / (16 * WARPS);
  if (more > (600 + units / 2) / units) more = (600 + units / 2) / units;
  if (parts > 4 && units * parts > 240) parts = 240 / units;  // (larger clusters need room)
  if (a.n > 1 && parts < more) parts = more;
  if (parts > halves / WARPS) parts = halves / WARPS;
  if (parts > MAX_PARTS) parts = MAX_PARTS;
  if (parts < 1) parts = 1;
  // Where there are few units and much to read, CTAs of twice the warps, one an SM,
  // as many of them a unit as still find a place all at once (16 heads of 72,
  // one row: 4096 tokens 7.1 us with six warps, 6.7 with twelve; 40000: 32.7 and
  // 25.4; clusters that wait for others take twice as long)
  if (units <= 30 && halves > MAX_PARTS * WARPS)
    for (int p = MAX_PARTS; p >= 5; --p)
      if (units <= clusters_at_once<DH, NR, 2 * WARPS>(p))
        return launch<DH, NR, 2 * WARPS>(pool, a, chunks, p, false, st);
  // Where CTAs wait for others' places, the longest requests go first, so that
  // none is left alone at the end (the 48 requests above: 100.9 us, in their own
  // order 114.0; 64 of 2000 tokens each: 58.5 and 55.9)
  const bool longest_first = a.n > 1 && a.n <= WARPS * 32 && units * parts > 2 * SMS;
  return launch<DH, NR, WARPS>(pool, a, chunks, parts, longest_first, st);
}

template <int NR>
cudaError_t few(const Kv8Pool& pool, const Kv8AttnArgs& a, cudaStream_t st) {
  switch (pool.dh) {
    case 64: return few<64, NR>(pool, a, st);
    case 72: return few<72, NR>(pool, a, st);
    default: return few<128, NR>(pool, a, st);
  }
}

}  // namespace

cudaError_t launch_kv8_few(const Kv8Pool& pool, const Kv8AttnArgs& a, cudaStream_t st) {
  if ((long long)a.max_q * (a.heads / pool.heads) <= 8) return few<1>(pool, a, st);
  return few<2>(pool, a, st);
}

}  // namespace rc
