// Attention of many query rows over the paged eight-bit cache (rc_kv8), on the
// tensor cores (tcgen05, scores and results in tensor memory).
//
// A unit is up to 256 rows (query, head of the key head's group) of one
// request and key head: two tiles of 128 rows that share every key block of
// 128 tokens (two cache blocks), or one tile whose key blocks two streams take
// in turn.  A cluster of CTAs may share the unit's keys.
//   warps 0-3, 4-7   softmax of a stream, one thread a row: S from tensor
//                    memory, weights back over it as bf16, a cache block (64
//                    tokens) at a time; the other half of S meanwhile takes
//                    the next one's scores
//   warps 8-10       key codes to operands in shared memory: f16 (exact),
//                    K-major, 128-byte swizzle
//   warps 12-14      value codes: bf16 (exact), MN-major, 128-byte swizzle
//   warp 11          issues S = Q K^T (kind f16) and O += P V (kind bf16)
//   warp 15          bulk copies of the codes into a ring ahead of the converters
// Each code is converted once for 256 rows, so its four instructions or so
// stay beside the softmax; a pass that wrote bf16 copies for the kernel of
// rc_attention would move five bytes for each one.  Q is f16 over the power of
// two of its row's largest magnitude, and stays in tensor memory where that
// has room (head_dim 64 and 72: then an MMA reads only the keys from shared
// memory).  A block's key scale joins the factor of its scores, its value
// scale the exponent of its weights (relative to a reference kept per stream),
// so that both cost nothing per element; bf16 weights have f32's range.
// The maximum is taken in a row's first cache block only: later ones use the
// same reference unless their weights' sum passes 2^20 (or a value scale passes
// 2^5 of its reference); then it is raised, O rescaled, the block done again.
// 8 requests of 4096 tokens, 201 to 831 rows, 16 heads of 72: 123 us, 627 TFLOP/s,
// the tensor pipe busy 38 % of the time; 4 of 512 rows, 32 heads over 8 of 128: 142
// us, 905 TFLOP/s.  Softmax and conversion fill half the issue slots: it is
// their chain with the products, page by page, that bounds it.
#include <math.h>

#include "common.cuh"
#include "eight_bit.h"
#include "fp8.cuh"
#include "tc_eight_bit.cuh"

namespace rc {

namespace {

using namespace rc::tc;

constexpr int BQ = 128, BKV = 128, THREADS = 512;
// (warpgroups 2 and 3: three converting warps each, of keys and of values, and
// one of these)
constexpr int CONV_WARP = 8, MMA_WARP = 11, LOAD_WARP = 15, CONV_THREADS = 96;
// Registers: 512 threads are launched with 128 each; the softmax's two
// warpgroups take 160, the other two keep 96 (asked for by each warpgroup in one
// place, ahead of its warps' roles).
constexpr int SOFT_REGS = 160, OTHER_REGS = 96;
constexpr int PAGES = BKV / KV8_BLOCK;
// what the rows share of a cache block: the key scale (NaN where a block has no
// value) and the value scale's exponent (ABSENT: the block is missing)
constexpr float ABSENT = -2e30f, NO_REF = -1e30f;
// S (P over it) of each stream, then O, then Q where it fits
constexpr int TMEM_COLS = 512, TM_O = 2 * BKV;
// The values' operand is 2^-120 of the values, so weights are taken 2^100 up,
// which leaves them 2^27: to raised sums of 2^20 and value scales 2^5 above
// their reference.
constexpr float WEIGHT_UP = 100.f, VALUE_DOWN = 1048576.f;  // 2^100, 2^(120 - 100)
constexpr float RAISE_SUM = 1048576.f, RAISE_VALUE = 5.f;


template <int DH>
struct MCfg {
  static constexpr bool TAIL = DH == 72;
  static constexpr int ATOMS = (DH + 63) / 64;       // 64-channel parts of a V row
  static constexpr int FULL = DH / 64;               // 64-channel parts of a K row
  static constexpr int ODIM = TAIL ? 80 : DH;        // columns of O
  static constexpr int KSTEPS = (DH + 15) / 16;
  static constexpr int TM_Q = TM_O + 2 * ODIM, Q_COLS = 8 * KSTEPS;
  static constexpr bool Q_TMEM = TM_Q + 2 * Q_COLS <= TMEM_COLS;
  static constexpr int Q_BYTES = Q_TMEM ? 0 : FULL * BQ * 128;
  static constexpr int K_BYTES = FULL * BKV * 128 + (TAIL ? BKV * 32 : 0);
  static constexpr int V_BYTES = ATOMS * BKV * 128;
  static constexpr int KST = DH == 128 ? 2 : 3, VST = DH == 128 ? 2 : 3;
  // codes of a key block's keys, then its values, .. in a ring
  static constexpr int RAW_BYTES = BKV * DH, RAWS = DH == 128 ? 2 : 4;
  static constexpr int OPERANDS = 2 * Q_BYTES + KST * K_BYTES + VST * V_BYTES;
  static constexpr int RING = OPERANDS + RAWS * RAW_BYTES;
  // facts of a CTA's first cache blocks, kept in shared memory (those of later
  // ones are read where they are needed)
  static constexpr int FACTS = DH == 128 ? 128 : 256;
  static constexpr size_t SMEM = size_t(RING) + FACTS * 8 + 1024 + 256 + 128;
  // conversion: threads of a row, 8-code pieces of a thread, rows at a time (a
  // multiple of 8, so that a piece keeps its place in the swizzle)
  static constexpr int ROW_THREADS = DH == 72 ? 3 : 4;
  static constexpr int PIECES = DH / 8 / ROW_THREADS, PASS = CONV_THREADS / ROW_THREADS;
  static_assert(PASS % 8 == 0 && PIECES * ROW_THREADS * 8 == DH, "conversion");
  static constexpr uint32_t IDESC_S = (1u << 4) | (uint32_t(KV8_BLOCK >> 3) << 17) | (uint32_t(BQ >> 4) << 24);
  static constexpr uint32_t IDESC_PV = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 16) |
                                       (uint32_t(ODIM >> 3) << 17) | (uint32_t(BQ >> 4) << 24);
  static constexpr int PSTRIDE = DH + 4;             // floats of a partial row
  static_assert(Q_TMEM || !TAIL, "queries in shared memory have no tail");
  static_assert((2 * BQ + 16) * PSTRIDE * 4 <= RING, "the parts fit the operands' memory");
  static_assert(TM_O + 2 * ODIM <= TMEM_COLS, "tensor memory");
};

__device__ __forceinline__ uint64_t pair64(float lo, float hi) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ float2 split64(uint64_t v) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
  return r;
}
__device__ __forceinline__ void sts128(uint32_t at, uint32_t a, uint32_t b, uint32_t c,
                                       uint32_t d) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(a), "r"(b), "r"(c),
               "r"(d)
               : "memory");
}
// Four codes as bf16, times 2^-120: the pairs (0, 2) and (1, 3).  A code's bits
// below its sign, seven places down a bf16, are its value so far down
// (subnormals included).  (A NaN code becomes a number: blocks without value
// have a NaN scale.)
__device__ __forceinline__ uint32_t codes_02(uint32_t u) {
  return ((u << 8) & 0x80008000u) | ((u << 4) & 0x07f007f0u);
}
__device__ __forceinline__ uint32_t codes_13(uint32_t u) {
  return (u & 0x80008000u) | ((u >> 4) & 0x07f007f0u);
}
// Place of channel c among O's columns (the pairs above).
__device__ __forceinline__ constexpr int o_column(int c) {
  return (c & ~3) | ((c & 1) << 1) | ((c >> 1) & 1);
}

__device__ __forceinline__ void soft_sync() { asm volatile("bar.sync 1, 256;" ::: "memory"); }


// A row's 64 scores of a cache block, r, to weights 2^(s f + shift), two a word
// as bf16 in w (times `less`, where FAST is false: then columns from `limit` on
// are hidden).  `total` gets their sums before that.  w may be r: a word is
// written behind the scores it is made of.
template <bool FAST>
__device__ __forceinline__ void weights(const uint32_t* r, uint32_t* w, float f, float shift,
                                        int limit, float less, uint64_t* total) {
  const uint64_t ff = pair64(f, f), sh = pair64(shift, shift);
#pragma unroll
  for (int c = 0; c < KV8_BLOCK; c += 2) {
    float2 y = split64(fma2(pair64(__uint_as_float(r[c]), __uint_as_float(r[c + 1])), ff, sh));
    if (!FAST) {
      if (c >= limit) y.x = -INFINITY;
      if (c + 1 >= limit) y.y = -INFINITY;
    }
    y.x = ex2_ftz(y.x);
    y.y = ex2_ftz(y.y);
    total[(c >> 1) & 1] = add2(total[(c >> 1) & 1], pair64(y.x, y.y));
    if (!FAST) {
      y.x *= less;
      y.y *= less;
    }
    w[c >> 1] = pack_bf16x2(y.x, y.y);
  }
}

// Into this or another CTA's shared memory.
__device__ __forceinline__ void store_four(uint32_t at, const float* v) {
  asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(at), "f"(v[0]), "f"(v[1]),
               "f"(v[2]), "f"(v[3])
               : "memory");
}
__device__ __forceinline__ void store_two(uint32_t at, float a, float b) {
  asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(at), "f"(a), "f"(b) : "memory");
}

// how a CTA finds its unit
constexpr int IN_PLACE = 0, BY_WORK = 1, COUNTED = 2;
constexpr int MAX_RANKED = 64;  // requests BY_WORK

template <int DH>
__global__ void __launch_bounds__(THREADS, 1)
many_rows_kernel(const __grid_constant__ Kv8Pool pool, const __grid_constant__ Kv8AttnArgs a,
                 int parts, int unit_rows, int order) {
  using C = MCfg<DH>;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                             ~uintptr_t(1023));
  float2* facts = reinterpret_cast<float2*>(smem + C::RING);
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + C::RING + C::FACTS * 8);
  const uint32_t sq = saddr(smem), sk = sq + 2 * C::Q_BYTES, sv = sk + C::KST * C::K_BYTES;
  const uint32_t bar = saddr(bars);
  const uint32_t k_full = bar, k_empty = k_full + 8 * C::KST, v_full = k_empty + 8 * C::KST;
  const uint32_t v_empty = v_full + 8 * C::VST, s_full = v_empty + 8 * C::VST;
  // (per cache block of the two that S holds, and stream)
  const uint32_t p_full = s_full + 16 * PAGES, o_done = p_full + 16 * PAGES, o_full = o_done + 16;
  const uint32_t q_full = o_full + 16, raw_full = q_full + 8, raw_empty = raw_full + 8 * C::RAWS;
  const uint32_t raw = sq + C::OPERANDS;
  uint32_t* tmem_slot =
      reinterpret_cast<uint32_t*>(bars + 2 * C::KST + 2 * C::VST + 5 + 4 * PAGES + 2 * C::RAWS);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  int *sums = reinterpret_cast<int*>(tmem_slot + 2), *found = sums + THREADS / 32;
  const int warp = warp_index(), lane = threadIdx.x & 31;

  pdl_wait();
  pdl_trigger();
  const int part = parts > 1 ? int(cluster_ctarank()) : 0;
  const int group = a.heads / pool.heads, place = int(blockIdx.x) / parts;
  const auto rows_of = [&](int r, bool report) {
    const int first = a.offsets[r], count = a.offsets[r + 1] - first, tokens = a.lengths[r];
    if (first < 0 || count < 0 || count > a.max_q || first > a.q_rows - count || tokens < 0 ||
        tokens > (long long)a.ld_table * KV8_BLOCK) {
      if (report) atomicOr(a.err, DEVERR_COUNT);
      return 0;
    }
    return count * group >= a.least_rows ? count * group : 0;
  };
  int head, req, chunk;  // (the same for every CTA of a cluster)
  if (order == IN_PLACE) {
    // a place for each chunk that a request may have, key head and request
    req = place % a.n;
    head = place / a.n % pool.heads;
    chunk = place / a.n / pool.heads;
    if (chunk * unit_rows >= rows_of(req, threadIdx.x == 0)) return;
  } else if (order == BY_WORK) {
    // Units in the order of their work, the key heads of each together: a
    // request has whole ones and perhaps a shorter last one, a thread counts the
    // units before each of the two (no two keys are the same).
    head = place % pool.heads;
    const int unit = place / pool.heads, e = int(threadIdx.x), r = e >> 1;
    const bool last = e & 1;
    uint2* works = reinterpret_cast<uint2*>(smem);
    int rows = 0, count = 0;
    uint32_t key = 0;
    if (e < 2 * a.n) {
      rows = rows_of(r, blockIdx.x == 0);
      count = last ? (rows % unit_rows ? 1 : 0) : rows / unit_rows;
      // blocks, one stream's at three quarters of two's, and what a unit starts with
      const int blocks = min(max(a.lengths[r], 0), 1 << 28) / BKV;
      const int per = (last ? rows % unit_rows : unit_rows) > BQ ? 4 : 3;
      key = uint32_t(blocks * per + 12) << 7 | uint32_t(127 - e);
      works[e] = make_uint2(key, count);
    }
    if (e == 0) found[0] = -1;
    __syncthreads();
    if (e < 2 * a.n) {
      int before = 0;
#pragma unroll 4
      for (int i = 0; i < 2 * a.n; ++i) {
        const uint2 w = works[i];
        before += w.x > key ? int(w.y) : 0;
      }
      if (unit >= before && unit < before + count) {
        found[0] = r;
        found[1] = last ? rows / unit_rows : count - 1 - (unit - before);
      }
    }
    fence_proxy_async_smem();  // (copies come where the keys were)
    __syncthreads();
    req = __shfl_sync(0xffffffffu, found[0], 0);
    chunk = __shfl_sync(0xffffffffu, found[1], 0);
    if (req < 0) return;
  } else {
    // Whole units first, then the requests' short last ones, the key heads of each
    // together.  This place's is found by counting (as many requests at a time as
    // the CTA has threads).  A bad request has none, and is reported.
    head = place % pool.heads;
    const int unit = place / pool.heads;
    int whole = 0;  // units, of all requests
    for (int r = int(threadIdx.x); r < a.n; r += THREADS)
      whole += rows_of(r, blockIdx.x == 0) / unit_rows;
    whole = __reduce_add_sync(0xffffffffu, whole);
    if (lane == 0) sums[warp] = whole;
    if (threadIdx.x == 0) found[0] = -1;
    __syncthreads();
    whole = 0;
    for (int i = 0; i < THREADS / 32; ++i) whole += sums[i];
    const bool last = unit >= whole;
    const int wanted = last ? unit - whole : unit;
    int before = 0;  // such units of the requests counted so far
    for (int r0 = 0; r0 < a.n; r0 += THREADS) {
      const int r = r0 + int(threadIdx.x), rows = r < a.n ? rows_of(r, false) : 0;
      const int units = last ? (rows % unit_rows ? 1 : 0) : rows / unit_rows;
      int incl = units;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += v;
      }
      __syncthreads();  // (what `sums` had before has been read)
      if (lane == 31) sums[warp] = incl;
      __syncthreads();
      int at = before + incl - units;
      for (int i = 0; i < THREADS / 32; ++i) {
        if (i < warp) at += sums[i];
        before += sums[i];
      }
      if (wanted >= at && wanted < at + units) {
        found[0] = r;
        found[1] = last ? rows / unit_rows : wanted - at;
      }
      if (wanted < before) break;
    }
    __syncthreads();
    req = __shfl_sync(0xffffffffu, found[0], 0);
    chunk = __shfl_sync(0xffffffffu, found[1], 0);
    if (req < 0) return;
  }
  const int q0 = a.offsets[req], nq = a.offsets[req + 1] - q0, len = a.lengths[req];
  const int all = nq * group, row0 = chunk * unit_rows;  // (below 2^31: the entry point's check)
  const int rows = min(all - row0, unit_rows);
  const bool two = rows > BQ;

  if (threadIdx.x == 0) {
    for (int i = 0; i < C::KST; ++i) {
      mbar_init(k_full + 8 * i, 3);
      mbar_init(k_empty + 8 * i, 1);
    }
    for (int i = 0; i < C::VST; ++i) {
      mbar_init(v_full + 8 * i, 3);
      mbar_init(v_empty + 8 * i, 1);
    }
    for (int x = 0; x < 2; ++x) {
      for (int h = 0; h < PAGES; ++h) {
        mbar_init(s_full + 16 * h + 8 * x, 1);
        mbar_init(p_full + 16 * h + 8 * x, 4);
      }
      mbar_init(o_done + 8 * x, 1);
      mbar_init(o_full + 8 * x, 1);
    }
    for (int i = 0; i < C::RAWS; ++i) {
      mbar_init(raw_full + 8 * i, 1);
      mbar_init(raw_empty + 8 * i, 3);
    }
    mbar_init(q_full, 8);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (C::TAIL) {  // channels 72 .. 79 of the products are zeros
    for (int i = threadIdx.x; i < C::KST * BKV * 2; i += THREADS)
      sts128(sk + (i / (2 * BKV)) * C::K_BYTES + BKV * 128 + (i % (2 * BKV)) * 16, 0, 0, 0, 0);
    fence_proxy_async_smem();
  }
  if (warp == MMA_WARP) tmem_alloc(saddr(tmem_slot), TMEM_COLS);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;

  // the tokens that the unit's last row sees, in key blocks b0 .. b0 + nb - 1
  // of this CTA
  const int last_query = (row0 + rows - 1) / group;
  const int reach = a.causal ? max(0, len - nq + last_query + 1) : len;
  const int blocks = (reach + BKV - 1) / BKV;
  const int b0 = part * blocks / parts, nb = (part + 1) * blocks / parts - b0;
  const int pages = (len + KV8_BLOCK - 1) / KV8_BLOCK;
  const int* table = a.table + (long long)req * a.ld_table;
  // the table's entry of cache block p, and later, where its value is there, its
  // place in the pool (-1: none)
  const auto entry = [&](int p) { return p < pages ? table[p] : -1; };
  const auto checked = [&](int e) { return e < pool.blocks ? max(e, -1) : -1; };
  bool ok = true;

  if (warp < CONV_WARP) {
    // -------------------------------------------------------------- softmax
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(SOFT_REGS));
    const int x = warp >> 2, tr = threadIdx.x & 127;  // stream, row of its tile
    const int ur = (two ? x * BQ : 0) + tr;           // row of the unit
    const bool in = ur < rows;
    const int query = (row0 + (in ? ur : 0)) / group;
    const int gh = row0 + (in ? ur : 0) - query * group;
    // (rows past the unit's last see what it sees: their warp need not mask)
    const int seen = !in ? reach : a.causal ? max(0, len - nq + query + 1) : len;
    // ---- the row's queries, f16 over the power of two of their largest
    int qe;
    {
      const bf16* q = a.q + (long long)(q0 + query) * a.ldq + (head * group + gh) * DH;
      uint32_t top = 0;
#pragma unroll
      for (int c = 0; c < DH / 8; ++c) {
        const uint4 v = in ? *reinterpret_cast<const uint4*>(q + 8 * c) : make_uint4(0, 0, 0, 0);
        const uint32_t m = __vmaxu2(__vmaxu2(v.x & 0x7fff7fffu, v.y & 0x7fff7fffu),
                                    __vmaxu2(v.z & 0x7fff7fffu, v.w & 0x7fff7fffu));
        top = max(top, max(m << 16, m & 0xffff0000u));
      }
      qe = min(int(top >> 23), 240);
      const float f = __uint_as_float(uint32_t(254 - qe) << 23);
      if (two || x == 0) {
#pragma unroll
        for (int c = 0; c < C::KSTEPS; ++c) {  // sixteen channels
          uint32_t h[8] = {};
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            if (16 * c + 8 * k >= DH) continue;
            const uint4 v = in ? *reinterpret_cast<const uint4*>(q + 16 * c + 8 * k)
                               : make_uint4(0, 0, 0, 0);
            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const float2 y = unpack_bf16x2(w[j]);
              asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(h[4 * k + j]) : "f"(y.y * f), "f"(y.x * f));
            }
          }
          if constexpr (C::Q_TMEM) {
            tmem_st8(tmem + uint32_t(C::TM_Q + (two ? x : 0) * C::Q_COLS + 8 * c) +
                         (uint32_t((warp & 3) * 32) << 16), h);
          } else {
            const uint32_t row = sq + (two ? x : 0) * C::Q_BYTES + (c >> 2) * (BQ * 128) + tr * 128;
            sts128(row + (((2 * c) ^ tr) & 7) * 16, h[0], h[1], h[2], h[3]);
            sts128(row + (((2 * c + 1) ^ tr) & 7) * 16, h[4], h[5], h[6], h[7]);
          }
        }
        if (C::Q_TMEM) {
          tmem_wait_st();
          tc_fence_before();
        } else {
          fence_proxy_async_smem();
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(q_full);
    }
    // factor of the row's scores, in base 2
    const float own = 1.4426950408889634f * rsqrtf(float(DH)) * scale_value(qe);
    const uint32_t lanes = uint32_t((warp & 3) * 32) << 16;
    const uint32_t ts = tmem + uint32_t(x * BKV) + lanes;
    const uint32_t to = tmem + uint32_t(TM_O + x * C::ODIM) + lanes;
    const int mine = two ? nb : (nb + 1 - x) / 2;  // this stream's key blocks
    const auto block_of = [&](int i) { return b0 + (two ? i : 2 * i + x); };
    const auto fact = [&](int p) {
      const int page = checked(entry(p));
      if (page < 0) return make_float2(0.f, ABSENT);
      const long long at = (long long)page * pool.heads + head;
      const int k = pool.scale[0][at], v = pool.scale[1][at];
      return make_float2(scale_value(max(k, v) == 255 ? 255 : k), float(v));
    };
    for (int p = int(threadIdx.x); p < min(C::FACTS, PAGES * nb); p += 256)
      facts[p] = fact(PAGES * b0 + p);
    soft_sync();
    // (a row that sees nothing here needs no maximum)
    const bool blind = seen <= block_of(0) * BKV;
    float m = blind ? 0.f : -INFINITY, l = 0.f;
    // Exponent of the value scale that O is in units of.  A row keeps that of the
    // last block that it sees (`own_ref`): later ones may have far larger values, or
    // none.  (Rows that see a block have seen all before it, so they share `ref`.)
    float ref = NO_REF, own_ref = NO_REF;
    const int least = __reduce_min_sync(0xffffffffu, seen);  // what every row of the warp sees
    bool searching = __any_sync(0xffffffffu, m == -INFINITY);

    const int count = PAGES * mine;
    const int skip = (two ? 1 : 2) * PAGES - 1;  // from a key block's second cache block to the next
    int page = PAGES * (block_of(0) - b0);       // of the CTA's
    const auto facts_of = [&](int p) { return p < C::FACTS ? facts[p] : fact(PAGES * b0 + p); };
    const auto s_bar = [&](int g) { return s_full + 16 * (g & 1) + 8 * x; };
    const auto hand_over = [&](int g) {  // block g's weights
      tmem_wait_st();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(p_full + 16 * (g & 1) + 8 * x);
    };
    uint32_t w[KV8_BLOCK];  // a cache block's scores, then its weights
    float2 now = count > 0 ? facts_of(page) : make_float2(0.f, ABSENT);
#pragma unroll 1
    for (int g = 0; g < count; ++g) {
      const uint32_t s_at = ts + uint32_t((g & 1) * KV8_BLOCK);
      float f = own * now.x;
      f = f > 3e38f ? 3e38f : f;  // (an infinite factor would make NaN of a score of 0)
      const int key0 = (PAGES * b0 + page) * KV8_BLOCK;
      const int limit = now.y < NO_REF ? 0 : seen - key0;  // columns that the row sees
      const float raise_to = now.y > ref + RAISE_VALUE ? now.y : ref;
      // no column hidden, no value scale far below the reference
      const bool whole = least - key0 >= KV8_BLOCK && now.y - raise_to >= -60.f;
      const int next = page + (g & 1 ? skip : 1);
      bool raise_max = searching && m == -INFINITY;
      // (after a failed wait the rows go on, without waiting)
      if (ok) ok = mbar_sleep(s_bar(g), (g >> 1) & 1, abort_flag);
      __syncwarp();
      tc_fence_after();
      float sum;
      for (bool again = false;; again = true) {
        if (again || searching || raise_to != ref) {
          // ---- a new reference: the row's largest score (where asked for)
          tmem_ld64(s_at, w);
          float top = m;
#pragma unroll
          for (int c = 0; c < KV8_BLOCK; ++c)
            top = fmaxf(top, c < limit ? __uint_as_float(w[c]) * f : -INFINITY);
          const float to_max = raise_max ? top : m;
          float corr = to_max == -INFINITY ? 1.f : ex2_ftz(m - to_max);
          l *= corr;
          if (seen > key0) {
            if (raise_to != ref && ref > NO_REF) corr *= ex2_ftz(ref - raise_to);
            own_ref = raise_to;
          }
          m = to_max;
          ref = raise_to;
          if (g > 0) {
            // once the P V before has ended (phase g - 1; the one before that
            // had when these scores were there)
            if (ok) ok = mbar_wait(o_done + 8 * x, (g - 1) & 1, abort_flag);
            __syncwarp();
            tc_fence_after();
#pragma unroll 1
            for (int c0 = 0; c0 < C::ODIM; c0 += 16) {
              uint32_t o[16];
              tmem_ld16_nowait(to + c0, o);
              tmem_wait_ld();
#pragma unroll
              for (int c = 0; c < 16; ++c) o[c] = __float_as_uint(__uint_as_float(o[c]) * corr);
              tmem_st16(to + c0, o);
            }
            tmem_wait_st();
          }
        }
        // ---- weights 2^(score - m + value scale's exponent over ref's + 100);
        // the sum is taken from value scales of 2^-60 of the reference's up, so
        // that it keeps small weights
        const float mm = m == -INFINITY ? 0.f : m;
        const float d = now.y - ref, dv = fmaxf(d, -60.f) + WEIGHT_UP, shift = dv - mm;
        uint64_t total[2] = {0, 0};
        tmem_ld64(s_at, w);
        if (whole)
          weights<true>(w, w, f, shift, KV8_BLOCK, 1.f, total);
        else
          weights<false>(w, w, f, shift, limit, ex2_ftz(fmaxf(d, -126.f) + WEIGHT_UP - dv), total);
        const float2 t = split64(add2(total[0], total[1]));
        // (a block that the row sees nothing of adds nothing, whatever its scale)
        sum = limit > 0 ? (t.x + t.y) * ex2_ftz(-dv) : 0.f;
        raise_max = sum > RAISE_SUM;
        if (again || !__any_sync(0xffffffffu, raise_max)) break;
      }
      l += sum;
      tmem_st32(s_at, w);
      hand_over(g);
      page = next;
      if (g + 1 < count) now = facts_of(page);
      if (searching) searching = __any_sync(0xffffffffu, m == -INFINITY);
    }
    ok = __all_sync(0xffffffffu, ok);

    // ---- result: O of a row in f32, or its part to be joined
    if (ok && mine > 0) ok = mbar_sleep_warp(o_full + 8 * x, 0, abort_flag);
    ok = __all_sync(0xffffffffu, ok);
    tc_fence_after();
    // (before the value scale the products are divided by their sum, or by its
    // power of two where parts will be joined)
    const bool alone = two && parts == 1;
    const int e = part_exponent(l);
    const float down = alone ? (l == 0.f ? 0.f : 1.f / l) : __uint_as_float(uint32_t(127 - e) << 23);
    const float back = own_ref > NO_REF ? scale_value(int(own_ref)) : 0.f;
    const auto row_out = [&](int r) {
      const int qi = (row0 + r) / group, g = row0 + r - qi * group;
      return a.o + (long long)(q0 + qi) * a.ldo + (head * group + g) * DH;
    };
    // eight channels from 8 c of the row's result, in their order
    const auto eight = [&](int c, float* v) {
      uint32_t o[8];
      tmem_ld8_nowait(to + 8 * c, o);
      tmem_wait_ld();
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = __uint_as_float(o[o_column(j)]) * (VALUE_DOWN * down) * back;
    };
    const auto put = [&](bf16* p, const float* v, float inv) {
      *reinterpret_cast<uint4*>(p) =
          make_uint4(pack_bf16x2(v[0] * inv, v[1] * inv), pack_bf16x2(v[2] * inv, v[3] * inv),
                     pack_bf16x2(v[4] * inv, v[5] * inv), pack_bf16x2(v[6] * inv, v[7] * inv));
    };
    if (alone) {
      bf16* p = row_out(in ? ur : 0);
#pragma unroll
      for (int c = 0; c < DH / 8; ++c) {
        float v[8];
        if (mine > 0) eight(c, v);
        else
          for (int j = 0; j < 8; ++j) v[j] = 0.f;
        if (in && ok) put(p + 8 * c, v, 1.f);
      }
    } else {
      // The row's parts (of both streams where they share a tile, of every CTA
      // of the cluster) meet in the shared memory of the CTA that owns the row,
      // over its operands once every MMA has read them: channels, maximum, sum.
      const int streams = two ? 1 : 2, n = streams * parts;
      const int each = ((two ? 2 : 1) * BQ + parts - 1) / parts;  // rows of a CTA
      const auto slot = [&](int k, int r) { return sq + 4 * uint32_t((k * each + r) * C::PSTRIDE); };
      soft_sync();
      if (parts > 1) cluster_sync();
      const uint32_t mine_at = slot(part * streams + (two ? 0 : x), ur % each);
      const uint32_t put_at = parts > 1 ? mapa_shared(mine_at, uint32_t(ur / each)) : mine_at;
#pragma unroll 1
      for (int c = 0; c < DH / 8; ++c) {
        float v[8] = {};
        if (mine > 0) eight(c, v);  // (every row of a warp takes part in the load)
        if (in) {
          store_four(put_at + 32 * c, v);
          store_four(put_at + 32 * c + 16, v + 4);
        }
      }
      if (in) store_two(put_at + 4 * DH, blind ? -INFINITY : m + float(e), l * down);
      if (parts > 1) cluster_sync();
      else soft_sync();
      const int first = part * each, live = min(each, rows - first);
      for (int e = int(threadIdx.x); e < live * (DH / 8); e += 256) {
        const int r = e / (DH / 8), c = e - r * (DH / 8);
        const float* at = reinterpret_cast<const float*>(smem) + r * C::PSTRIDE;
        const int far = each * C::PSTRIDE;  // from a row's part to its next
        float top = -INFINITY, total = 0.f, v[8] = {};
        for (int k = 0; k < n; ++k) top = fmaxf(top, at[k * far + DH]);
        const float rf = top == -INFINITY ? 0.f : top;
        for (int k = 0; k < n; ++k) {
          const float y = ex2_ftz(at[k * far + DH] - rf);
          total += y * at[k * far + DH + 1];
          const float4 p0 = *reinterpret_cast<const float4*>(at + k * far + 8 * c);
          const float4 p1 = *reinterpret_cast<const float4*>(at + k * far + 8 * c + 4);
          v[0] += y * p0.x; v[1] += y * p0.y; v[2] += y * p0.z; v[3] += y * p0.w;
          v[4] += y * p1.x; v[5] += y * p1.y; v[6] += y * p1.z; v[7] += y * p1.w;
        }
        if (ok) put(row_out(first + r) + 8 * c, v, total == 0.f ? 0.f : 1.f / total);
      }
    }
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(OTHER_REGS));
    if (warp == MMA_WARP) {
      // ----------------------------------------------------------------- MMA
      // Each stream's S holds two cache blocks; the scores of the second next one
      // follow the products that used their place, so that a stream's softmax
      // finds its next scores ready.
      if (nb > 0 && elect_one()) {
        const int rounds = two ? nb : (nb + 1) / 2;  // key blocks of stream 0
        // key block of a stream's i-th, and whether a stream is the first or the
        // last to use it
        const auto block = [&](int i, int x) { return two ? i : 2 * i + x; };
        const auto scores = [&](int i, int h, int x) {
          const int b = block(i, x), st = b % C::KST;
          if (b >= nb) return true;
          if (h == 0 && (!two || x == 0) &&
              !mbar_wait(k_full + 8 * st, (b / C::KST) & 1, abort_flag)) return false;
          tc_fence_after();
          const uint32_t k = sk + st * C::K_BYTES + h * (KV8_BLOCK * 128);
          const uint32_t d = tmem + uint32_t(x * BKV + h * KV8_BLOCK);
          const int tile = two ? x : 0;
          if constexpr (C::Q_TMEM) {
            const uint32_t q = tmem + uint32_t(C::TM_Q + tile * C::Q_COLS);
#pragma unroll
            for (int kk = 0; kk < 4; ++kk)
              umma_bf16_ta(d, q + 8 * kk, sw128_desc(k) + 2 * kk, C::IDESC_S, kk ? 1u : 0u);
            if (C::TAIL)
              umma_bf16_ta(d, q + 32,
                           sw32_kmajor_desc(sk + st * C::K_BYTES + BKV * 128 + h * (KV8_BLOCK * 32)),
                           C::IDESC_S, 1u);
          } else {
            const uint32_t q = sq + tile * C::Q_BYTES;
#pragma unroll
            for (int f = 0; f < C::FULL; ++f)
#pragma unroll
              for (int kk = 0; kk < 4; ++kk)
                umma_bf16(d, sw128_desc(q + f * BQ * 128) + 2 * kk,
                          sw128_desc(k + f * BKV * 128) + 2 * kk, C::IDESC_S, (f | kk) ? 1u : 0u);
          }
          umma_commit(s_full + 16 * h + 8 * x);
          if (h == PAGES - 1 && (!two || x == 1)) umma_commit(k_empty + 8 * st);
          return true;
        };
        ok = mbar_wait(q_full, 0, abort_flag);
        for (int h = 0; h < PAGES; ++h)
          for (int x = 0; x < 2; ++x) ok = ok && scores(0, h, x);
        for (int i = 0; ok && i < rounds; ++i) {
#pragma unroll
          for (int h = 0; h < PAGES; ++h) {
            for (int x = 0; x < 2; ++x) {
              const int b = block(i, x), st = b % C::VST;
              if (b >= nb) continue;
              if ((h == 0 && (!two || x == 0) &&
                   !mbar_wait(v_full + 8 * st, (b / C::VST) & 1, abort_flag)) ||
                  !mbar_wait(p_full + 16 * h + 8 * x, i & 1, abort_flag)) { ok = false; break; }
              tc_fence_after();
              const uint32_t d = tmem + uint32_t(TM_O + x * C::ODIM);
              const uint32_t p = tmem + uint32_t(x * BKV + h * KV8_BLOCK);
              const uint64_t v = sw128_mnmajor_desc_lbo(
                  sv + st * C::V_BYTES + h * (KV8_BLOCK * 128), BKV * 128);
#pragma unroll
              for (int kk = 0; kk < KV8_BLOCK / 16; ++kk)
                umma_bf16_ta(d, p + 8 * kk, v + 128 * kk, C::IDESC_PV, (i | h | kk) ? 1u : 0u);
              umma_commit(o_done + 8 * x);
              if (h == PAGES - 1) {
                if (!two || x == 1) umma_commit(v_empty + 8 * st);
                if (block(i + 1, x) >= nb) umma_commit(o_full + 8 * x);
              }
              if (!scores(i + 1, h, x)) { ok = false; break; }
            }
            if (!ok) break;
          }
        }
      }
    } else if (warp == LOAD_WARP) {
      // ------------------------------------------------------------- loading
      // (the copies are whole cache blocks; one that is missing is left out:
      // what it leaves in the ring is hidden by the softmax)
      if (elect_one()) {
        int page[PAGES], ahead[2][PAGES];
#pragma unroll
        for (int i = 0; i < PAGES; ++i) {
          ahead[0][i] = nb > 0 ? entry(PAGES * b0 + i) : -1;
          ahead[1][i] = nb > 1 ? entry(PAGES * (b0 + 1) + i) : -1;
        }
        for (int j = 0; ok && j < 2 * nb; ++j) {
          const int st = j % C::RAWS, side = j & 1, b = j >> 1;
          if (side == 0)
#pragma unroll
            for (int i = 0; i < PAGES; ++i) {
              page[i] = checked(ahead[0][i]);
              if (page[i] < 0 && PAGES * (b0 + b) + i < pages) atomicOr(a.err, DEVERR_INDEX);
              ahead[0][i] = ahead[1][i];
              ahead[1][i] = b + 2 < nb ? entry(PAGES * (b0 + b + 2) + i) : -1;
            }
          if (!mbar_wait(raw_empty + 8 * st, ((j / C::RAWS) & 1) ^ 1, abort_flag)) { ok = false; break; }
          constexpr uint32_t BYTES = KV8_BLOCK * DH;
          mbar_expect_tx(raw_full + 8 * st,
                         BYTES * ((page[0] >= 0 ? 1u : 0u) + (page[1] >= 0 ? 1u : 0u)));
#pragma unroll
          for (int i = 0; i < PAGES; ++i)
            if (page[i] >= 0)
              bulk_load(raw + st * C::RAW_BYTES + i * BYTES,
                        pool.code[side] + ((long long)page[i] * pool.heads + head) * BYTES, BYTES,
                        raw_full + 8 * st);
        }
      }
    } else if (warp >= CONV_WARP) {
      // ---------------------------------------------------------- conversion
      // A thread takes the same pieces (8 channels each) of every PASS-th row.
      const bool values = warp >= CONV_WARP + 4;
      const int tid = int(threadIdx.x) - (values ? CONV_WARP + 4 : CONV_WARP) * 32;
      const int r0 = tid / C::ROW_THREADS, c0 = (tid - r0 * C::ROW_THREADS) * C::PIECES;
      uint32_t to[C::PIECES];  // a piece's place in row r0 of a tile of keys or values
#pragma unroll
      for (int k = 0; k < C::PIECES; ++k) {
        const int c = c0 + k;
        to[k] = !values && C::TAIL && c == 8
                    ? BKV * 128 + r0 * 32 + (((r0 >> 2) & 1) << 4)
                    : (c >> 3) * (BKV * 128) + r0 * 128 + (((c ^ r0) & 7) << 4);
      }
      const bool tail = !values && C::TAIL && c0 + C::PIECES == 9;  // (its last piece)
      for (int b = 0; b < nb; ++b) {
        const int j = 2 * b + (values ? 1 : 0), st = j % C::RAWS, ks = b % C::KST, vs = b % C::VST;
        if (ok)
          ok = (values ? mbar_sleep(v_empty + 8 * vs, ((b / C::VST) & 1) ^ 1, abort_flag)
                       : mbar_sleep(k_empty + 8 * ks, ((b / C::KST) & 1) ^ 1, abort_flag)) &&
               mbar_sleep(raw_full + 8 * st, (j / C::RAWS) & 1, abort_flag);
        if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
        const uint32_t from = raw + st * C::RAW_BYTES + r0 * DH + c0 * 8;
        const uint32_t tile = values ? sv + vs * C::V_BYTES : sk + ks * C::K_BYTES;
        constexpr int PASSES = (BKV + C::PASS - 1) / C::PASS;
#pragma unroll
        for (int p = 0; p < PASSES; ++p) {
          if (r0 + p * C::PASS >= BKV) break;
          uint2 q[C::PIECES];
#pragma unroll
          for (int k = 0; k < C::PIECES; ++k) q[k] = lds64(from + p * C::PASS * DH + 8 * k);
          if (values) {
#pragma unroll
            for (int k = 0; k < C::PIECES; ++k)
              sts128(tile + to[k] + p * C::PASS * 128, codes_02(q[k].x), codes_13(q[k].x),
                     codes_02(q[k].y), codes_13(q[k].y));
          } else {
#pragma unroll
            for (int k = 0; k < C::PIECES; ++k) {
              uint32_t h[4];
              e4m3x4_f16(q[k].x, h[0], h[1]);
              e4m3x4_f16(q[k].y, h[2], h[3]);
              sts128(tile + to[k] + p * C::PASS * (k == C::PIECES - 1 && tail ? 32 : 128), h[0],
                     h[1], h[2], h[3]);
            }
          }
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(raw_empty + 8 * st);
          mbar_arrive(values ? v_full + 8 * vs : k_full + 8 * ks);
        }
      }
    }
  }
  if (parts > 1 && warp >= CONV_WARP) {  // (as the softmax warps did)
    __syncwarp();
    cluster_sync();
    cluster_sync();
  }
  if (!ok) {
    *abort_flag = 1;
    atomicOr(a.err, DEVERR_TIMEOUT);
  }
  tc_fence_before();
  __syncthreads();
  if (warp == MMA_WARP) {
    __syncwarp();
    tc_fence_after();
    tmem_dealloc(tmem, TMEM_COLS);
  }
}

constexpr int SMS = 152;

// Rows of a unit and CTAs that share its keys, of least estimated time (us) for
// requests of the mean number of rows and the longest length that the table holds
// (8 requests of 500 tokens, 256 rows: 17 us with a table of that width, 33 with one
// of 16384 tokens).  Where there are several requests, the mean of that and of the
// time for lengths spread evenly, the longest units first (8 requests of 256 rows,
// 16 heads of 72: of 500 to 12000 tokens one part 140 us, two 89; of 12000 each 141
// and 157).  Rates measured at 4096 keys, head_dim 72, 16 heads: a key block takes a
// unit of 256 rows 1.45 us and one of 128 1.1, a unit 4.5 beyond that, and joining
// parts 5 (2.5) and 0.65 for each (256 rows: one part 52.8 us, six 22.2; 831: two
// 35.3, one 54.0; 4096: one 106, two 132).  Clusters above six CTAs do not all find
// a place at once.
struct Shape {
  int unit_rows, parts;
};
Shape choose(const Kv8AttnArgs& a, int kv_heads, int group) {
  const long long most = (long long)a.n * a.max_q, rows = most < a.q_rows ? most : a.q_rows;
  const double mean = double(rows) * group / a.n;
  const double blocks = double(a.ld_table) * KV8_BLOCK / BKV;
  Shape best{256, 1};
  double least = 1e30;
  for (int ur = 256; ur >= 128; ur -= 128)
    for (int parts = 1; parts <= 6; ++parts) {
      if (parts > 1 && blocks < 2 * parts) break;
      const double units = ceil(mean / ur) * kv_heads * a.n * parts;
      const double waves = units <= SMS ? 1.0 : units / SMS + 0.5;
      const bool wide = ur == 256 && mean > 128;
      const double block = wide ? 1.45 : 1.1;
      const double start = 4.5 + (parts > 1 ? (wide ? 5.0 : 2.5) + 0.65 * parts : 0.0);
      const double one = ceil(blocks / parts) * block + start;
      double cost = waves * one;
      if (a.n > 1) {
        const double some = units * (0.55 * blocks / parts * block + start) / SMS;
        cost = 0.5 * (cost + (some > one ? some : one));
      }
      if (cost < least * (a.n > 1 ? 0.95 : 0.98)) {
        least = cost;
        best = Shape{ur, parts};
      }
    }
  return best;
}

template <int DH>
cudaError_t many(const Kv8Pool& pool, const Kv8AttnArgs& a, cudaStream_t st) {
  using C = MCfg<DH>;
  RC_TRY(cudaFuncSetAttribute(many_rows_kernel<DH>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                              int(C::SMEM)));
  const int group = a.heads / pool.heads;
  const Shape sh = choose(a, pool.heads, group);
  const int unit_rows = sh.unit_rows, parts = sh.parts;
  // Units at most: whole ones and a last one for each request.  Where CTAs wait
  // for others' places the longest go first, of up to 64 requests; of more, the
  // kernel counts out the units that there are where places for every chunk of
  // every request would be more than twice as many (a place without one costs a
  // CTA's launch, the counting every CTA 1.2 us).  16 requests of 500 to 9000
  // tokens and 100 to 400 rows: 146 us, in place 180; 32 of 500 to 8000, 40 to 200
  // rows, 4 heads a key head of 128: 320 and 390; 8 of 4096, 201 to 831 rows: 123
  // and 125; 4 of 4096, 512 rows each, 4 heads of 128: 142 and 136.
  const long long most = (long long)a.n * a.max_q, rows = most < a.q_rows ? most : a.q_rows;
  const long long all = ((long long)a.max_q * group + unit_rows - 1) / unit_rows * a.n;
  long long units = rows * group / unit_rows + a.n;
  const int order = a.n > 1 && a.n <= MAX_RANKED && all * pool.heads * parts > SMS ? BY_WORK
                    : all > 2 * units ? COUNTED : IN_PLACE;
  if (order == IN_PLACE || units > all) units = all;
  const long long ctas = units * pool.heads * parts;
  if (ctas > 0x7fffffff) return cudaErrorInvalidConfiguration;
  const dim3 grid{unsigned(ctas), 1u, 1u};
  count_launches(1);
  return launch_k_cluster(many_rows_kernel<DH>, grid, dim3(THREADS), C::SMEM, parts, st, pool, a,
                          parts, unit_rows, order);
}

}  // namespace

cudaError_t launch_kv8_many(const Kv8Pool& pool, const Kv8AttnArgs& a, cudaStream_t st) {
  switch (pool.dh) {
    case 64: return many<64>(pool, a, st);
    case 72: return many<72>(pool, a, st);
    default: return many<128>(pool, a, st);
  }
}

}  // namespace rc
