// Products of each expert's rows with its quantised matrix (rc_experts_linear):
// y[p] = act(x[source[p]] W_e^T + b_e), on the block-scaled e4m3 MMA of the
// tensor core, with the work shared out on the device (only it knows how many rows
// each expert has).
//
// Persistent CTAs of 16 warps, as in rc_fp8_linear: warp 0 brings the rows of x
// (gathered by TMA, four rows an instruction and lane), warp 2 W, warp 1 issues
// the MMAs, warps 4..7 put the scale bytes into tensor memory, warps 8..15 drain
// the accumulator.  Each CTA first lists the experts that have rows, with the
// tiles of BM rows before each; a tile's number names its rows by a search there,
// and its columns.  Rows of an accumulator do not mix, so what a tile holds beyond
// its expert's rows (stale shared memory, the next expert's rows) is only never
// written.
#include <float.h>

#include "../../include/regioncache.h"
#include "block.h"
#include "common.cuh"
#include "fp8.cuh"
#include "tc_chunks.cuh"

namespace rc {

namespace {

using namespace rc::tc;

constexpr int BM = 128, BK = 128;
constexpr int THREADS = 512;
constexpr int SCALE_WARP = 4, EPI_WARP = 8, EPI_WARPS = 8;
constexpr int STAGE_A = BM * BK;
constexpr int RING_BYTES = 172 * 1024, MAX_STAGES = 7;
// tensor memory: accumulators at 0 and ACC_BN (one, where a tile is wider), then a
// ring of scale words: a batch holds, for each WORD_KB blocks, 4 columns for x and
// 8 for W
constexpr int ACC_BN = 192, MAX_BN = 256, SCALE_COL = 2 * ACC_BN, TMEM_COLS = 512;
constexpr int WORD_KB = 4, SCALE_BATCH = 16, SCALE_GROUPS = SCALE_BATCH / WORD_KB;
constexpr int SCALE_STEP = 12, SCALE_SLOT = SCALE_GROUPS * SCALE_STEP, SCALES = 2;
static_assert(SCALE_COL + SCALES * SCALE_SLOT <= TMEM_COLS, "tensor memory");
// the batch's words in shared memory: 128 rows of x, four shared rows of W
constexpr int SCALE_ROWS = 128 + 4, SCALE_BYTES = SCALE_GROUPS * SCALE_ROWS * 4;
// the experts that have rows: tiles before, first row, end, number
constexpr int MAX_E = RC_EXPERTS_MAX;
struct Tables {
  int first[MAX_E], row[MAX_E], end[MAX_E];
  uint16_t expert[MAX_E];
  unsigned long long parts[THREADS / 32];
};
constexpr int TOPS_BYTES = 2 * EPI_WARPS * 32 * 4;
constexpr size_t SMEM_BYTES = size_t(RING_BYTES) + EPI_WARPS * CHUNK_STAGING + SCALE_BYTES +
                              TOPS_BYTES + sizeof(Tables) + 1024 + 256;
static_assert(SMEM_BYTES <= 227 * 1024, "shared memory");
static_assert(MAX_BN * 129 * 4 <= RING_BYTES, "a split tile's part");

struct Plan {
  int bn, stages, nt, kb, parts, accs, most;  // most: tiles of TM rows there can be
};
template <bool PAIR>
__host__ __device__ constexpr int stage_bytes(int bn) {
  return STAGE_A + (PAIR ? bn / 2 : bn) * BK;
}

enum Kind { BF16, F32, CODES };
template <Kind>
struct TypeOf { typedef bf16 T; };
template <>
struct TypeOf<F32> { typedef float T; };
template <>
struct TypeOf<CODES> { typedef uint8_t T; };

// v / (1 + 2^e).  Quotient and power on the special-function unit are good to a
// few steps of f32.
__device__ __forceinline__ float over_one_plus(float v, float e) {
  return __fdividef(v, 1.f + ex2_ftz(e));
}
// GELU by its sigmoid: (1 + tanh a) / 2 = 1 / (1 + exp(-2 a)).
__device__ __forceinline__ float act_gelu(float v) {
  const float k = -2.f * 0.7978845608028654f * 1.4426950408889634f;  // sqrt(2 / pi), log2 e
  return over_one_plus(v, k * v * fmaf(0.044715f * v, v, 1.f));
}
__device__ __forceinline__ float act_silu(float v) {
  return over_one_plus(v, -1.4426950408889634f * v);
}
__device__ __forceinline__ float act_of(int act, float v) {
  return act == RC_ACT_GELU ? act_gelu(v) : act == RC_ACT_SILU ? act_silu(v) : v;
}

// Barriers of the four scale warps, and of the two epilogue warps of a row.
__device__ __forceinline__ void scale_sync() { asm volatile("bar.sync 1, 128;" ::: "memory"); }
__device__ __forceinline__ void rows_sync(int sp) {
  asm volatile("bar.sync %0, 64;" ::"r"(2 + sp) : "memory");
}

// How CTAs work together, as in rc_fp8_linear.  PAIRS: clusters of two share each
// MMA (M = 256).  SPLIT: a cluster shares a tile's blocks of columns, each CTA
// leaves its part in shared memory, and the parts are added there in order.
enum Mode { ALONE, PAIRS, SPLIT };

template <Kind OUT, Mode MODE>
__global__ void __launch_bounds__(THREADS, 1)
experts_linear_kernel(const __grid_constant__ CUtensorMap tmX,
                      const __grid_constant__ CUtensorMap tmG,
                      const __grid_constant__ CUtensorMap tmW,
                      const __grid_constant__ CUtensorMap tmY,
                      const __grid_constant__ ExpertsArgs a, const __grid_constant__ Plan pl) {
  using T = typename TypeOf<OUT>::T;
  constexpr bool PAIR = MODE == PAIRS;
  constexpr int CTAS = PAIR ? 2 : 1, TM = BM * CTAS;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                             ~uintptr_t(1023));
  uint8_t* stg = smem + RING_BYTES;
  uint32_t* words = reinterpret_cast<uint32_t*>(stg + EPI_WARPS * CHUNK_STAGING);
  uint32_t* tops = words + SCALE_BYTES / 4;
  Tables& tab = *reinterpret_cast<Tables*>(tops + TOPS_BYTES / 4);
  uint64_t* bars = reinterpret_cast<uint64_t*>(&tab + 1);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 2 * MAX_STAGES + 2 * SCALES + 4);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  const uint32_t full0 = saddr(bars), empty0 = full0 + 8 * MAX_STAGES;
  const uint32_t sfull0 = empty0 + 8 * MAX_STAGES, sempty0 = sfull0 + 8 * SCALES;
  const uint32_t tfull0 = sempty0 + 8 * SCALES, tempty0 = tfull0 + 16;

  const int warp = warp_index(), lane = threadIdx.x & 31;
  const uint32_t rank = PAIR ? cluster_ctarank() : 0;  // in a pair
  if (threadIdx.x == 0) {
    for (int s = 0; s < MAX_STAGES; ++s) {
      mbar_init(full0 + 8 * s, PAIR ? 1 : 2);  // (x's and W's loads)
      mbar_init(empty0 + 8 * s, 1);
    }
    for (int s = 0; s < SCALES; ++s) {
      mbar_init(sfull0 + 8 * s, 4 * CTAS);
      mbar_init(sempty0 + 8 * s, 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(tfull0 + 8 * i, 1);
      mbar_init(tempty0 + 8 * i, EPI_WARPS * CTAS);
    }
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    if (PAIR) tmem_alloc_pair(saddr(tmem_slot), TMEM_COLS);
    else tmem_alloc(saddr(tmem_slot), TMEM_COLS);
  }
  pdl_wait();
  pdl_trigger();
  // the experts that have rows (thread t looks at two; counts of experts and of
  // tiles are summed in one word)
  int entries, m_tiles;
  {
    int lo[2], hi[2];
    unsigned long long mine = 0;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int e = 2 * int(threadIdx.x) + j;
      lo[j] = hi[j] = 0;
      if (e < a.experts) {
        lo[j] = a.offsets[e], hi[j] = a.offsets[e + 1];
        if (lo[j] < 0 || lo[j] > hi[j] || hi[j] > a.pairs) {
          if (blockIdx.x == 0) atomicOr(a.err, DEVERR_COUNT);
          lo[j] = hi[j] = 0;
        }
      }
      if (hi[j] > lo[j]) mine += (1ull << 32) + unsigned((hi[j] - lo[j] - 1) / TM + 1);
    }
    unsigned long long sum = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const unsigned long long v = __shfl_up_sync(~0u, sum, o);
      if (lane >= o) sum += v;
    }
    if (lane == 31) tab.parts[warp] = sum;
    __syncthreads();
    unsigned long long before = sum - mine, all = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 32; ++w) {
      if (w < warp) before += tab.parts[w];
      all += tab.parts[w];
    }
#pragma unroll
    for (int j = 0; j < 2; ++j)
      if (hi[j] > lo[j]) {
        const int i = int(before >> 32);
        tab.first[i] = int(before & 0xffffffffu);
        tab.row[i] = lo[j], tab.end[i] = hi[j];
        tab.expert[i] = uint16_t(2 * threadIdx.x + j);
        before += (1ull << 32) + unsigned((hi[j] - lo[j] - 1) / TM + 1);
      }
    // (offsets that descend can name rows twice)
    entries = int(all >> 32), m_tiles = int(min(all & 0xffffffffull, (unsigned long long)pl.most));
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  if (PAIR) cluster_sync();  // (the peer's barriers are ready)

  const int BN = pl.bn, STAGES = pl.stages, ACCS = pl.accs;
  const int STAGE = stage_bytes<PAIR>(BN);
  const bool gated = a.act == RC_ACT_GATED_SILU;
  const int half_bn = BN / 2, cols_out = gated ? half_bn : BN;  // outputs of a tile
  const int e_rows = a.w.rows / a.experts, N = gated ? 2 * a.n : a.n;
  const int tiles = m_tiles * pl.nt;
  // this CTA's (or pair's) tiles pos, pos + G .. and, of each, its blocks
  // k0 .. k0 + KB - 1
  const int parts = MODE == SPLIT ? pl.parts : 1;
  const int part_of = MODE == SPLIT ? int(cluster_ctarank()) : 0;
  const int k0 = part_of * pl.kb / parts, KB = (part_of + 1) * pl.kb / parts - k0;
  const int G = int(gridDim.x) / (CTAS * parts), pos = int(blockIdx.x) / (CTAS * parts);
  bool ok = true;

  // tile t: its expert, first place, places left there and number among the columns
  struct Tile { int expert, place, left, n; };
  const auto tile_of = [&](int t) {
    const int q = t / pl.nt;
    int lo = 0, hi = entries;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (tab.first[mid] <= q) lo = mid;
      else hi = mid;
    }
    const int p = tab.row[lo] + (q - tab.first[lo]) * TM;
    return Tile{tab.expert[lo], p, tab.end[lo] - p, t - q * pl.nt};
  };
  // rows of a CTA of this tile (the second of a pair may have none)
  const auto rows_of = [&](const Tile& t, int r) { return max(0, min(BM, t.left - r * BM)); };
  // the row of x of a place (row 0 for one outside, which is reported)
  const auto row_of = [&](int place) {
    if (!a.source) return place;
    const int r = a.source[place];
    if (r >= 0 && r < a.x.rows) return r;
    atomicOr(a.err, DEVERR_INDEX);
    return 0;
  };
  // many neighbouring rows come as one box
  const auto in_box = [&](int rows) { return !a.source && rows > 32; };

  if (warp == 0) {
    // ---------------------------------------------------------------- TMA: x
    int stage = 0;
    uint32_t phase = 0;
    for (int t = pos; ok && t < tiles; t += G) {
      const Tile tl = tile_of(t);
      const int rows = rows_of(tl, int(rank)), place = tl.place + int(rank) * BM;
      const bool box = in_box(rows);
      int r[4] = {0, 0, 0, 0};
      if (!box) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (4 * lane + j < rows) r[j] = row_of(place + 4 * lane + j);
      }
      const auto bytes = [&](int n) { return in_box(n) ? STAGE_A : (n + 3) / 4 * 4 * BK; };
      int expect = bytes(rows_of(tl, 0));
      if (PAIR) expect += bytes(rows_of(tl, 1)) + BN * BK;
      for (int kb = 0; kb < KB; ++kb) {
        ok = __all_sync(~0u, mbar_wait(empty0 + 8 * stage, phase ^ 1, abort_flag));
        if (!ok) break;
        const uint32_t st = saddr(smem + stage * STAGE), fb = full0 + 8 * stage;
        const uint32_t bar = PAIR ? mapa_shared(fb, 0) : fb;
        // (a barrier may see bytes before it is told of them: its phase still
        // needs that arrival)
        if (rank == 0 && lane == 0) mbar_expect_tx(fb, uint32_t(expect));
        if (box) {
          if (elect_one()) {
            if (PAIR) tma_load_2d_pair(st, &tmX, bar, (k0 + kb) * BK, place);
            else tma_load_2d(st, &tmX, bar, (k0 + kb) * BK, place);
          }
        } else if (4 * lane < rows) {
          tma_gather4<PAIR>(st + lane * 4 * BK, &tmG, bar, (k0 + kb) * BK, r);
        }
        __syncwarp();
        if (++stage == STAGES) { stage = 0; phase ^= 1; }
      }
    }
  } else if (warp == 2) {
    // ---------------------------------------------------------------- TMA: W
    if (elect_one()) {
      int stage = 0;
      uint32_t phase = 0;
      for (int t = pos; ok && t < tiles; t += G) {
        const Tile tl = tile_of(t);
        const int n0 = tl.expert * e_rows + tl.n * cols_out;
        for (int kb = 0; kb < KB; ++kb) {
          if (!mbar_wait(empty0 + 8 * stage, phase ^ 1, abort_flag)) { ok = false; break; }
          const uint32_t st = saddr(smem + stage * STAGE) + STAGE_A, fb = full0 + 8 * stage;
          const int c = (k0 + kb) * BK;
          if (PAIR) {  // both CTAs' bytes land on rank 0's barrier (warp 0 told it of them)
            tma_load_2d_pair(st, &tmW, mapa_shared(fb, 0), c,
                             n0 + int(rank) * (gated ? a.n : half_bn));
          } else {
            mbar_expect_tx(fb, uint32_t(STAGE - STAGE_A));
            tma_load_2d(st, &tmW, fb, c, n0);
            if (gated) tma_load_2d(st + half_bn * BK, &tmW, fb, c, n0 + a.n);
          }
          if (++stage == STAGES) { stage = 0; phase ^= 1; }
        }
      }
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------ MMA issuer
    if (rank == 0 && elect_one()) {
      const uint32_t idesc = IDESC_E4M3 | (uint32_t(BN >> 3) << 17) | (uint32_t(CTAS) << 27);
      const uint64_t da = sw128_desc(saddr(smem)), db = sw128_desc(saddr(smem + STAGE_A));
      int stage = 0, acc = 0, sc = 0;
      uint32_t phase = 0, acc_phase = 0, sc_phase = 0;
      uint64_t so = 0;     // the stage's offset in the descriptors' address field
      bool ready = false;  // the current stage was seen full already
      for (int t = pos; ok && t < tiles; t += G) {
        if (!mbar_wait(tempty0 + 8 * acc, acc_phase ^ 1, abort_flag)) { ok = false; break; }
        const uint32_t d = tmem + uint32_t(acc * ACC_BN);
        uint32_t accumulate = 0;
        for (int kb = 0; ok && kb < KB;) {
          if (!mbar_wait(sfull0 + 8 * sc, sc_phase, abort_flag)) { ok = false; break; }
          uint32_t sa = tmem + uint32_t(SCALE_COL + sc * SCALE_SLOT);
          const int end = min(kb + SCALE_BATCH, KB);
          while (ok && kb < end) {
#pragma unroll
            for (int byte = 0; byte < WORD_KB; ++byte) {
              if (kb >= end) break;
              if (!ready && !mbar_wait(full0 + 8 * stage, phase, abort_flag)) { ok = false; break; }
              const uint64_t da_ = da + so, db_ = db + so;
              const uint32_t eb = empty0 + 8 * stage;
              ++kb;
              so += uint64_t(STAGE >> 4);
              if (++stage == STAGES) { stage = 0; phase ^= 1; so = 0; }
              // (the next stage's test runs beside this one's MMAs)
              ready = mbar_test(full0 + 8 * stage, phase);
              tc_fence_after();
              const uint32_t id = idesc | uint32_t(byte) << 4 | uint32_t(byte) << 29;
#pragma unroll
              for (int kk = 0; kk < BK / 32; ++kk) {
                if (PAIR)
                  umma_e4m3_scaled_pair(d, da_ + 2 * kk, db_ + 2 * kk, id, sa, sa + 4, accumulate);
                else
                  umma_e4m3_scaled(d, da_ + 2 * kk, db_ + 2 * kk, id, sa, sa + 4, accumulate);
                accumulate = 1;
              }
              if (PAIR) umma_commit_pair(eb);
              else umma_commit(eb);
            }
            sa += SCALE_STEP;
          }
          if (!ok) break;
          if (PAIR) umma_commit_pair(sempty0 + 8 * sc);
          else umma_commit(sempty0 + 8 * sc);
          if (++sc == SCALES) { sc = 0; sc_phase ^= 1; }
        }
        if (!ok) break;
        if (PAIR) umma_commit_pair(tfull0 + 8 * acc);
        else umma_commit(tfull0 + 8 * acc);
        if (++acc == ACCS) { acc = 0; acc_phase ^= 1; }
      }
    }
  } else if (warp >= SCALE_WARP && warp < EPI_WARP) {
    // -------------------------------------------------------- scale words
    // A thread loads a batch's bytes of one row of x, and 64 of them one byte of the
    // blocks of 128 rows of W that a tile can meet: two for each half of a gated
    // tile, three otherwise.  The bytes of the next batch are under way while this
    // one's words go by way of shared memory into tensor memory.
    const int tid = int(threadIdx.x) - SCALE_WARP * 32;
    const uint32_t part = uint32_t((warp & 3) * 32) << 16;
    const int slot = tid / SCALE_BATCH, u = tid % SCALE_BATCH, e_blocks = e_rows / 128;
    uint8_t bx[SCALE_BATCH], bw = 0;
    bool in = false;  // the thread's row is one of the expert's
    int xrow = 0, t_of = -1;
    Tile tl = {};
    const auto fetch = [&](int t, int kb) {
      if (t != t_of) {
        t_of = t;
        tl = tile_of(t);
        in = tid < rows_of(tl, int(rank));
        xrow = in ? row_of(tl.place + int(rank) * BM + tid) : 0;
      }
      const uint8_t* p = a.x.scales + xrow;
      if (in) {
#pragma unroll
        for (int i = 0; i < SCALE_BATCH; ++i)
          bx[i] = p[(long long)min(k0 + kb + i, pl.kb - 1) * a.x.lds];
      }
      if (slot < 4) {
        const int n0 = tl.n * cols_out + (gated && slot >= 2 ? a.n : 0);
        const int block = min(n0 / 128 + (gated ? slot & 1 : slot), e_blocks - 1);
        bw = a.w.scales[(long long)min(k0 + kb + u, pl.kb - 1) * a.w.lds +
                        tl.expert * e_blocks + block];
      }
    };
    int sc = 0, t = pos, kb = 0;
    uint32_t sc_phase = 0;
    if (t < tiles) fetch(t, kb);
    while (t < tiles) {
      scale_sync();  // (the batch before has been taken)
#pragma unroll
      for (int g = 0; g < SCALE_GROUPS; ++g)
        words[g * SCALE_ROWS + tid] =
            in ? uint32_t(bx[4 * g]) | uint32_t(bx[4 * g + 1]) << 8 |
                     uint32_t(bx[4 * g + 2]) << 16 | uint32_t(bx[4 * g + 3]) << 24
               : 0x7f7f7f7fu;
      if (slot < 4)
        reinterpret_cast<uint8_t*>(words + u / WORD_KB * SCALE_ROWS + 128 + slot)[u % WORD_KB] = bw;
      scale_sync();
      // which of the four words each row of the tile takes
      const int n0 = tl.n * cols_out;
      int of[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int r = 32 * i + lane;
        of[i] = !gated ? (n0 % 128 + r) / 128
                       : r < half_bn ? (n0 % 128 + r) / 128
                                     : 2 + ((n0 + a.n) % 128 + r - half_bn) / 128;
        of[i] = 128 + min(of[i], 3);
      }
      kb += SCALE_BATCH;
      if (kb >= KB) { kb = 0; t += G; }
      if (t < tiles) fetch(t, kb);
      if (ok) ok = mbar_sleep(sempty0 + 8 * sc, sc_phase ^ 1, abort_flag);
      // (after a failed wait the warp goes on to the barriers, without work)
      ok = __all_sync(0xffffffffu, ok);
      if (ok) {
        tc_fence_after();
        uint32_t v[SCALE_SLOT];
#pragma unroll
        for (int g = 0; g < SCALE_GROUPS; ++g) {
#pragma unroll
          for (int i = 0; i < 4; ++i) v[g * SCALE_STEP + i] = words[g * SCALE_ROWS + 32 * i + lane];
#pragma unroll
          for (int i = 0; i < 8; ++i) v[g * SCALE_STEP + 4 + i] = words[g * SCALE_ROWS + of[i]];
        }
        const uint32_t ta = tmem + uint32_t(SCALE_COL + sc * SCALE_SLOT) + part;
        tmem_st16(ta, v);
        tmem_st32(ta + 16, v + 16);
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          if (PAIR) mbar_arrive_cluster(mapa_shared(sfull0 + 8 * sc, 0));
          else mbar_arrive(sfull0 + 8 * sc);
        }
      }
      if (++sc == SCALES) { sc = 0; sc_phase ^= 1; }
    }
  } else if (warp >= EPI_WARP) {
    // ------------------------------------------------------------ epilogue
    // A warp takes 32 rows (a quarter of the tile's) and half of the chunks of 32
    // outputs: every second, or with codes every second pair, so that two warps
    // hold the 128 columns of a scale between them.
    const int sp = warp & 3, half = (warp - EPI_WARP) >> 2;
    const uint32_t tempty_r0 = PAIR ? mapa_shared(tempty0, 0) : tempty0;
    uint8_t* own = stg + (warp - EPI_WARP) * CHUNK_STAGING;
    constexpr int BUFS = OUT == F32 ? 1 : 2;  // staging of this many chunks
    constexpr int CHUNKS = MAX_BN / 64;
    const auto chunk_of = [&](int i) {
      return OUT == CODES ? (i >> 1) * 4 + half * 2 + (i & 1) : half + 2 * i;
    };
    T* const y = static_cast<T*>(OUT == CODES ? a.y8.codes : a.y);
    const int ldy = OUT == CODES ? a.y8.ld : a.ldy;
    int acc = 0, buf = 0, turn = 0;
    uint32_t acc_phase = 0;
    for (int t = pos; t < tiles; t += G) {
      const Tile tl = tile_of(t);
      const int left = rows_of(tl, int(rank)) - sp * 32;  // the warp's rows, from `r0`
      const int r0 = tl.place + int(rank) * BM + sp * 32;
      // (the bias before the accumulator is ready)
      float ba[CHUNKS], bb[CHUNKS];
#pragma unroll
      for (int i = 0; i < CHUNKS; ++i) {
        const int ch = chunk_of(i), c = tl.n * cols_out + ch * 32 + lane;
        const bool there = a.bias && ch * 32 < cols_out && c < a.n;
        ba[i] = there ? __ldg(a.bias + (long long)tl.expert * N + c) : 0.f;
        bb[i] = there && gated ? __ldg(a.bias + (long long)tl.expert * N + a.n + c) : 0.f;
      }
      if (ok) ok = mbar_sleep_warp(tfull0 + 8 * acc, acc_phase, abort_flag);
      // (after a failed wait the warp goes on to the barriers, without work)
      tc_fence_after();
      const uint32_t tb = tmem + uint32_t(acc * ACC_BN) + (uint32_t(sp * 32) << 16);
      // the outputs of chunk i (all 32 rows of the warp)
      const auto outputs = [&](int i, float* v) {
        const int ch = chunk_of(i);
        tmem_ld32(tb + uint32_t(ch * 32), v);
        if (a.bias)
#pragma unroll
          for (int j = 0; j < 32; ++j) v[j] += __shfl_sync(0xffffffffu, ba[i], j);
        if (gated) {
          float w[32];
          tmem_ld32(tb + uint32_t(half_bn + ch * 32), w);
#pragma unroll
          for (int j = 0; j < 32; ++j)
            v[j] = act_silu(v[j]) * (w[j] + __shfl_sync(0xffffffffu, bb[i], j));
        } else if (a.act != RC_ACT_NONE) {
#pragma unroll
          for (int j = 0; j < 32; ++j) v[j] = act_of(a.act, v[j]);
        }
      };
      if (MODE == SPLIT) {  // (every MMA is done: the operand ring is free)
        float* to = reinterpret_cast<float*>(smem) + sp * 32 + lane;
        for (int ch = half; ok && left > 0 && ch < BN / 32; ch += 2) {
          float v[32];
          tmem_ld32(tb + uint32_t(ch * 32), v);
          if (lane < left)
#pragma unroll
            for (int j = 0; j < 32; ++j) to[(ch * 32 + j) * 129] = v[j];
        }
      } else if constexpr (OUT == CODES) {
#pragma unroll
        for (int g = 0; g < CHUNKS / 2; ++g) {
          const int c0 = tl.n * cols_out + g * 128;
          if (left <= 0 || g * 128 >= cols_out || c0 >= a.n) break;  // (both warps alike)
          float v[2][32];
          uint32_t top = 0;
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            if (ok) outputs(2 * g + i, v[i]);
#pragma unroll
            for (int j = 0; j < 32; ++j) {
              if (c0 + (half * 2 + i) * 32 + j >= a.n) v[i][j] = 0.f;
              top = max(top, __float_as_uint(v[i][j]) & 0x7fffffffu);
            }
          }
          uint32_t* to = tops + turn * EPI_WARPS * 32;
          to[(warp - EPI_WARP) * 32 + lane] = top;
          rows_sync(sp);
          top = max(top, to[((warp - EPI_WARP) ^ 4) * 32 + lane]);
          turn ^= 1;
          if (!ok) continue;
          const int b = scale_byte(top);
          const uint64_t inv = both(scale_inverse(b));
          if (half == 0 && lane < left)
            a.y8.scales[(long long)(c0 / 128) * a.y8.lds + r0 + lane] = uint8_t(b);
          uint4 q[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            uint32_t w[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const float* s = v[k >> 1] + 16 * (k & 1) + 4 * j;
              w[j] = __byte_perm(e4m3x2(s[0], s[1], inv), e4m3x2(s[2], s[3], inv), 0x5410);
            }
            q[k] = make_uint4(w[0], w[1], w[2], w[3]);
          }
          const int c = c0 + half * 64;
          // (64 codes are as wide as 32 bf16 values; a box of bytes that crosses the last
          // column is cut off at 16 of them only)
          if (left >= 32 && (c + 64 <= a.n || a.n % 16 == 0)) {
            if (lane == 0) tma_store_wait_read<BUFS - 1>();  // this buffer's chunk has been read
            __syncwarp();
            const uint32_t s0 = saddr(own + buf * (CHUNK_STAGING / 2));
#pragma unroll
            for (int k = 0; k < 4; ++k)
              asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(
                               s0 + lane * 64 + 16 * (k ^ ((lane >> 1) & 3))),
                           "r"(q[k].x), "r"(q[k].y), "r"(q[k].z), "r"(q[k].w)
                           : "memory");
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0 && c < a.n) tma_store_2d(&tmY, s0, c, r0);
            buf ^= 1;
          } else if (lane < left) {
            uint8_t* dst = y + (long long)(r0 + lane) * ldy + c;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const int n = a.n - c - 16 * k;
              if (n >= 16) {
                *reinterpret_cast<uint4*>(dst + 16 * k) = q[k];
              } else {
                const uint32_t w[4] = {q[k].x, q[k].y, q[k].z, q[k].w};
#pragma unroll
                for (int j = 0; j < 16; ++j)
                  if (j < n) dst[16 * k + j] = uint8_t(w[j >> 2] >> (8 * (j & 3)));
              }
            }
          }
        }
      } else if (ok) {
#pragma unroll
        for (int i = 0; i < CHUNKS; ++i) {
          const int ch = chunk_of(i), c0 = tl.n * cols_out + ch * 32;
          if (left <= 0 || ch * 32 >= cols_out || c0 >= a.n) break;
          float v[32];
          outputs(i, v);
          if (a.tma && left >= 32) {
            if (lane == 0) tma_store_wait_read<BUFS - 1>();  // this buffer's chunk has been read
            __syncwarp();
            store_chunk<T>(&tmY, own + buf * (CHUNK_STAGING / 2), lane, v, r0, c0);
            if (BUFS == 2) buf ^= 1;
          } else {
            // (an earlier chunk may still be read from where this one goes)
            if (lane == 0) tma_store_wait_read<0>();
            __syncwarp();
            write_chunk(y + (long long)r0 * ldy + c0, ldy, left, a.n - c0, own, lane, v);
          }
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0 && ok) {
        if (PAIR) mbar_arrive_cluster(tempty_r0 + 8 * acc);
        else mbar_arrive(tempty0 + 8 * acc);
      }
      if (++acc == ACCS) { acc = 0; acc_phase ^= 1; }
    }
    if (MODE != SPLIT && lane == 0) tma_store_wait_read<0>();
  }
  if (MODE == SPLIT) {
    cluster_sync();
    if (pos < tiles) {
      // the rows' chunks of 32 outputs (128 with codes), dealt to the cluster's warps
      const Tile tl = tile_of(pos);
      const int rows = rows_of(tl, 0);
      constexpr int LANES = OUT == CODES ? 4 : 1;  // columns of a lane
      const int chunks = cols_out / (32 * LANES);
      const auto sum = [&](int col, int row) {
        float v = 0.f;
        for (int p = 0; p < parts; ++p) {
          float s;
          asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(s)
                       : "r"(mapa_shared(saddr(smem) + 4u * uint32_t(col * 129 + row),
                                         uint32_t(p))));
          v += s;
        }
        return v;
      };
      for (int u = part_of + warp * parts; u < rows * chunks; u += parts * (THREADS / 32)) {
        const int row = u % rows, ch = u / rows, place = tl.place + row;
        const int c0 = tl.n * cols_out + ch * 32 * LANES;
        if (c0 >= a.n) continue;
        float v[LANES];
#pragma unroll
        for (int i = 0; i < LANES; ++i) {
          const int col = (ch * LANES + i) * 32 + lane, c = c0 + i * 32 + lane;
          v[i] = 0.f;
          if (c >= a.n) continue;
          const float* b = a.bias ? a.bias + (long long)tl.expert * N + c : nullptr;
          v[i] = sum(col, row) + (b ? __ldg(b) : 0.f);
          v[i] = gated ? act_silu(v[i]) * (sum(half_bn + col, row) + (b ? __ldg(b + a.n) : 0.f))
                       : act_of(a.act, v[i]);
        }
        if constexpr (OUT == CODES) {
          uint32_t top = 0;
#pragma unroll
          for (int i = 0; i < LANES; ++i) top = max(top, __float_as_uint(v[i]) & 0x7fffffffu);
          top = __reduce_max_sync(~0u, top);
          const int b = scale_byte(top);
          const float inv = scale_inverse(b);
#pragma unroll
          for (int i = 0; i < LANES; ++i)
            if (c0 + i * 32 + lane < a.n)
              a.y8.codes[(long long)place * a.y8.ld + c0 + i * 32 + lane] =
                  uint8_t(e4m3x2(v[i] * inv, 0.f));
          if (lane == 0) a.y8.scales[(long long)(c0 / 128) * a.y8.lds + place] = uint8_t(b);
        } else if (c0 + lane < a.n) {
          static_cast<T*>(a.y)[(long long)place * a.ldy + c0 + lane] = T(v[0]);
        }
      }
    }
  }
  if (!ok) {
    *abort_flag = 1;
    atomicOr(a.err, DEVERR_TIMEOUT);
  }
  tc_fence_before();
  __syncthreads();
  // no CTA leaves while a peer may still load, commit, arrive or read there
  if (MODE != ALONE) cluster_sync();
  if (warp == 1) {
    __syncwarp();
    tc_fence_after();
    if (PAIR) tmem_dealloc_pair(tmem, TMEM_COLS);
    else tmem_dealloc(tmem, TMEM_COLS);
  }
}

constexpr int SMS = 152;

// Codes [rows][n] in boxes of 64 x 32 whose rows are swizzled over their own width.
cudaError_t tma_map_codes(const Fp8Mat& y, int rows, CUtensorMap* out) {
  auto fn = tma_encode_fn();
  if (!fn) return cudaErrorNotSupported;
  const cuuint64_t dims[2] = {cuuint64_t(y.cols), cuuint64_t(rows)};
  const cuuint64_t strides[1] = {cuuint64_t(y.ld)};
  const cuuint32_t box[2] = {64, 32}, es[2] = {1, 1};
  const CUresult r = fn(out, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, y.codes, dims, strides, box, es,
                        CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_64B,
                        CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

// The most tiles of `high` rows that `pairs` places of the experts can make.
long long most_tiles(const ExpertsArgs& a, int high) {
  const long long used = a.pairs < a.experts ? a.pairs : a.experts;
  return used + (a.pairs - used) / high;
}

struct Choice {
  Mode mode;
  int bn, parts;
};

template <Kind OUT, Mode MODE>
cudaError_t go(ExpertsArgs a, const Choice& ch, cudaStream_t st) {
  constexpr bool PAIR = MODE == PAIRS;
  using T = typename TypeOf<OUT>::T;
  // (an attribute of the current device, so set for each call)
  RC_TRY(cudaFuncSetAttribute(experts_linear_kernel<OUT, MODE>,
                              cudaFuncAttributeMaxDynamicSharedMemorySize, int(SMEM_BYTES)));
  const bool gated = a.act == RC_ACT_GATED_SILU;
  const int bn = ch.bn, cols_out = gated ? bn / 2 : bn;
  Plan pl;
  pl.bn = bn;
  const int fit = RING_BYTES / stage_bytes<PAIR>(bn);
  pl.stages = fit < MAX_STAGES ? fit : MAX_STAGES;
  pl.nt = (a.n - 1) / cols_out + 1;
  pl.kb = (a.x.cols - 1) / BK + 1;
  pl.parts = ch.parts;
  pl.accs = bn > ACC_BN ? 1 : 2;
  pl.most = int(most_tiles(a, PAIR ? 2 * BM : BM));
  const long long tiles = (long long)pl.most * pl.nt;
  if (tiles > 0x7fffffff - SMS) return cudaErrorInvalidValue;
  CUtensorMap mx, mg, mw, my;
  RC_TRY(tma_map_bytes(a.x.codes, a.x.rows, a.x.cols, a.x.ld, BM, &mx));
  RC_TRY(tma_map_bytes(a.x.codes, a.x.rows, a.x.cols, a.x.ld, 1, &mg));
  RC_TRY(tma_map_bytes(a.w.codes, a.w.rows, a.w.cols, a.w.ld, PAIR || gated ? bn / 2 : bn, &mw));
  my = mx;  // (not used without tma)
  if constexpr (OUT == CODES) {
    RC_TRY(tma_map_codes(a.y8, a.pairs, &my));
  } else {
    const uintptr_t row = uintptr_t(a.ldy) * sizeof(T);
    a.tma = ((reinterpret_cast<uintptr_t>(a.y) | row) & 15u) == 0;
    if (a.tma) RC_TRY(tma_map_chunks(static_cast<T*>(a.y), a.pairs, a.n, a.ldy, &my));
  }
  count_launches(1);
  const int cluster = PAIR ? 2 : ch.parts, slots = SMS / cluster;
  const unsigned ctas =
      unsigned(cluster * (MODE == SPLIT || tiles < slots ? int(tiles) : slots));
  if (MODE != ALONE)
    return launch_k_cluster(experts_linear_kernel<OUT, MODE>, dim3(ctas), dim3(THREADS),
                            SMEM_BYTES, cluster, st, mx, mg, mw, my, a, pl);
  return launch_k(experts_linear_kernel<OUT, MODE>, dim3(ctas), dim3(THREADS), SMEM_BYTES, st, mx,
                  mg, mw, my, a, pl);
}

// The tile width, and how CTAs share a tile, of least estimated duration (SM
// cycles; rates as rc_fp8_linear's), for experts with even shares of the places.
Choice choose(const ExpertsArgs& a, bool codes) {
  const bool gated = a.act == RC_ACT_GATED_SILU;
  const int kb = (a.x.cols - 1) / BK + 1;
  const long long used = a.pairs < a.experts ? a.pairs : a.experts;
  const double rows = double(a.pairs) / double(used);  // of an expert
  // (uneven shares: half a tile more for each expert)
  const auto m_tiles = [&](int high) { return rows <= high / 2 ? double(used)
                                                               : a.pairs / double(high) + 0.5 * used; };
  Choice best{ALONE, gated ? 256 : 128, 1};
  double least = 1e30;
  const auto look = [&](Mode mode, int bn, int parts) {
    const long long nt = (a.n - 1) / (gated ? bn / 2 : bn) + 1;
    const double tiles = m_tiles(mode == PAIRS ? 2 * BM : BM) * nt;
    const double x = rows < BM ? rows / BM : 1;  // of a full tile's rows
    double cost;
    if (mode == SPLIT) {
      if (most_tiles(a, BM) * nt * parts > SMS - 8) return;
      cost = (kb + parts - 1) / parts * (60 + 160 * x + 1.83 * bn) + 4.0 * bn + 600 + 800 * parts;
    } else {
      const double slots = mode == PAIRS ? SMS / 2 : SMS;
      const double waves = tiles <= slots ? 1 : ceil(tiles / slots - 0.05);
      cost = waves * (mode == PAIRS ? kb * (405 + 0.42 * bn) + 9.5 * bn
                                    : kb * (60 + 160 * x + 1.83 * bn) + 7.0 * bn);
      if (bn > ACC_BN) cost += (waves - 1) * 12.0 * bn;  // (the only accumulator is drained)
      if (mode == PAIRS) cost += 3000;
    }
    if (cost < least) {
      least = cost;
      best = Choice{mode, bn, parts};
    }
  };
  for (int bn = MAX_BN; bn >= 64; bn -= 32) {
    if (codes ? bn % (gated ? 256 : 128) : gated && bn % 64) continue;
    look(ALONE, bn, 1);
    if (rows > BM && bn >= 128) look(PAIRS, bn, 1);
    for (int parts = 2; parts <= 4 && parts <= kb; ++parts) look(SPLIT, bn, parts);
  }
  return best;
}

template <Kind OUT>
cudaError_t linear(const ExpertsArgs& a, cudaStream_t st) {
  const Choice c = choose(a, OUT == CODES);
  if (c.mode == PAIRS) return go<OUT, PAIRS>(a, c, st);
  if (c.mode == SPLIT) return go<OUT, SPLIT>(a, c, st);
  return go<OUT, ALONE>(a, c, st);
}

}  // namespace

cudaError_t launch_experts_linear(const ExpertsArgs& a, cudaStream_t st) {
  if (a.y8.codes) return linear<CODES>(a, st);
  return a.f32 ? linear<F32>(a, st) : linear<BF16>(a, st);
}

}  // namespace rc
