// Product of two quantised matrices (rc_fp8): y = x W^T + b on the
// block-scaled e4m3 MMA of the tensor core, which multiplies each row's
// products of 32 columns by that row's power-of-two scale (a byte in tensor
// memory) before it adds them, so a block of 128 columns costs four MMAs and
// no extra pass over the accumulator.
//
// Persistent CTAs of 16 warps: warp 0 loads x by TMA, warp 2 W (128 columns =
// 128 bytes a row, 128-byte swizzle; what lies outside the matrix reads as
// zero), warp 1 issues the MMAs, warps 4..7 put the scale bytes into tensor
// memory, warps 8..15 drain the accumulator.  A row's word there holds the
// bytes of four consecutive blocks, of which an MMA names one; the words of
// sixteen blocks (2048 columns) are stored and handed over together.  The
// hand-over is what must be rare: with one for every block, and bytes loaded
// where they were needed, 16384 x 1152 x 4608 took 301 us; with one for every
// four, and loads a batch ahead, 82; now 66 with f32 results (2.6 PFLOP/s, 2.9 at
// 60 with bf16).  What is left there: 384 tiles of 256 x 192 on 76 pairs are 5.05
// rounds and take six, and a pair's block of columns takes 486 cycles, of which
// its MMAs fill 384.  Two accumulators of up to 192 columns (or one of up to 256, where a CTA has one
// tile) and two batches of scale words fill the 512 columns of tensor memory.
#include "common.cuh"
#include "eight_bit.h"
#include "fp8.cuh"
#include "tc_eight_bit.cuh"
#include "tma_host.h"

namespace rc {

namespace {

using namespace rc::tc;

constexpr int BM = 128, BK = 128;
constexpr int THREADS = 512;
constexpr int SCALE_WARP = 4, EPI_WARP = 8, EPI_WARPS = 8;
constexpr int STAGE_A = BM * BK;
constexpr int RING_BYTES = 187 * 1024, MAX_STAGES = 7;
constexpr int STAGING_WARP = 32 * 128;  // 32 rows of 32 columns per epilogue warp
// tensor memory: accumulators at 0 and PAIR_BN, then a ring of scale words: a
// batch holds, for each WORD_KB blocks, 4 columns for x and 8 for W
constexpr int PAIR_BN = 192, MAX_BN = 256, SCALE_COL = 2 * PAIR_BN, TMEM_COLS = 512;
constexpr int WORD_KB = 4, SCALE_BATCH = 16, SCALE_GROUPS = SCALE_BATCH / WORD_KB;
constexpr int SCALE_STEP = 12, SCALE_SLOT = SCALE_GROUPS * SCALE_STEP, SCALES = 2;
static_assert(SCALE_COL + SCALES * SCALE_SLOT <= TMEM_COLS, "tensor memory");
// the batch's words in shared memory: up to 128 rows of x, up to 256 of W
constexpr int SCALE_ROWS = 128 + MAX_BN, SCALE_BYTES = SCALE_GROUPS * SCALE_ROWS * 4;
constexpr size_t SMEM_BYTES =
    size_t(RING_BYTES) + EPI_WARPS * STAGING_WARP + SCALE_BYTES + 1024 + 256;
// Instruction descriptor of kind::mxf8f6f4: e4m3 x e4m3 into f32, both
// K-major, power-of-two scale bytes; N >> 3 at bit 17, M >> 7 at bit 27, the
// byte of each scale word that the MMA takes at bits 4 (W) and 29 (x).
constexpr uint32_t IDESC = 1u << 23;

struct Plan {
  int bn, stages, mt, nt, tiles, kb, parts;
  int n_first;  // neighbouring tiles share rows of x (otherwise of W)
  __device__ __forceinline__ int m(int t) const { return n_first ? t / nt : t % mt; }
  __device__ __forceinline__ int n(int t) const { return n_first ? t % nt : t / mt; }
};
template <bool PAIR>
__host__ __device__ constexpr int stage_bytes(int bn) {
  return STAGE_A + (PAIR ? bn / 2 : bn) * BK;
}

template <class T>
struct Out {
  T* y;
  const float* bias;
  int ldy, rows, n;
  bool tma;  // y's rows are 16-byte aligned: chunks leave by TMA
  unsigned* err;
};

// One warp's 32 x 32 chunk of the accumulator (lane = row r0 + lane, v = its
// columns c0 .., `bias` that of column c0 + lane), by way of the warp's own
// shared memory.
// TMA: in the layout of a box of 32 columns with a swizzle as wide as its rows
// (which also keeps the row-per-lane writes free of bank conflicts); what lies
// outside y is not written.
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
// Any alignment: neighbouring lanes write neighbouring columns.
template <class T>
__device__ __forceinline__ void write_chunk(const Out<T>& o, uint8_t* stg, int lane,
                                            const float* v, int r0, int c0) {
  float* s = reinterpret_cast<float*>(stg);
#pragma unroll
  for (int j = 0; j < 32; ++j) s[lane * 32 + (j ^ lane)] = v[j];
  __syncwarp();
  const int rows = min(32, o.rows - r0);
  if (lane < o.n - c0) {
    T* y = o.y + (long long)r0 * o.ldy + c0 + lane;
    for (int row = 0; row < rows; ++row, y += o.ldy) *y = T(s[row * 32 + (lane ^ row)]);
  }
  __syncwarp();  // the staging area is rewritten by the next chunk
}

// Named barrier of the four scale warps.
__device__ __forceinline__ void scale_sync() { asm volatile("bar.sync 1, 128;" ::: "memory"); }

// How CTAs work together.  PAIR: clusters of two share each MMA (M = 256): a
// CTA loads its own 128 rows of x and half of the W tile.  SPLIT: a cluster
// shares a tile's blocks of columns; each CTA leaves its part in shared
// memory, and the parts are added there in the order of the ranks.
enum Mode { ALONE, PAIRS, SPLIT };

template <class T, Mode MODE>
__global__ void __launch_bounds__(THREADS, 1)
fp8_linear_kernel(const __grid_constant__ CUtensorMap tmX, const __grid_constant__ CUtensorMap tmW,
                  const __grid_constant__ CUtensorMap tmY,
                  const __grid_constant__ Fp8Mat x, const __grid_constant__ Fp8Mat w,
                  const __grid_constant__ Out<T> out, const __grid_constant__ Plan pl) {
  constexpr bool PAIR = MODE == PAIRS;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                             ~uintptr_t(1023));
  uint8_t* stg = smem + RING_BYTES;
  uint32_t* words = reinterpret_cast<uint32_t*>(stg + EPI_WARPS * STAGING_WARP);
  uint64_t* bars = reinterpret_cast<uint64_t*>(stg + EPI_WARPS * STAGING_WARP + SCALE_BYTES);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 2 * MAX_STAGES + 2 * SCALES + 4);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  const uint32_t full0 = saddr(bars), empty0 = full0 + 8 * MAX_STAGES;
  const uint32_t sfull0 = empty0 + 8 * MAX_STAGES, sempty0 = sfull0 + 8 * SCALES;
  const uint32_t tfull0 = sempty0 + 8 * SCALES, tempty0 = tfull0 + 16;

  const int warp = warp_index(), lane = threadIdx.x & 31;
  const uint32_t rank = PAIR ? cluster_ctarank() : 0;  // in a pair
  constexpr int CTAS = PAIR ? 2 : 1;
  if (threadIdx.x == 0) {
    for (int s = 0; s < MAX_STAGES; ++s) {
      mbar_init(full0 + 8 * s, PAIR ? 1 : 2);  // (x's and W's loads)
      mbar_init(empty0 + 8 * s, 1);
    }
    for (int s = 0; s < SCALES; ++s) {
      mbar_init(sfull0 + 8 * s, 4 * CTAS);
      mbar_init(sempty0 + 8 * s, 1);
    }
    for (int a = 0; a < 2; ++a) {
      mbar_init(tfull0 + 8 * a, 1);
      mbar_init(tempty0 + 8 * a, EPI_WARPS * CTAS);
    }
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    if (PAIR) tmem_alloc_pair(saddr(tmem_slot), TMEM_COLS);
    else tmem_alloc(saddr(tmem_slot), TMEM_COLS);
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  if (PAIR) cluster_sync();  // (the peer's barriers are ready)

  const int BN = pl.bn, STAGES = pl.stages;
  const int STAGE = stage_bytes<PAIR>(BN);
  // this CTA's (or pair's) tiles pos, pos + G .. and, of each, its blocks
  // k0 .. k0 + KB - 1
  const int parts = MODE == SPLIT ? pl.parts : 1;
  const int part_of = MODE == SPLIT ? int(cluster_ctarank()) : 0;
  const int k0 = part_of * pl.kb / parts, KB = (part_of + 1) * pl.kb / parts - k0;
  const int G = int(gridDim.x) / (CTAS * parts), pos = int(blockIdx.x) / (CTAS * parts);
  bool ok = true;

  if (warp == 0 || warp == 2) {
    // ------------------------------------------------------------ TMA: x, W
    if (elect_one()) {
      pdl_wait();
      if (warp == 0) pdl_trigger();
      int stage = 0;
      uint32_t phase = 0;
      for (int t = pos; ok && t < pl.tiles; t += G) {
        const int m = pl.m(t) * CTAS + int(rank), nn = pl.n(t);
        for (int kb = 0; kb < KB; ++kb) {
          if (!mbar_wait(empty0 + 8 * stage, phase ^ 1, abort_flag)) { ok = false; break; }
          const uint32_t st = saddr(smem + stage * STAGE), fb = full0 + 8 * stage;
          // (a barrier may see bytes before it is told of them: its phase still
          // needs that arrival)
          if (PAIR) {  // both CTAs' bytes land on rank 0's barrier
            const uint32_t f0 = mapa_shared(fb, 0);
            if (warp == 0) {
              if (rank == 0) mbar_expect_tx(fb, 2 * STAGE);
              tma_load_2d_pair(st, &tmX, f0, (k0 + kb) * BK, m * BM);
            } else {
              tma_load_2d_pair(st + STAGE_A, &tmW, f0, (k0 + kb) * BK,
                               nn * BN + int(rank) * (BN / 2));
            }
          } else if (warp == 0) {
            mbar_expect_tx(fb, STAGE_A);
            tma_load_2d(st, &tmX, fb, (k0 + kb) * BK, m * BM);
          } else {
            mbar_expect_tx(fb, STAGE - STAGE_A);
            tma_load_2d(st + STAGE_A, &tmW, fb, (k0 + kb) * BK, nn * BN);
          }
          if (++stage == STAGES) { stage = 0; phase ^= 1; }
        }
      }
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------ MMA issuer
    if (rank == 0 && elect_one()) {
      const uint32_t idesc =
          IDESC | (uint32_t(BN >> 3) << 17) | (uint32_t(PAIR ? 2 : 1) << 27);
      const uint64_t da = sw128_desc(saddr(smem)), db = sw128_desc(saddr(smem + STAGE_A));
      int stage = 0, acc = 0, sc = 0;
      uint32_t phase = 0, acc_phase = 0, sc_phase = 0;
      uint64_t so = 0;     // the stage's offset in the descriptors' address field
      bool ready = false;  // the current stage was seen full already
      for (int t = pos; ok && t < pl.tiles; t += G) {
        if (!mbar_wait(tempty0 + 8 * acc, acc_phase ^ 1, abort_flag)) { ok = false; break; }
        const uint32_t d = tmem + uint32_t(acc * PAIR_BN);
        uint32_t accumulate = 0;
        // (what a block's issue needs beyond its stage is constant or one
        // addition a group away: the issuing thread is what bounds small tiles)
        for (int kb = 0; ok && kb < KB;) {
          if (!mbar_wait(sfull0 + 8 * sc, sc_phase, abort_flag)) { ok = false; break; }
          uint32_t sa = tmem + uint32_t(SCALE_COL + sc * SCALE_SLOT);
          const int end = min(kb + SCALE_BATCH, KB);
          while (ok && kb < end) {
#pragma unroll
            for (int byte = 0; byte < WORD_KB; ++byte) {
              if (kb >= end) break;
              if (!ready && !mbar_wait(full0 + 8 * stage, phase, abort_flag)) { ok = false; break; }
              const uint64_t a = da + so, b = db + so;
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
                  umma_e4m3_scaled_pair(d, a + 2 * kk, b + 2 * kk, id, sa, sa + 4, accumulate);
                else
                  umma_e4m3_scaled(d, a + 2 * kk, b + 2 * kk, id, sa, sa + 4, accumulate);
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
        if (++acc == 2) { acc = 0; acc_phase ^= 1; }
      }
    }
  } else if (warp >= SCALE_WARP && warp < EPI_WARP) {
    // -------------------------------------------------------- scale words
    pdl_wait();
    // The bytes of the next batch are under way (without a branch, from
    // clamped places) while this one's words go by way of shared memory into
    // tensor memory.  A thread loads sixteen blocks' bytes of one row of x and
    // of two of W; where 128 rows share a scale, one byte of the three shared
    // rows that a tile can meet.  Rows and blocks that there are none of
    // multiply zeros and take the scale 1.
    const int tid = int(threadIdx.x) - SCALE_WARP * 32;
    const uint32_t part = uint32_t((warp & 3) * 32) << 16;
    uint8_t bx[SCALE_BATCH], bw[2][SCALE_BATCH];
    const auto load = [&](const Fp8Mat& o, int row0, int r, int kb, uint8_t* b) {
      if (o.group == 1) {
        const uint8_t* p = o.scales + min(row0 + r, o.rows - 1);
#pragma unroll
        for (int u = 0; u < SCALE_BATCH; ++u)
          b[u] = p[(long long)min(k0 + kb + u, pl.kb - 1) * o.lds];
      } else {
        const int e = min(row0 / 128 + r / SCALE_BATCH, (o.rows - 1) / 128);
        b[0] = o.scales[(long long)min(k0 + kb + r % SCALE_BATCH, pl.kb - 1) * o.lds + e];
      }
    };
    // the words of up to `most` rows, or of three shared ones, at `to`
    const auto keep = [&](const Fp8Mat& o, int row0, int r, int most, const uint8_t* b,
                          uint32_t* to) {
      if (o.group == 1) {
        if (r >= most) return;
        const bool in = row0 + r < o.rows;
#pragma unroll
        for (int g = 0; g < SCALE_GROUPS; ++g)
          to[g * SCALE_ROWS + r] =
              in ? uint32_t(b[4 * g]) | uint32_t(b[4 * g + 1]) << 8 |
                       uint32_t(b[4 * g + 2]) << 16 | uint32_t(b[4 * g + 3]) << 24
                 : 0x7f7f7f7fu;
      } else if (r < 3 * SCALE_BATCH) {
        const int u = r % SCALE_BATCH;
        reinterpret_cast<uint8_t*>(to + u / WORD_KB * SCALE_ROWS + r / SCALE_BATCH)[u % WORD_KB] =
            b[0];
      }
    };
    const int m_rows = x.group == 1 ? 1 : 0, w_rows = w.group == 1 ? 1 : 0;
    const auto fetch = [&](int t, int kb) {
      load(x, (pl.m(t) * CTAS + int(rank)) * BM, tid, kb, bx);
      load(w, pl.n(t) * BN, tid, kb, bw[0]);
      if (w_rows) load(w, pl.n(t) * BN, tid + 128, kb, bw[1]);
    };
    int sc = 0, t = pos, kb = 0;
    uint32_t sc_phase = 0;
    if (t < pl.tiles) fetch(t, kb);
    while (t < pl.tiles) {
      const int x0 = (pl.m(t) * CTAS + int(rank)) * BM, w0 = pl.n(t) * BN;
      scale_sync();  // (the batch before has been taken)
      keep(x, x0, tid, 128, bx, words);
      keep(w, w0, tid, MAX_BN, bw[0], words + 128);
      if (w_rows) keep(w, w0, tid + 128, MAX_BN, bw[1], words + 128);
      scale_sync();
      kb += SCALE_BATCH;
      if (kb >= KB) { kb = 0; t += G; }
      if (t < pl.tiles) fetch(t, kb);
      if (ok) ok = mbar_sleep(sempty0 + 8 * sc, sc_phase ^ 1, abort_flag);
      // (after a failed wait the warp goes on to the barriers, without work)
      ok = __all_sync(0xffffffffu, ok);
      if (ok) {
        tc_fence_after();
        uint32_t v[SCALE_SLOT];
#pragma unroll
        for (int g = 0; g < SCALE_GROUPS; ++g) {
#pragma unroll
          for (int i = 0; i < 4; ++i)
            v[g * SCALE_STEP + i] = words[g * SCALE_ROWS + (m_rows ? 32 * i + lane : 0)];
#pragma unroll
          for (int i = 0; i < 8; ++i)
            v[g * SCALE_STEP + 4 + i] =
                words[g * SCALE_ROWS + 128 +
                      (w_rows ? 32 * i + lane : (w0 + 32 * i + lane) / 128 - w0 / 128)];
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
    pdl_wait();
    const int sp = warp & 3, half = (warp - EPI_WARP) >> 2;
    const uint32_t tempty_r0 = PAIR ? mapa_shared(tempty0, 0) : tempty0;
    uint8_t* own = stg + (warp - EPI_WARP) * STAGING_WARP;
    constexpr int BUFS = sizeof(T) == 4 ? 1 : 2;  // staging of this many chunks
    int acc = 0, buf = 0;
    uint32_t acc_phase = 0;
    for (int t = pos; t < pl.tiles; t += G) {
      const int m = pl.m(t) * CTAS + int(rank), nn = pl.n(t);
      // (the bias before the accumulator is ready)
      float bias[MAX_BN / 64];
#pragma unroll
      for (int i = 0; i < MAX_BN / 64; ++i) {
        const int c = nn * BN + (half + 2 * i) * 32 + lane;
        bias[i] = out.bias && c < out.n ? __ldg(out.bias + c) : 0.f;
      }
      if (!mbar_sleep_warp(tfull0 + 8 * acc, acc_phase, abort_flag)) { ok = false; break; }
      tc_fence_after();
      const uint32_t tb = tmem + uint32_t(acc * PAIR_BN) + (uint32_t(sp * 32) << 16);
#pragma unroll
      for (int i = 0; i < MAX_BN / 64; ++i) {
        const int ch = half + 2 * i, r0 = m * BM + sp * 32, c0 = nn * BN + ch * 32;
        if (ch >= BN / 32 || r0 >= out.rows || c0 >= out.n) break;
        float v[32];
        tmem_ld32(tb + uint32_t(ch * 32), v);
        if (MODE == SPLIT) {  // (every MMA is done: the operand ring is free)
          float* to = reinterpret_cast<float*>(smem + (ch * 4 + sp) * 4096);
#pragma unroll
          for (int j = 0; j < 32; ++j) to[32 * j + lane] = v[j];
          continue;
        }
        if (out.bias)
#pragma unroll
          for (int j = 0; j < 32; ++j) v[j] += __shfl_sync(0xffffffffu, bias[i], j);
        if (out.tma) {
          if (lane == 0) tma_store_wait_read<BUFS - 1>();  // this buffer's chunk has been read
          __syncwarp();
          store_chunk<T>(&tmY, own + buf * (STAGING_WARP / 2), lane, v, r0, c0);
          if (BUFS == 2) buf ^= 1;
        } else {
          write_chunk(out, own, lane, v, r0, c0);
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) {
        if (PAIR) mbar_arrive_cluster(tempty_r0 + 8 * acc);
        else mbar_arrive(tempty0 + 8 * acc);
      }
      if (++acc == 2) { acc = 0; acc_phase ^= 1; }
    }
    if (MODE != SPLIT && lane == 0) tma_store_wait_read<0>();
  }
  if (MODE == SPLIT) {
    // chunk u of the tile (32 rows x 32 columns) is finished by CTA u mod
    // parts of the cluster, by one of its epilogue warps
    cluster_sync();
    if (warp >= EPI_WARP) {
      const int m = pl.m(pos), nn = pl.n(pos);
      uint8_t* own = stg + (warp - EPI_WARP) * STAGING_WARP;
      for (int u = part_of + (warp - EPI_WARP) * parts; u < BN / 8; u += EPI_WARPS * parts) {
        const int r0 = m * BM + (u & 3) * 32, c0 = nn * BN + (u >> 2) * 32;
        if (r0 >= out.rows || c0 >= out.n) continue;
        const float b = out.bias && c0 + lane < out.n ? __ldg(out.bias + c0 + lane) : 0.f;
        float v[32] = {};
        for (int p = 0; p < parts; ++p) {
          const uint32_t from = mapa_shared(saddr(smem + u * 4096), uint32_t(p)) + 4 * lane;
#pragma unroll
          for (int j = 0; j < 32; ++j) {
            float a;
            asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(a) : "r"(from + 128 * j));
            v[j] += a;
          }
        }
#pragma unroll
        for (int j = 0; j < 32; ++j) v[j] += __shfl_sync(0xffffffffu, b, j);
        if (out.tma) {
          if (lane == 0) tma_store_wait_read<0>();
          __syncwarp();
          store_chunk<T>(&tmY, own, lane, v, r0, c0);
        } else {
          write_chunk(out, own, lane, v, r0, c0);
        }
      }
      if (lane == 0) tma_store_wait_read<0>();
    }
  }
  if (!ok) {
    *abort_flag = 1;
    atomicOr(out.err, DEVERR_TIMEOUT);
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

template <class T, Mode MODE>
cudaError_t go(const Fp8Mat& x, const Fp8Mat& w, const Out<T>& o, int bn, int parts,
               cudaStream_t st) {
  constexpr bool PAIR = MODE == PAIRS;
  // (an attribute of the current device, so set for each call)
  RC_TRY(cudaFuncSetAttribute(fp8_linear_kernel<T, MODE>,
                              cudaFuncAttributeMaxDynamicSharedMemorySize, int(SMEM_BYTES)));
  Plan pl;
  pl.bn = bn;
  const int fit = RING_BYTES / stage_bytes<PAIR>(bn);
  pl.stages = fit < MAX_STAGES ? fit : MAX_STAGES;
  const int rows = BM * (PAIR ? 2 : 1);
  pl.mt = int((x.rows + (long long)rows - 1) / rows);
  pl.nt = int((w.rows + (long long)bn - 1) / bn);
  pl.kb = (x.cols + BK - 1) / BK;
  pl.parts = parts;
  pl.n_first = w.rows < x.rows;
  const long long tiles = (long long)pl.mt * pl.nt;
  if (tiles > 0x7fffffff - SMS) return cudaErrorInvalidValue;
  pl.tiles = int(tiles);
  CUtensorMap mx, mw, my;
  RC_TRY(tma_map_bytes(x.codes, x.rows, x.cols, x.ld, BM, &mx));
  RC_TRY(tma_map_bytes(w.codes, w.rows, w.cols, w.ld, PAIR ? bn / 2 : bn, &mw));
  my = mx;  // (not used without out.tma)
  if (o.tma) RC_TRY(tma_map_chunks(o.y, o.rows, o.n, o.ldy, &my));
  count_launches(1);
  const int cluster = PAIR ? 2 : parts, slots = SMS / cluster;
  const unsigned ctas =
      unsigned(cluster * (MODE == SPLIT || pl.tiles < slots ? pl.tiles : slots));
  if (MODE != ALONE)
    return launch_k_cluster(fp8_linear_kernel<T, MODE>, dim3(ctas), dim3(THREADS), SMEM_BYTES,
                            cluster, st, mx, mw, my, x, w, o, pl);
  return launch_k(fp8_linear_kernel<T, MODE>, dim3(ctas), dim3(THREADS), SMEM_BYTES, st, mx, mw,
                  my, x, w, o, pl);
}

// The tile width, and how CTAs share a tile, of least estimated duration (SM
// cycles).  Rates measured on products of 1152 and 4608 columns at 39 to 16384
// rows: a CTA's block of columns takes 220 + 1.83 BN (its loads: TMA brings
// about 70 B/clk to an SM), a pair's 405 + 0.42 BN, and a tile's change 7 to
// 9.5 BN more; a launch of pairs takes 3000 longer (16384 x
// 1152 x 4608: pairs of 192 60.0 us, alone 68.2; 831 x 3456 x 1152: 8.9 and
// 7.3; 4096 x 1152 x 4608: alone at 128 21.2 us, pairs 24.1).  Adding
// the parts of a split tile takes 600 + 800 a part (39 x 1152 x 4608: one CTA
// a tile 9.4 us, four 7; 39 x 1152 x 1152: one 4.9, two 5.9).  Clusters above
// four CTAs do not all find a place at once and take twice as long.
struct Choice {
  Mode mode;
  int bn, parts;
};
Choice choose(long long rows, long long n, int kb) {
  Choice best{ALONE, 64, 1};
  double least = 1e30;
  const auto look = [&](Mode mode, int bn, int parts) {
    const long long high = mode == PAIRS ? 2 * BM : BM;
    const long long tiles = ((rows + high - 1) / high) * ((n + bn - 1) / bn);
    double cost;
    if (mode == SPLIT) {
      if (tiles * parts > SMS - 8) return;
      cost = (kb + parts - 1) / parts * (220 + 1.83 * bn) + 7.0 * bn + 600 + 800 * parts;
    } else {
      const long long slots = mode == PAIRS ? SMS / 2 : SMS, waves = (tiles + slots - 1) / slots;
      cost = double(waves) * (mode == PAIRS ? kb * (405 + 0.42 * bn) + 9.5 * bn
                                            : kb * (220 + 1.83 * bn) + 7.0 * bn);
      if (mode == PAIRS) cost += 3000;
    }
    if (cost < least) {
      least = cost;
      best = Choice{mode, bn, parts};
    }
  };
  for (int bn = MAX_BN; bn >= 64; bn -= 32) {
    // (the wider tiles have one accumulator: no second tile)
    if (bn > PAIR_BN && ((rows + BM - 1) / BM) * ((n + bn - 1) / bn) > SMS) continue;
    look(ALONE, bn, 1);
    if (rows > BM && bn >= 128 && bn <= PAIR_BN) look(PAIRS, bn, 1);
  }
  for (int parts = 2; parts <= 4 && parts <= kb; ++parts) look(SPLIT, 64, parts);
  return best;
}

template <class T>
cudaError_t linear(const Fp8Mat& x, const Fp8Mat& w, const float* b, T* y, int ldy, unsigned* err,
                   cudaStream_t st) {
  const uintptr_t row = uintptr_t(ldy) * sizeof(T);
  const Out<T> o{y, b, ldy, x.rows, w.rows,
                 ((reinterpret_cast<uintptr_t>(y) | row) & 15u) == 0, err};
  const Choice c = choose(x.rows, w.rows, (x.cols + BK - 1) / BK);
  if (c.mode == PAIRS) return go<T, PAIRS>(x, w, o, c.bn, 1, st);
  if (c.mode == SPLIT) return go<T, SPLIT>(x, w, o, c.bn, c.parts, st);
  return go<T, ALONE>(x, w, o, c.bn, 1, st);
}

}  // namespace

cudaError_t launch_fp8_linear(const Fp8Mat& x, const Fp8Mat& w, const float* b, void* y, int ldy,
                              bool f32, unsigned* err, cudaStream_t st) {
  if (f32) return linear(x, w, b, static_cast<float*>(y), ldy, err, st);
  return linear(x, w, b, static_cast<bf16*>(y), ldy, err, st);
}

}  // namespace rc
