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
// bytes of four consecutive blocks, of which an MMA names one, so a word is
// written (in each of the four lane partitions) once for 512 columns; with a
// word and a handshake for every block the scale warps held up the MMAs
// (16384 x 1152 x 4608: 301 us).  Two accumulators of up to 224 columns and
// a ring of scale words fill the 512 columns of tensor memory.
#include "common.cuh"
#include "fp8.cuh"
#include "kernels.h"
#include "tc_common.cuh"
#include "tma_host.h"

namespace rc {

namespace {

using namespace rc::tc;

constexpr int BM = 128, BK = 128;
constexpr int THREADS = 512;
constexpr int SCALE_WARP = 4, EPI_WARP = 8, EPI_WARPS = 8;
constexpr int STAGE_A = BM * BK;
constexpr int RING_BYTES = 188 * 1024, MAX_STAGES = 7;
constexpr int STAGING_WARP = 32 * 128;  // 32 rows of 32 f32 per epilogue warp
// tensor memory: accumulators at 0 and MAX_BN, then a ring of scale words
// (4 columns for x, up to 7 for W), each for WORD_KB blocks
constexpr int MAX_BN = 224, SCALE_COL = 2 * MAX_BN, SCALE_STEP = 12, TMEM_COLS = 512;
constexpr int SCALES = 5, WORD_KB = 4;
// the scale words of a batch of blocks in shared memory: 128 rows of x, then
// up to 224 of W
constexpr int SCALE_BATCH = 16, SCALE_ROWS = 128 + MAX_BN;
constexpr int SCALE_BYTES = SCALE_BATCH / WORD_KB * SCALE_ROWS * 4;
constexpr size_t SMEM_BYTES =
    size_t(RING_BYTES) + EPI_WARPS * STAGING_WARP + SCALE_BYTES + 1024 + 256;
static_assert(SCALE_COL + SCALES * SCALE_STEP <= TMEM_COLS, "tensor memory");
// Instruction descriptor of kind::mxf8f6f4: e4m3 x e4m3 into f32, both
// K-major, power-of-two scale bytes; N >> 3 at bit 17, M >> 7 at bit 27, the
// byte of each scale word that the MMA takes at bits 4 (W) and 29 (x).
constexpr uint32_t IDESC = 1u << 23;

struct Plan {
  int bn, stages, mt, nt, tiles, kb;
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
  bool wide;  // rows are 16-byte aligned
  unsigned* err;
};

// One warp's 32 x 32 chunk of the accumulator (lane = row r0 + lane, v = its
// columns c0 ..): through shared memory, XOR-swizzled in 16-byte units, so
// that neighbouring lanes write neighbouring columns.
template <class T>
__device__ __forceinline__ void write_chunk(const Out<T>& o, uint8_t* stg, int lane,
                                            const float* v, int r0, int c0) {
  const uint32_t s0 = saddr(stg);
#pragma unroll
  for (int j = 0; j < 8; ++j)
    asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(
                     s0 + lane * 128 + 16 * (j ^ (lane & 7))),
                 "f"(v[4 * j]), "f"(v[4 * j + 1]), "f"(v[4 * j + 2]), "f"(v[4 * j + 3])
                 : "memory");
  __syncwarp();
  const int rows = min(32, o.rows - r0), cols = min(32, o.n - c0);
  if (o.wide && cols == 32) {
    constexpr int PER = 16 / sizeof(T), GROUPS = 32 / PER, STEP = 32 / GROUPS;
    const int g = lane % GROUPS;
    float b[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) b[i] = o.bias ? __ldg(o.bias + c0 + g * PER + i) : 0.f;
#pragma unroll
    for (int p = 0; p < 32 / STEP; ++p) {
      const int row = p * STEP + lane / GROUPS;
      float x[PER];
#pragma unroll
      for (int i = 0; i < PER / 4; ++i) {
        const float4 q = *reinterpret_cast<const float4*>(
            stg + row * 128 + 16 * ((g * (PER / 4) + i) ^ (row & 7)));
        x[4 * i] = q.x + b[4 * i];
        x[4 * i + 1] = q.y + b[4 * i + 1];
        x[4 * i + 2] = q.z + b[4 * i + 2];
        x[4 * i + 3] = q.w + b[4 * i + 3];
      }
      if (row < rows) {
        T* dst = o.y + (long long)(r0 + row) * o.ldy + c0 + g * PER;
        if constexpr (sizeof(T) == 4)
          *reinterpret_cast<float4*>(dst) = make_float4(x[0], x[1], x[2], x[3]);
        else
          *reinterpret_cast<uint4*>(dst) =
              make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]),
                         pack_bf16x2(x[PER - 4], x[PER - 3]), pack_bf16x2(x[PER - 2], x[PER - 1]));
      }
    }
  } else if (lane < cols) {
    const float b = o.bias ? __ldg(o.bias + c0 + lane) : 0.f;
    for (int row = 0; row < rows; ++row) {
      const float x = *reinterpret_cast<const float*>(stg + row * 128 +
                                                      16 * ((lane >> 2) ^ (row & 7)) +
                                                      4 * (lane & 3)) + b;
      o.y[(long long)(r0 + row) * o.ldy + c0 + lane] = T(x);
    }
  }
  __syncwarp();  // the staging area is rewritten by the next chunk
}

// Named barrier of the four scale warps.
__device__ __forceinline__ void scale_sync() { asm volatile("bar.sync 1, 128;" ::: "memory"); }

// PAIR: clusters of two CTAs share each MMA (M = 256): a CTA loads its own 128
// rows of x and half of the W tile.
template <class T, bool PAIR>
__global__ void __launch_bounds__(THREADS, 1)
fp8_linear_kernel(const __grid_constant__ CUtensorMap tmX, const __grid_constant__ CUtensorMap tmW,
                  const __grid_constant__ Fp8Mat x, const __grid_constant__ Fp8Mat w,
                  const __grid_constant__ Out<T> out, const __grid_constant__ Plan pl) {
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                             ~uintptr_t(1023));
  uint8_t* stg = smem + RING_BYTES;
  uint32_t* sw_words = reinterpret_cast<uint32_t*>(stg + EPI_WARPS * STAGING_WARP);
  uint64_t* bars = reinterpret_cast<uint64_t*>(stg + EPI_WARPS * STAGING_WARP + SCALE_BYTES);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 2 * MAX_STAGES + 2 * SCALES + 4);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  const uint32_t full0 = saddr(bars), empty0 = full0 + 8 * MAX_STAGES;
  const uint32_t sfull0 = empty0 + 8 * MAX_STAGES, sempty0 = sfull0 + 8 * SCALES;
  const uint32_t tfull0 = sempty0 + 8 * SCALES, tempty0 = tfull0 + 16;

  const int warp = warp_index(), lane = threadIdx.x & 31;
  const uint32_t rank = PAIR ? cluster_ctarank() : 0;
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

  const int BN = pl.bn, STAGES = pl.stages, KB = pl.kb;
  const int STAGE = stage_bytes<PAIR>(BN);
  const int G = int(gridDim.x) / CTAS, pos = int(blockIdx.x) / CTAS;
  bool ok = true;

  if (warp == 0 || (warp == 2 && !PAIR)) {
    // ------------------------------------------------- TMA: x (and W for pairs), W
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
          if (PAIR) {  // (both CTAs' bytes land on rank 0's barrier)
            if (rank == 0) mbar_expect_tx(fb, 2 * STAGE);
            const uint32_t f0 = mapa_shared(fb, 0);
            tma_load_2d_pair(st, &tmX, f0, kb * BK, m * BM);
            tma_load_2d_pair(st + STAGE_A, &tmW, f0, kb * BK, nn * BN + int(rank) * (BN / 2));
          } else if (warp == 0) {
            mbar_expect_tx(fb, STAGE_A);
            tma_load_2d(st, &tmX, fb, kb * BK, m * BM);
          } else {
            mbar_expect_tx(fb, STAGE - STAGE_A);
            tma_load_2d(st + STAGE_A, &tmW, fb, kb * BK, nn * BN);
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
      bool ready = false;  // the current stage was seen full already
      for (int t = pos; ok && t < pl.tiles; t += G) {
        if (!mbar_wait(tempty0 + 8 * acc, acc_phase ^ 1, abort_flag)) { ok = false; break; }
        const uint32_t d = tmem + uint32_t(acc * MAX_BN);
        for (int kb = 0; kb < KB; ++kb) {
          const int byte = kb % WORD_KB;
          if (byte == 0 && !mbar_wait(sfull0 + 8 * sc, sc_phase, abort_flag)) { ok = false; break; }
          if (!ready && !mbar_wait(full0 + 8 * stage, phase, abort_flag)) { ok = false; break; }
          const uint64_t so = uint64_t((stage * STAGE) >> 4);
          const uint32_t eb = empty0 + 8 * stage;
          if (++stage == STAGES) { stage = 0; phase ^= 1; }
          // (the next stage's test runs beside this one's MMAs)
          ready = mbar_test(full0 + 8 * stage, phase);
          tc_fence_after();
          const uint32_t sa = tmem + uint32_t(SCALE_COL + sc * SCALE_STEP), sb = sa + 4;
          const uint32_t id = idesc | uint32_t(byte) << 4 | uint32_t(byte) << 29;
#pragma unroll
          for (int kk = 0; kk < BK / 32; ++kk) {
            if (PAIR)
              umma_e4m3_scaled_pair(d, da + so + 2 * kk, db + so + 2 * kk, id, sa, sb,
                                    (kb | kk) ? 1u : 0u);
            else
              umma_e4m3_scaled(d, da + so + 2 * kk, db + so + 2 * kk, id, sa, sb,
                               (kb | kk) ? 1u : 0u);
          }
          if (PAIR) umma_commit_pair(eb);
          else umma_commit(eb);
          if (byte == WORD_KB - 1 || kb == KB - 1) {
            if (PAIR) umma_commit_pair(sempty0 + 8 * sc);
            else umma_commit(sempty0 + 8 * sc);
            if (++sc == SCALES) { sc = 0; sc_phase ^= 1; }
          }
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
    const int sx = x.group == 1 ? 0 : 7, sw = w.group == 1 ? 0 : 7;
    const uint32_t part = uint32_t((warp & 3) * 32) << 16;
    // A batch is the bytes of SCALE_BATCH blocks: each of the 128 threads loads
    // those of one row of x and of two of W, without a branch and from clamped
    // places, so that the loads are under way together (beside the operand
    // stream one round trip takes longer than the MMAs of four blocks), packs
    // them into words and leaves the words in shared memory, where every warp
    // takes what it stores.  The next batch's loads run meanwhile.  Rows and
    // blocks that there are none of multiply zeros and take the scale 1.
    const int tid = int(threadIdx.x) - SCALE_WARP * 32;
    uint32_t next[3][SCALE_BATCH / WORD_KB];
    const auto load = [&](int t, int kb) {
      const int m = pl.m(t) * CTAS + int(rank), nn = pl.n(t);
#pragma unroll
      for (int i = 0; i < 3; ++i) {
        const int r = i == 0 ? m * BM + tid : nn * BN + (i - 1) * 128 + tid;
        const int rows = i == 0 ? x.rows : w.rows;
        const uint8_t* p = i == 0 ? x.scales + (min(r, rows - 1) >> sx)
                                  : w.scales + (min(r, rows - 1) >> sw);
        const long long step = i == 0 ? x.lds : w.lds;
#pragma unroll
        for (int g = 0; g < SCALE_BATCH / WORD_KB; ++g) {
          uint32_t b[WORD_KB];
#pragma unroll
          for (int u = 0; u < WORD_KB; ++u) b[u] = p[min(kb + g * WORD_KB + u, KB - 1) * step];
          const uint32_t word = b[0] | b[1] << 8 | b[2] << 16 | b[3] << 24;
          next[i][g] = r < rows ? word : 0x7f7f7f7fu;
        }
      }
    };
    int sc = 0, t = pos, kb = 0;
    uint32_t sc_phase = 0;
    if (t < pl.tiles) load(t, kb);
    while (t < pl.tiles) {
      scale_sync();  // (the batch before has been taken)
#pragma unroll
      for (int i = 0; i < 3; ++i)
#pragma unroll
        for (int g = 0; g < SCALE_BATCH / WORD_KB; ++g)
          if (i < 2 || tid < SCALE_ROWS - 256) sw_words[g * SCALE_ROWS + i * 128 + tid] = next[i][g];
      scale_sync();
      const int groups = (min(KB - kb, SCALE_BATCH) + WORD_KB - 1) / WORD_KB;
      kb += SCALE_BATCH;
      if (kb >= KB) { kb = 0; t += G; }
      if (t < pl.tiles) load(t, kb);
      for (int g = 0; g < groups; ++g) {
        uint32_t v[12];
#pragma unroll
        for (int i = 0; i < 11; ++i) v[i] = sw_words[g * SCALE_ROWS + 32 * i + lane];
        v[11] = 0x7f7f7f7fu;
        if (ok) ok = mbar_wait(sempty0 + 8 * sc, sc_phase ^ 1, abort_flag);
        // (after a failed wait the warp goes on to the barriers, without work)
        ok = __all_sync(0xffffffffu, ok);
        if (ok) {
          tc_fence_after();
          const uint32_t ta = tmem + uint32_t(SCALE_COL + sc * SCALE_STEP) + part;
          tmem_st4(ta, v[0], v[1], v[2], v[3]);
          tmem_st8(ta + 4, v + 4);
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
    }
  } else if (warp >= EPI_WARP) {
    // ------------------------------------------------------------ epilogue
    pdl_wait();
    const int sp = warp & 3, half = (warp - EPI_WARP) >> 2;
    const uint32_t tempty_r0 = PAIR ? mapa_shared(tempty0, 0) : tempty0;
    int acc = 0;
    uint32_t acc_phase = 0;
    for (int t = pos; t < pl.tiles; t += G) {
      const int m = pl.m(t) * CTAS + int(rank), nn = pl.n(t);
      if (!mbar_sleep_warp(tfull0 + 8 * acc, acc_phase, abort_flag)) { ok = false; break; }
      tc_fence_after();
      const uint32_t tb = tmem + uint32_t(acc * MAX_BN) + (uint32_t(sp * 32) << 16);
#pragma unroll 1
      for (int ch = half; ch < BN / 32; ch += 2) {
        float v[32];
        tmem_ld32(tb + uint32_t(ch * 32), v);
        const int r0 = m * BM + sp * 32, c0 = nn * BN + ch * 32;
        if (r0 < out.rows && c0 < out.n)
          write_chunk(out, stg + (warp - EPI_WARP) * STAGING_WARP, lane, v, r0, c0);
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) {
        if (PAIR) mbar_arrive_cluster(tempty_r0 + 8 * acc);
        else mbar_arrive(tempty0 + 8 * acc);
      }
      if (++acc == 2) { acc = 0; acc_phase ^= 1; }
    }
  }
  if (!ok) {
    *abort_flag = 1;
    atomicOr(out.err, DEVERR_TIMEOUT);
  }
  tc_fence_before();
  __syncthreads();
  // no CTA leaves while its peer may still load, commit or arrive into it
  if (PAIR) cluster_sync();
  if (warp == 1) {
    __syncwarp();
    tc_fence_after();
    if (PAIR) tmem_dealloc_pair(tmem, TMEM_COLS);
    else tmem_dealloc(tmem, TMEM_COLS);
  }
}

constexpr int SMS = 152;

template <class T, bool PAIR>
cudaError_t go(const Fp8Mat& x, const Fp8Mat& w, const Out<T>& o, int bn, cudaStream_t st) {
  // (an attribute of the current device, so set for each call)
  RC_TRY(cudaFuncSetAttribute(fp8_linear_kernel<T, PAIR>,
                              cudaFuncAttributeMaxDynamicSharedMemorySize, int(SMEM_BYTES)));
  Plan pl;
  pl.bn = bn;
  const int fit = RING_BYTES / stage_bytes<PAIR>(bn);
  pl.stages = fit < MAX_STAGES ? fit : MAX_STAGES;
  const int rows = BM * (PAIR ? 2 : 1);
  pl.mt = int((x.rows + (long long)rows - 1) / rows);
  pl.nt = int((w.rows + (long long)bn - 1) / bn);
  pl.kb = (x.cols + BK - 1) / BK;
  pl.n_first = w.rows < x.rows;
  const long long tiles = (long long)pl.mt * pl.nt;
  if (tiles > 0x7fffffff - SMS) return cudaErrorInvalidValue;
  pl.tiles = int(tiles);
  CUtensorMap mx, mw;
  RC_TRY(tma_map_bytes(x.codes, x.rows, x.cols, x.ld, BM, &mx));
  RC_TRY(tma_map_bytes(w.codes, w.rows, w.cols, w.ld, PAIR ? bn / 2 : bn, &mw));
  count_launches(1);
  const int slots = PAIR ? SMS / 2 : SMS, used = pl.tiles < slots ? pl.tiles : slots;
  if (PAIR)
    return launch_k_cluster(fp8_linear_kernel<T, true>, dim3(unsigned(2 * used)), dim3(THREADS),
                            SMEM_BYTES, 2, st, mx, mw, x, w, o, pl);
  return launch_k(fp8_linear_kernel<T, false>, dim3(unsigned(used)), dim3(THREADS), SMEM_BYTES, st,
                  mx, mw, x, w, o, pl);
}

template <class T>
cudaError_t linear(const Fp8Mat& x, const Fp8Mat& w, const float* b, T* y, int ldy, unsigned* err,
                   cudaStream_t st) {
  const uintptr_t row = x.rows > 1 ? uintptr_t(ldy) * sizeof(T) : 0;
  const Out<T> o{y, b, ldy, x.rows, w.rows,
                 ((reinterpret_cast<uintptr_t>(y) | row) & 15u) == 0, err};
  const long long mt = (x.rows + BM - 1LL) / BM;
  const auto tiles = [&](int bn) { return mt * ((w.rows + bn - 1LL) / bn); };
  if (x.rows > BM && tiles(192) >= SMS) return go<T, true>(x, w, o, 192, st);
  if (tiles(128) >= SMS) return go<T, false>(x, w, o, 128, st);
  return go<T, false>(x, w, o, 64, st);
}

}  // namespace

cudaError_t launch_fp8_linear(const Fp8Mat& x, const Fp8Mat& w, const float* b, void* y, int ldy,
                              bool f32, unsigned* err, cudaStream_t st) {
  if (f32) return linear(x, w, b, static_cast<float*>(y), ldy, err, st);
  return linear(x, w, b, static_cast<bf16*>(y), ldy, err, st);
}

}  // namespace rc
