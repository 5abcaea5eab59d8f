// Products of each expert's rows with its quantised matrix (rc_experts_linear):
// y[p] = act(x[source[p]] W_e^T + b_e), on the block-scaled e4m3 MMA of the
// tensor core, with the work shared out on the device (only it knows how many rows
// each expert has).
//
// Persistent CTAs of 28 warps, as in rc_fp8_linear: warps 0, 3 and 24..27 bring the
// rows of x, warp 2 W, warp 1 issues the MMAs, warps 4..7 put the scale bytes into
// tensor memory, warps 8..23 drain the accumulator.  Rows are gathered by TMA, four an
// instruction, of which a warp issues one in 60 to 130 cycles: 16384 x 2 rows, 1152 x
// 4608, GELU, took 508 us with one warp, 290 with two; now 186 (neighbouring rows, in
// one box, without the activation: 144).  What bounds it more than the tensor core (90
// us; its pipe is busy 40 % of the time) are the gathers, 110 cycles each where the epilogue
// takes the issue slots (59 % of all) beside them, 60 alone; the roles' code has to stay in
// the SM's instruction cache (at 96 KB it did not: 180 us for neighbouring rows), and
// nothing may be spilled (registers for 28 warps: 72).
// Each CTA first lists the experts that have rows, with the tiles of BM rows before
// each; a tile's number names its rows by a search there, and its columns.  Rows of
// an accumulator do not mix, so what a tile holds beyond its expert's rows (stale
// shared memory, the next expert's rows) is only never written.
#include "../../include/regioncache.h"
#include "block.h"
#include "common.cuh"
#include "experts_act.cuh"
#include "fp8.cuh"
#include "tc_eight_bit.cuh"
#include "tma_host.h"

namespace rc {

namespace {

using namespace rc::tc;

constexpr int BM = 128, BK = 128;
constexpr int SCALE_WARP = 4, EPI_WARP = 8, EPI_WARPS = 16, MORE_X_WARP = 24;
constexpr int X_WARPS = 6, THREADS = 32 * (MORE_X_WARP + X_WARPS - 2);
constexpr int STAGE_A = BM * BK;
constexpr int RING_BYTES = 168 * 1024, MAX_STAGES = 6;
// tensor memory: accumulators at 0 and ACC_BN (one, where a tile is wider), then a
// ring of scale words: a batch holds, for each WORD_KB blocks, 4 columns for x and
// 8 for W
constexpr int ACC_BN = 192, MAX_BN = 256, SCALE_COL = 2 * ACC_BN, TMEM_COLS = 512;
constexpr int WORD_KB = 4, SCALE_BATCH = 16, SCALE_GROUPS = SCALE_BATCH / WORD_KB;
constexpr int SCALE_STEP = 12, SCALE_SLOT = SCALE_GROUPS * SCALE_STEP, SCALES = 2;
static_assert(SCALE_COL + SCALES * SCALE_SLOT <= TMEM_COLS && MAX_BN + 128 <= SCALE_COL,
              "tensor memory");
// the batch's words in shared memory: 128 rows of x, four shared rows of W
constexpr int SCALE_ROWS = 128 + 4, SCALE_BYTES = SCALE_GROUPS * SCALE_ROWS * 4;
// the experts that have rows: tiles before, first row, end, number
constexpr int MAX_E = RC_EXPERTS_MAX;
struct Tables {
  int first[MAX_E], row[MAX_E], end[MAX_E];
  uint16_t expert[MAX_E];
  unsigned long long parts[THREADS / 32];
};
constexpr int LIST = 256;  // tiles of a CTA that are looked up once
constexpr int CHUNKS = MAX_BN / 128;  // of an epilogue warp, at most
constexpr int BIAS_BYTES = EPI_WARPS * CHUNKS * 32 * 4;
constexpr int MOST_FOURS = 16, FOURS = X_WARPS * MOST_FOURS;  // of rows of x, of a warp
constexpr int STAGING = 32 * 64;  // of an epilogue warp: 32 rows of 64 bytes
constexpr size_t SMEM_BYTES = size_t(RING_BYTES) + EPI_WARPS * STAGING + SCALE_BYTES +
                              LIST * 16 + BIAS_BYTES + FOURS * 16 +
                              sizeof(Tables) + 1024 + 192;
static_assert(SMEM_BYTES <= 227 * 1024, "shared memory");
static_assert(MAX_BN * 129 * 4 <= RING_BYTES, "a split tile's part");

struct Plan {
  int bn, stages, groups, nt, kb, parts, accs, most;  // most: tiles of TM rows there can be
};
template <bool PAIR>
__host__ __device__ constexpr int stage_bytes(int bn) {
  return STAGE_A + (PAIR ? bn / 2 : bn) * BK;
}

template <ExpertsOut>
struct TypeOf { typedef bf16 T; };
template <>
struct TypeOf<OUT_F32> { typedef float T; };
template <>
struct TypeOf<OUT_CODES> { typedef uint8_t T; };

// Sums with their bias (in shared memory, 16-byte aligned).
template <int N>
__device__ __forceinline__ void add_bias(float* v, const float* bias) {
#pragma unroll
  for (int j = 0; j < N; j += 4) {
    const float4 b = *reinterpret_cast<const float4*>(bias + j);
    const float2 lo = f2_add(make_float2(v[j], v[j + 1]), make_float2(b.x, b.y));
    const float2 hi = f2_add(make_float2(v[j + 2], v[j + 3]), make_float2(b.z, b.w));
    v[j] = lo.x, v[j + 1] = lo.y, v[j + 2] = hi.x, v[j + 3] = hi.y;
  }
}

// A warp's 32 rows of 64 bytes to y by TMA, by way of its shared memory, in the
// layout of a box with a swizzle as wide as its rows (which also keeps the writes free
// of bank conflicts); what lies outside y is not written.  First `put_pieces`, N
// pieces of 16 bytes from piece `k0` on (lane = row, `q` its bytes).
template <int N>
__device__ __forceinline__ void put_pieces(uint8_t* stg, int lane, int k0, const uint32_t* q) {
  const uint32_t s0 = saddr(stg) + lane * 64;
#pragma unroll
  for (int k = 0; k < N; ++k)
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(
                     s0 + 16 * ((k0 + k) ^ ((lane >> 1) & 3))),
                 "r"(q[4 * k]), "r"(q[4 * k + 1]), "r"(q[4 * k + 2]), "r"(q[4 * k + 3])
                 : "memory");
}
// The lane's four, read back.
__device__ __forceinline__ void get_pieces(const uint8_t* stg, int lane, float* q) {
  const uint32_t s0 = saddr(stg) + lane * 64;
#pragma unroll
  for (int k = 0; k < 4; ++k)
    asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];"
                 : "=f"(q[4 * k]), "=f"(q[4 * k + 1]), "=f"(q[4 * k + 2]), "=f"(q[4 * k + 3])
                 : "r"(s0 + 16 * (k ^ ((lane >> 1) & 3)))
                 : "memory");
}
__device__ __forceinline__ void store_box(const CUtensorMap* map, uint8_t* stg, int lane, int r0,
                                          int c0) {
  fence_proxy_async_smem();
  __syncwarp();
  if (lane == 0) tma_store_2d(map, saddr(stg), c0, r0);
}
// The box before has been read.
__device__ __forceinline__ void box_free(int lane) {
  if (lane == 0) tma_store_wait_read<0>();
  __syncwarp();
}
// Sixteen columns (lane = row) of any alignment: the first `rows` rows and `cols`
// columns at y, neighbouring lanes neighbouring columns.
template <class T>
__device__ __forceinline__ void write_columns(T* y, long long ldy, int rows, int cols,
                                              uint8_t* stg, int lane, const float* v) {
  box_free(lane);
  float* s = reinterpret_cast<float*>(stg);
#pragma unroll
  for (int j = 0; j < 16; ++j) s[lane * 16 + (j ^ (lane & 15))] = v[j];
  __syncwarp();
  const int c = lane & 15;
  if (c < cols)
    for (int r = lane >> 4; r < min(32, rows); r += 2)
      y[r * ldy + c] = T(s[r * 16 + (c ^ (r & 15))]);
  __syncwarp();
}

// Barriers of the four scale warps, and of the four epilogue warps of a row.
__device__ __forceinline__ void scale_sync() { asm volatile("bar.sync 1, 128;" ::: "memory"); }
__device__ __forceinline__ void rows_sync(int sp) {
  asm volatile("bar.sync %0, 128;" ::"r"(2 + sp) : "memory");
}

// How CTAs work together, as in rc_fp8_linear.  PAIRS: clusters of two share each
// MMA (M = 256).  SPLIT: a cluster shares a tile's blocks of columns, each CTA
// leaves its part in shared memory, and the parts are added there in order.
enum Mode { ALONE, PAIRS, SPLIT };

template <ExpertsOut OUT, Mode MODE>
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
  uint32_t* words = reinterpret_cast<uint32_t*>(stg + EPI_WARPS * STAGING);
  int4* list = reinterpret_cast<int4*>(words + SCALE_BYTES / 4);
  float* biases = reinterpret_cast<float*>(list + LIST);
  int4* fours = reinterpret_cast<int4*>(biases + BIAS_BYTES / 4);
  Tables& tab = *reinterpret_cast<Tables*>(fours + FOURS);
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
      // (the MMAs, and the stage's warps of x, of which none gets a turn of the ring
      // behind: some have nothing to load for a tile)
      mbar_init(empty0 + 8 * s, 1 + X_WARPS / pl.groups);
    }
    for (int s = 0; s < SCALES; ++s) {
      mbar_init(sfull0 + 8 * s, 4 * CTAS);
      mbar_init(sempty0 + 8 * s, 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(tfull0 + 8 * i, 1);
      // (of a pair, the second's warps are told of by its warp 1: an arrival in
      // another CTA waits for the thread's stores)
      mbar_init(tempty0 + 8 * i, EPI_WARPS + (PAIR && rank == 0 ? 1 : 0));
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
    // (offsets that descend can name rows twice: any sum of tiles fits below)
    constexpr unsigned long long ONE = 1ull << 48, TILES = ONE - 1;
    const auto most = [&](unsigned long long v) {
      return int(min(v & TILES, (unsigned long long)pl.most));
    };
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
      if (hi[j] > lo[j]) mine += ONE + unsigned((hi[j] - lo[j] - 1) / TM + 1);
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
        const int i = int(before >> 48);
        tab.first[i] = most(before);
        tab.row[i] = lo[j], tab.end[i] = hi[j];
        tab.expert[i] = uint16_t(2 * threadIdx.x + j);
        before += ONE + unsigned((hi[j] - lo[j] - 1) / TM + 1);
      }
    entries = int(all >> 48), m_tiles = most(all);
  }
  // this CTA's (or pair's) tiles pos, pos + G ..: expert, first place, places left there
  // and number among the columns.  The first LIST of them are found here, once for all
  // warps.
  const int parts = MODE == SPLIT ? pl.parts : 1;
  const int G = int(gridDim.x) / (CTAS * parts), pos = int(blockIdx.x) / (CTAS * parts);
  struct Tile { int expert, place, left, n; };
  const auto search = [&](int t) {
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
  const int own_tiles = m_tiles * pl.nt > pos ? (m_tiles * pl.nt - pos - 1) / G + 1 : 0;
  __syncthreads();
  if (threadIdx.x < min(LIST, own_tiles)) {
    const Tile t = search(pos + int(threadIdx.x) * G);
    list[threadIdx.x] = make_int4(t.expert, t.place, t.left, t.n);
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  if (PAIR) cluster_sync();  // (the peer's barriers are ready)

  const auto tile_of = [&](int i) {
    if (i >= LIST) return search(pos + i * G);
    const int4 t = list[i];
    return Tile{t.x, t.y, t.z, t.w};
  };

  const int BN = pl.bn, STAGES = pl.stages, ACCS = pl.accs;
  const int STAGE = stage_bytes<PAIR>(BN);
  const bool gated = a.act == RC_ACT_GATED_SILU;
  const int half_bn = BN / 2, cols_out = gated ? half_bn : BN;  // outputs of a tile
  const int e_rows = a.w.rows / a.experts, N = gated ? 2 * a.n : a.n;
  // of each tile, this CTA's blocks k0 .. k0 + KB - 1
  const int part_of = MODE == SPLIT ? int(cluster_ctarank()) : 0;
  const int k0 = part_of * pl.kb / parts, KB = (part_of + 1) * pl.kb / parts - k0;
  bool ok = true;

  // rows of a CTA of this tile (the second of a pair may have none)
  const auto rows_of = [&](const Tile& t, int r) { return max(0, min(BM, t.left - r * BM)); };
  // the row of x of a place as it stands in `source`, and then (row 0 for one outside,
  // which is reported)
  const auto source_of = [&](int place) { return a.source ? a.source[place] : place; };
  const auto row_of = [&](int r) {
    if (r >= 0 && r < a.x.rows) return r;
    atomicOr(a.err, DEVERR_INDEX);
    return 0;
  };
  // many neighbouring rows come as one box
  const auto in_box = [&](int rows) { return !a.source && rows > 32; };

  if (warp < SCALE_WARP || warp >= MORE_X_WARP) {
    if (warp == 0 || warp == 3 || warp >= MORE_X_WARP) {
      // ---------------------------------------------------------------- TMA: x
      // Groups of its warps take the ring's stages in turn (a stage is always the same
      // group's, so that it waits for its own last use), a block's fours of rows dealt
      // to a group's warps; one thread of each issues them (a lane's own operands
      // would be brought to uniform registers lane by lane).  Lane i < MOST looks up
      // the warp's i-th four, a tile ahead (and at their bounds only when they are
      // needed: the wait for them took a quarter of the warp's time).
      const int w = warp == 0 ? 0 : warp == 3 ? 1 : warp - MORE_X_WARP + 2;
      const int groups = pl.groups, of = X_WARPS / groups, group = w / of, wi = w - group * of;
      int4* own = fours + w * MOST_FOURS;
      int stage = group, next = group;  // the warp's next block, from the tile's first
      uint32_t phase = 0;
      int tile = 0;
      Tile tl = {};
      int r[4];
      const auto look_up = [&] {
        tl = tile_of(tile);
        const int rows = rows_of(tl, int(rank)), at = 4 * (wi + of * lane);
#pragma unroll
        for (int j = 0; j < 4; ++j)
          r[j] = lane < MOST_FOURS && at + j < rows
                     ? source_of(tl.place + int(rank) * BM + at + j) : 0;
      };
      if (tile < own_tiles) look_up();
      while (ok && tile < own_tiles) {
        const int rows = rows_of(tl, int(rank)), place = tl.place + int(rank) * BM;
        const bool box = in_box(rows);
        const auto bytes = [&](int n) { return in_box(n) ? STAGE_A : (n + 3) / 4 * 4 * BK; };
        int expect = bytes(rows_of(tl, 0));
        if (PAIR) expect += bytes(rows_of(tl, 1)) + BN * BK;
        if (lane < MOST_FOURS)
          own[lane] = make_int4(row_of(r[0]), row_of(r[1]), row_of(r[2]), row_of(r[3]));
        __syncwarp();
        ++tile;
        if (tile < own_tiles) look_up();
        const int fours_here = box ? 0 : (rows + 3) / 4;  // (of which this warp has every of-th)
#pragma unroll 1
        for (; next < KB; next += groups) {
          ok = mbar_sleep_warp(empty0 + 8 * stage, phase ^ 1, abort_flag);
          if (!ok) break;
          if (elect_one()) {
            const uint32_t st = saddr(smem + stage * STAGE), fb = full0 + 8 * stage;
            const uint32_t bar = PAIR ? mapa_shared(fb, 0) : fb;
            const int c = (k0 + next) * BK;
            // (a barrier may see bytes before it is told of them: its phase still
            // needs that arrival)
            if (rank == 0 && wi == 0) mbar_expect_tx(fb, uint32_t(expect));
            const int4* rows4 = own;
            uint32_t to = st + wi * 4 * BK;
#pragma unroll 4
            for (int i = wi; i < fours_here; i += of, to += of * 4 * BK)
              tma_gather4<PAIR>(to, &tmG, bar, c, *rows4++);
            if (box && wi == 0) {
              if (PAIR) tma_load_2d_pair(st, &tmX, bar, c, place);
              else tma_load_2d(st, &tmX, bar, c, place);
            }
            mbar_arrive(empty0 + 8 * stage);
          }
          __syncwarp();
          stage += groups;
          if (stage >= STAGES) { stage -= STAGES; phase ^= 1; }
        }
        next -= KB;
      }
    } else if (warp == 2) {
      // ---------------------------------------------------------------- TMA: W
      if (elect_one()) {
        int stage = 0;
        uint32_t phase = 0;
        for (int tile = 0; ok && tile < own_tiles; ++tile) {
          const Tile tl = tile_of(tile);
          const int n0 = tl.expert * e_rows + tl.n * cols_out;
          for (int kb = 0; kb < KB; ++kb) {
            if (!mbar_sleep(empty0 + 8 * stage, phase ^ 1, abort_flag)) { ok = false; break; }
            const uint32_t st = saddr(smem + stage * STAGE) + STAGE_A, fb = full0 + 8 * stage;
            const int c = (k0 + kb) * BK;
            if (PAIR) {  // both CTAs' bytes land on rank 0's barrier
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
      if (PAIR && rank == 1 && elect_one()) {
        int acc = 0;
        uint32_t acc_phase = 0;
        for (int tile = 0; ok && tile < own_tiles; ++tile) {
          ok = mbar_sleep(tempty0 + 8 * acc, acc_phase, abort_flag);
          if (!ok) break;
          tc_fence_after();
          tc_fence_before();
          mbar_arrive_cluster(mapa_shared(tempty0 + 8 * acc, 0));
          if (++acc == ACCS) { acc = 0; acc_phase ^= 1; }
        }
      }
      if (rank == 0 && elect_one()) {
        const uint32_t idesc = IDESC_E4M3 | (uint32_t(BN >> 3) << 17) | (uint32_t(CTAS) << 27);
        const uint64_t da = sw128_desc(saddr(smem)), db = sw128_desc(saddr(smem + STAGE_A));
        int stage = 0, acc = 0, sc = 0;
        uint32_t phase = 0, acc_phase = 0, sc_phase = 0;
        uint64_t so = 0;     // the stage's offset in the descriptors' address field
        bool ready = false;  // the current stage was seen full already
        for (int tile = 0; ok && tile < own_tiles; ++tile) {
          if (!mbar_wait(tempty0 + 8 * acc, acc_phase ^ 1, abort_flag)) { ok = false; break; }
          const uint32_t d = tmem + uint32_t(acc * ACC_BN);
          uint32_t accumulate = 0;
          for (int kb = 0; ok && kb < KB;) {
            if (!mbar_wait(sfull0 + 8 * sc, sc_phase, abort_flag)) { ok = false; break; }
            uint32_t sa = tmem + uint32_t(SCALE_COL + sc * SCALE_SLOT);
            const int end = min(kb + SCALE_BATCH, KB);
            // (one copy of this loop: the roles' code together has to stay in the SM's
            // instruction cache)
            for (int byte = 0; kb < end; ++kb) {
              if (!ready && !mbar_wait(full0 + 8 * stage, phase, abort_flag)) { ok = false; break; }
              const uint64_t da_ = da + so, db_ = db + so;
              const uint32_t eb = empty0 + 8 * stage;
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
              if (++byte == WORD_KB) byte = 0, sa += SCALE_STEP;
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
    }
  } else if (warp < EPI_WARP) {
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
    int xrow = 0;
    Tile tl = {};
    int tile = 0;
    const auto fetch = [&](int kb) {
      if (kb == 0) {
        tl = tile_of(tile);
        in = tid < rows_of(tl, int(rank));
        xrow = in ? row_of(source_of(tl.place + int(rank) * BM + tid)) : 0;
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
    int sc = 0, kb = 0;
    uint32_t sc_phase = 0;
    if (tile < own_tiles) fetch(0);
    while (tile < own_tiles) {
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
      if (kb >= KB) kb = 0, ++tile;
      if (tile < own_tiles) fetch(kb);
      if (ok) ok = mbar_sleep(sempty0 + 8 * sc, sc_phase ^ 1, abort_flag);
      // (after a failed wait the warp goes on to the barriers, without work)
      ok = __all_sync(0xffffffffu, ok);
      if (ok) {
        tc_fence_after();
        const uint32_t ta = tmem + uint32_t(SCALE_COL + sc * SCALE_SLOT) + part;
#pragma unroll 1
        for (int g = 0; g < SCALE_GROUPS; ++g) {
          uint32_t v[SCALE_STEP];
#pragma unroll
          for (int i = 0; i < 4; ++i) v[i] = words[g * SCALE_ROWS + 32 * i + lane];
#pragma unroll
          for (int i = 0; i < 8; ++i) v[4 + i] = words[g * SCALE_ROWS + of[i]];
          tmem_st4(ta + g * SCALE_STEP, v);
          tmem_st8(ta + g * SCALE_STEP + 4, v + 4);
        }
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
  } else {
    // ------------------------------------------------------------ epilogue
    // A warp takes 32 rows (a quarter of the tile's) and every fourth chunk of 32
    // outputs, so that with codes four warps hold the 128 columns of a scale.  (With
    // eight warps, two chunks' work under way for each scheduler: 16384 x 2 rows, 1152 x
    // 4608 with GELU, 259 us.)
    const int sp = warp & 3, part = (warp - EPI_WARP) >> 2;
    uint8_t* own = stg + (warp - EPI_WARP) * STAGING;
    float* own_bias = biases + (warp - EPI_WARP) * CHUNKS * 32;
    T* const y = static_cast<T*>(OUT == OUT_CODES ? a.y8.codes : a.y);
    const int ldy = OUT == OUT_CODES ? a.y8.ld : a.ldy;
    // the bias of a lane's columns (of a gated tile, a chunk's and then that of the
    // factors), a tile ahead
    int tile = 0;
    Tile tl = {};
    float bias[CHUNKS];
    const auto fetch = [&] {
      tl = tile_of(tile);
#pragma unroll
      for (int i = 0; i < CHUNKS; ++i) {
        const int ch = gated ? part : part + 4 * i, c = tl.n * cols_out + ch * 32 + lane;
        bias[i] = 0.f;
        if (a.bias && ch * 32 < cols_out && c < a.n)
          bias[i] = __ldg(a.bias + (long long)tl.expert * N + c + (gated && i > 0 ? a.n : 0));
      }
    };
    const bool in_place = OUT == OUT_CODES && ACCS > 1;
    int acc = 0, turn = 0;
    uint32_t acc_phase = 0;
    if (tile < own_tiles) fetch();
    while (tile < own_tiles) {
      const int left = rows_of(tl, int(rank)) - sp * 32;  // the warp's rows, from `r0`
      const int r0 = tl.place + int(rank) * BM + sp * 32, n0 = tl.n * cols_out;
      __syncwarp();
#pragma unroll
      for (int i = 0; i < CHUNKS; ++i) own_bias[i * 32 + lane] = bias[i];
      __syncwarp();
      ++tile;
      if (tile < own_tiles) fetch();
      // the warp's chunks that hold outputs (with codes, all four of a scale's columns)
      int chunks = 0;
#pragma unroll
      for (int i = 0; i < CHUNKS; ++i)
        if (left > 0 && (part + 4 * i) * 32 < cols_out &&
            n0 + (OUT == OUT_CODES ? 4 * i : part + 4 * i) * 32 < a.n)
          chunks = i + 1;
      if (ok) ok = mbar_sleep_warp(tfull0 + 8 * acc, acc_phase, abort_flag);
      // (after a failed wait the warp goes on to the barriers, without work)
      tc_fence_after();
      const uint32_t tb = tmem + uint32_t(acc * ACC_BN) + (uint32_t(sp * 32) << 16);
      const auto release = [&] {  // (what the warp had to read of the accumulator is read)
        tc_fence_before();
        __syncwarp();
        if (lane == 0 && ok) mbar_arrive(tempty0 + 8 * acc);
      };
      // the gated sums of sixteen columns and of their factors
      const auto gate = [&](const float* bias, float* v, float* w) {
        add_bias<16>(v, bias);
        add_bias<16>(w, bias + 32);
        activate<16, false>(v);
#pragma unroll
        for (int j = 0; j < 16; j += 2) {
          const float2 o = f2_mul(make_float2(v[j], v[j + 1]), make_float2(w[j], w[j + 1]));
          v[j] = o.x, v[j + 1] = o.y;
        }
      };
      // sixteen outputs from column `h` of chunk i on (all 32 rows of the warp)
      const auto outputs = [&](int i, int h, float* v) {
        const uint32_t at = tb + uint32_t((part + 4 * i) * 32 + h);
        const bool last = !in_place && h == 16 && i == chunks - 1;
        tmem_ld16(at, v);
        if (OUT != OUT_CODES && gated) {
          add_bias<16>(v, own_bias + h);
          activate<16, false>(v);
#pragma unroll
          for (int k = 0; k < 16; k += 8) {  // (few registers at a time)
            float w[8];
            tmem_ld8(at + uint32_t(half_bn + k), w);
            if (k == 8 && last) release();
            add_bias<8>(w, own_bias + 32 + h + k);
#pragma unroll
            for (int j = 0; j < 8; j += 2) {
              const float2 o = f2_mul(make_float2(v[k + j], v[k + j + 1]),
                                      make_float2(w[j], w[j + 1]));
              v[k + j] = o.x, v[k + j + 1] = o.y;
            }
          }
        } else {
          if (last) release();
          add_bias<16>(v, own_bias + i * 32 + h);
          if (a.act == RC_ACT_GELU) activate<16, true>(v);
          else if (a.act == RC_ACT_SILU) activate<16, false>(v);
        }
      };
      if (MODE == SPLIT) {  // (every MMA is done: the operand ring is free)
        float* to = reinterpret_cast<float*>(smem) + sp * 32 + lane;
        for (int ch = part; ok && left > 0 && ch < BN / 32; ch += 4) {
          float v[32];
          tmem_ld32(tb + uint32_t(ch * 32), v);
          if (lane < left)
#pragma unroll
            for (int j = 0; j < 32; ++j) to[(ch * 32 + j) * 129] = v[j];
        }
      } else if (chunks == 0) {
        release();
      } else {
#pragma unroll 1
        for (int i = 0; i < chunks; ++i) {  // (with codes, the four warps of the rows alike)
          const int c0 = n0 + (part + 4 * i) * 32;
          if constexpr (OUT == OUT_CODES) {
            // the outputs wait in tensor memory until the scale is known: where their
            // sums were, or beside an only accumulator, which is free again the sooner
            const uint32_t at = in_place ? tb + uint32_t((part + 4 * i) * 32)
                                         : tmem + uint32_t(MAX_BN + part * 32) +
                                               (uint32_t(sp * 32) << 16);
            uint32_t top = 0;
            const auto largest = [&](int h, float* v) {  // (outputs behind the last are 0)
#pragma unroll
              for (int j = 0; j < 16; ++j) {
                if (c0 + h + j >= a.n) v[j] = 0.f;
                top = max(top, __float_as_uint(v[j]) & 0x7fffffffu);
              }
            };
            if (gated && ok) {
              // Half of the sums go beside the accumulator as they are, the others into
              // registers: it is free again before anything is computed (4128 x 2 rows of
              // 16 experts, 1152 x 2 x 2304: 62.9 us, with activations first 65.7).
              float v[16], w[16];
              const uint32_t from = tb + uint32_t(part * 32);
              tmem_ld16(from + 16, v);
              tmem_st16(at, reinterpret_cast<const uint32_t*>(v));
              tmem_ld16(from + uint32_t(half_bn) + 16, w);
              tmem_st16(at + 16, reinterpret_cast<const uint32_t*>(w));
#pragma unroll 1
              for (int h = 0; h < 32; h += 16) {
                tmem_ld16(h ? at : from, v);
                tmem_ld16(h ? at + 16 : from + uint32_t(half_bn), w);
                if (h == 0) {
                  release();
                  tmem_wait_st();
                }
                gate(own_bias + h, v, w);
                largest(h, v);
                if (h == 0) put_pieces<4>(own, lane, 0, reinterpret_cast<const uint32_t*>(v));
                else tmem_st16(at + 16, reinterpret_cast<const uint32_t*>(v));
              }
            }
#pragma unroll 1
            for (int h = 0; !gated && ok && h < 32; h += 16) {
              float v[16];
              outputs(i, h, v);
              largest(h, v);
              tmem_st16(at + uint32_t(h), reinterpret_cast<const uint32_t*>(v));
            }
            tmem_wait_st();
            // (behind the ring's stages, which with codes' tiles, of 128 columns or 256, take
            // 144 KB at most)
            static_assert(RING_BYTES - 144 * 1024 >= 2 * EPI_WARPS * 32 * 4, "the largest");
            uint32_t* to =
                reinterpret_cast<uint32_t*>(smem + STAGES * STAGE) + turn * EPI_WARPS * 32 +
                sp * 32 + lane;
            to[part * 128] = top;
            rows_sync(sp);
#pragma unroll
            for (int k = 0; k < 4; ++k) top = max(top, to[k * 128]);
            turn ^= 1;
            if (!ok) continue;
            const int b = scale_byte(top);
            const uint64_t inv = both(scale_inverse(b));
            if (part == 0 && lane < left)
              a.y8.scales[(long long)(c0 / 128) * a.y8.lds + r0 + lane] = uint8_t(b);
            uint8_t* dst = y + (long long)(r0 + lane) * ldy + c0;
#pragma unroll 1
            for (int h = 0; h < 32; h += 16, dst += 16) {
              float v[16];
              if (gated && h == 0) get_pieces(own, lane, v);
              else tmem_ld16(at + uint32_t(h), v);
              if (in_place && h == 16 && i == chunks - 1) release();
              uint32_t q[4];
#pragma unroll
              for (int k = 0; k < 4; ++k)
                q[k] = __byte_perm(e4m3x2(v[4 * k], v[4 * k + 1], inv),
                                   e4m3x2(v[4 * k + 2], v[4 * k + 3], inv), 0x5410);
              if (lane < left && c0 + h + 16 <= a.n) {
                *reinterpret_cast<uint4*>(dst) = make_uint4(q[0], q[1], q[2], q[3]);
              } else if (lane < left) {
#pragma unroll
                for (int j = 0; j < 15; ++j)
                  if (c0 + h + j < a.n) dst[j] = uint8_t(q[j >> 2] >> (8 * (j & 3)));
              }
            }
          } else {
            if (!ok) break;
            const bool box = a.tma && left >= 32;
#pragma unroll 1
            for (int h = 0; h < 32; h += 16) {
              float v[16];
              outputs(i, h, v);
              if (!box) {
                if (c0 + h < a.n)
                  write_columns(y + (long long)r0 * ldy + c0 + h, ldy, left, a.n - c0 - h, own,
                                lane, v);
                continue;
              }
              if (OUT == OUT_F32 || h == 0) box_free(lane);
              if constexpr (OUT == OUT_F32) {
                put_pieces<4>(own, lane, 0, reinterpret_cast<const uint32_t*>(v));
                if (c0 + h < a.n) store_box(&tmY, own, lane, r0, c0 + h);
              } else {
                uint32_t q[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) q[k] = pack_bf16x2(v[2 * k], v[2 * k + 1]);
                put_pieces<2>(own, lane, h / 8, q);
                if (h == 16) store_box(&tmY, own, lane, r0, c0);
              }
            }
          }
        }
      }
      if (++acc == ACCS) { acc = 0; acc_phase ^= 1; }
    }
    if (MODE != SPLIT && lane == 0) tma_store_wait_read<0>();
  }
  if (MODE == SPLIT) {
    cluster_sync();
    const int tile = 0;
    if (tile < own_tiles) {
      // the rows' chunks of 32 outputs (128 with codes), dealt to the cluster's warps
      const Tile tl = tile_of(tile);
      const int rows = rows_of(tl, 0);
      constexpr int LANES = OUT == OUT_CODES ? 4 : 1;  // columns of a lane
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
          if (gated) {
            const float w = sum(half_bn + col, row) + (b ? __ldg(b + a.n) : 0.f);
            v[i] = act_of(RC_ACT_SILU, v[i]) * w;
          } else {
            v[i] = act_of(a.act, v[i]);
          }
        }
        if constexpr (OUT == OUT_CODES) {
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

// y [rows][n] in boxes of 64 bytes x 32 rows, swizzled over their own width.
template <class T>
cudaError_t tma_map_boxes(T* y, int rows, int n, int ld, CUtensorMap* out) {
  auto fn = tma_encode_fn();
  if (!fn) return cudaErrorNotSupported;
  const cuuint64_t dims[2] = {cuuint64_t(n), cuuint64_t(rows)};
  const cuuint64_t strides[1] = {cuuint64_t(ld) * sizeof(T)};
  const cuuint32_t box[2] = {cuuint32_t(64 / sizeof(T)), 32}, es[2] = {1, 1};
  const CUresult r =
      fn(out, sizeof(T) == 4 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16,
         2, y, dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_64B,
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
// Stages of the ring: dealt to groups of x's six warps, of two or three, and so a
// multiple of the groups.
int stages_of(bool pair, int bn) {
  const int fit = RING_BYTES / (pair ? stage_bytes<true>(bn) : stage_bytes<false>(bn));
  return fit >= 6 ? 6 : fit >= 4 ? 4 : 3;
}

template <ExpertsOut OUT, Mode MODE>
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
  pl.stages = stages_of(PAIR, bn);
  pl.groups = pl.stages == 4 ? 2 : 3;
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
  if constexpr (OUT != OUT_CODES) {
    const uintptr_t row = uintptr_t(a.ldy) * sizeof(T);
    a.tma = ((reinterpret_cast<uintptr_t>(a.y) | row) & 15u) == 0;
    if (a.tma) RC_TRY(tma_map_boxes(static_cast<T*>(a.y), a.pairs, a.n, a.ldy, &my));
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
// cycles), for experts with even shares of the places.  A block of columns takes what
// rc_fp8_linear's does, or a stage's way round by the number of stages: 1000 of
// latencies, the MMAs, and 900 for 128 gathered rows (alone at 256 columns, three
// stages, the gated 4128 x 2 rows of 16 experts to codes took 67 us).
Choice choose(const ExpertsArgs& a, bool codes) {
  const bool gated = a.act == RC_ACT_GATED_SILU;
  const int kb = (a.x.cols - 1) / BK + 1;
  const long long used = a.pairs < a.experts ? a.pairs : a.experts;
  const double rows = double(a.pairs) / double(used);  // of an expert
  // (uneven shares: half a tile more for each expert)
  const auto m_tiles = [&](int high) {
    return rows <= high / 2 ? double(used) : a.pairs / double(high) + 0.5 * used;
  };
  Choice best{ALONE, gated ? 256 : 128, 1};
  double least = 1e30;
  const auto look = [&](Mode mode, int bn, int parts) {
    const long long nt = (a.n - 1) / (gated ? bn / 2 : bn) + 1;
    const double tiles = m_tiles(mode == PAIRS ? 2 * BM : BM) * nt;
    const double x = rows < BM ? rows / BM : 1;  // of a full tile's rows
    const double round = 1000 + 2.0 * bn + (a.source ? 900 * x : 100);
    double block = mode == PAIRS ? 405 + 0.42 * bn : 60 + 160 * x + 1.83 * bn;
    if (block < round / stages_of(mode == PAIRS, bn)) block = round / stages_of(mode == PAIRS, bn);
    double cost;
    if (mode == SPLIT) {
      if (most_tiles(a, BM) * nt * parts > SMS - 8) return;
      cost = (kb + parts - 1) / parts * block + 4.0 * bn + 600 + 800 * parts;
    } else {
      const double slots = mode == PAIRS ? SMS / 2 : SMS;
      const double waves = tiles <= slots ? 1 : ceil(tiles / slots - 0.05);
      cost = waves * kb * block + (mode == PAIRS ? 9.5 : 7.0) * bn;
      if (bn > ACC_BN) cost += (waves - 1) * 6.0 * bn;  // (the only accumulator is drained)
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

template <ExpertsOut OUT>
cudaError_t linear(const ExpertsArgs& a, cudaStream_t st) {
  const Choice c = choose(a, OUT == OUT_CODES);
  if (c.mode == PAIRS) return go<OUT, PAIRS>(a, c, st);
  if (c.mode == SPLIT) return go<OUT, SPLIT>(a, c, st);
  return go<OUT, ALONE>(a, c, st);
}

}  // namespace

cudaError_t launch_experts_linear(const ExpertsArgs& a, cudaStream_t st) {
  if (experts_few(a)) return launch_experts_few(a, st);
  if (a.y8.codes) return linear<OUT_CODES>(a, st);
  return a.f32 ? linear<OUT_F32>(a, st) : linear<OUT_BF16>(a, st);
}

}  // namespace rc
