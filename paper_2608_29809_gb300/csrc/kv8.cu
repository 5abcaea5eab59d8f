// Paged eight-bit cache (rc_kv8): block tables and slot maps, and the store.
#include "common.cuh"
#include "eight_bit.h"
#include "fp8.cuh"

namespace rc {

namespace {

constexpr int SMS = 152;

// ------------------------------------------------------- tables and slots
// One launch: every CTA sums the requests' rows and new blocks itself (at most
// KV8_MAX_REQUESTS of them, four a thread) and then writes its own part of the
// slot map, four slots a thread.  The rows of a new block include the block's
// first token, so the thread that maps that row also writes the block's table
// entry, and no CTA reads what another one writes.  700 fills, 1.4 million slots:
// 7.6 us (one slot a thread and request sums in every CTA: 17).
constexpr int TAB_THREADS = 1024;
constexpr int TAB_PER = KV8_MAX_REQUESTS / TAB_THREADS;  // requests of a thread
constexpr int TAB_SLOTS = 4;                             // slots of a thread at a time

struct Request {
  int len, cnt, held, fresh;  // tokens, rows, blocks before, new blocks
};
__device__ __forceinline__ int blocks_of(int tokens) {
  return (int)((unsigned(tokens) + KV8_BLOCK - 1) / KV8_BLOCK);
}
__device__ __forceinline__ Request request(const Kv8TablesArgs& a, int r, bool report) {
  Request q{0, 0, 0, 0};
  if (r >= a.n) return q;
  const int len = a.lengths[r], cnt = a.counts ? a.counts[r] : len;
  if (len < 0 || cnt < 0 || cnt > len || len > (long long)a.ld_table * KV8_BLOCK) {
    if (report) atomicOr(a.err, DEVERR_COUNT);
    return q;
  }
  q.len = len;
  q.cnt = cnt;
  q.held = blocks_of(a.positions ? len : len - cnt);
  q.fresh = blocks_of(len) - q.held;
  return q;
}

__global__ void __launch_bounds__(TAB_THREADS)
tables_kernel(const __grid_constant__ Kv8TablesArgs a, int rows_per_cta) {
  pdl_wait();
  pdl_trigger();
  // a request's first row (and behind the last one's), first free block, tokens
  extern __shared__ int s_tab[];
  const int n = a.n;
  int *s_row = s_tab, *s_free = s_row + n + 1, *s_len = s_free + n;
  __shared__ unsigned long long s_warp[32];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const bool first = blockIdx.x == 0;
  // rows in the high and blocks in the low half of one 64-bit sum, neither past
  // 2^31 - 1 (more than any call may have, so that a sum behind it is reported)
  const auto plus = [](unsigned long long u, unsigned long long v) {
    const unsigned lo = min(unsigned(u) + unsigned(v), 0x7fffffffu);
    const unsigned hi = min(unsigned(u >> 32) + unsigned(v >> 32), 0x7fffffffu);
    return (unsigned long long)hi << 32 | lo;
  };
  unsigned long long mine[TAB_PER], sum = 0;
  const int per = (n + TAB_THREADS - 1) / TAB_THREADS;
#pragma unroll
  for (int i = 0; i < TAB_PER; ++i) {
    const int r = tid * per + i;
    const Request q = i < per ? request(a, r, first) : Request{0, 0, 0, 0};
    mine[i] = (unsigned long long)(unsigned)q.cnt << 32 | unsigned(q.fresh);
    sum = plus(sum, mine[i]);
    if (i < per && r < n) s_len[r] = q.len;
  }
  unsigned long long incl = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const unsigned long long v = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl = plus(incl, v);
  }
  if (lane == 31) s_warp[warp] = incl;
  __syncthreads();
  unsigned long long before = lane < warp ? s_warp[lane] : 0;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) before = plus(before, __shfl_xor_sync(0xffffffffu, before, o));
  const unsigned long long others = __shfl_up_sync(0xffffffffu, incl, 1);
  unsigned long long at = lane > 0 ? plus(before, others) : before;
#pragma unroll
  for (int i = 0; i < TAB_PER; ++i) {
    const int r = tid * per + i;
    if (i < per && r < n) {
      s_row[r] = int(at >> 32);
      s_free[r] = int(at & 0xffffffffull);
      if (first) a.offsets[r] = s_row[r];
    }
    at = plus(at, mine[i]);
  }
  if (tid == TAB_THREADS - 1) {
    const int total = int(at >> 32), taken = int(at & 0xffffffffull);
    s_row[n] = total;
    if (first) {
      a.offsets[n] = total;
      *a.used = taken;
      if (total > a.n_slots || taken > a.n_free) atomicOr(a.err, DEVERR_COUNT);
    }
  }
  __syncthreads();
  const int total = min(s_row[n], a.n_slots);
  const long long i0 = (long long)blockIdx.x * rows_per_cta;
  const int i1 = int(min(i0 + rows_per_cta, (long long)a.n_slots));
  for (long long b = i0 + tid * TAB_SLOTS; b < i1; b += TAB_THREADS * TAB_SLOTS) {
    const int base = int(b);
    int slot[TAB_SLOTS], r = 0;
    if (base < total) {
      int hi = n;  // the last request with s_row[r] <= base
      while (hi - r > 1) {
        const int mid = (r + hi) >> 1;
        if (s_row[mid] <= base) r = mid;
        else hi = mid;
      }
    }
    int blk = -1, page = -1, in = -1;  // of the row before
#pragma unroll
    for (int k = 0; k < TAB_SLOTS; ++k) {
      const int i = base + k;
      slot[k] = -1;
      if (i >= total || i >= i1) continue;
      while (s_row[r + 1] <= i) ++r;  // (requests without rows are passed over)
      const int len = s_len[r], cnt = s_row[r + 1] - s_row[r];
      const int p = a.positions ? a.positions[i] : len - cnt + (i - s_row[r]);
      if (p < 0 || p >= len) {
        atomicOr(a.err, DEVERR_INDEX);
        continue;
      }
      if (p / KV8_BLOCK != blk || r != in) {
        blk = p / KV8_BLOCK;
        in = r;
        int* entry = a.table + (long long)r * a.ld_table + blk;
        const int held = blocks_of(a.positions ? len : len - cnt);
        if (blk < held) {
          page = *entry;
        } else {
          const unsigned f = unsigned(s_free[r]) + unsigned(blk - held);  // (below 2^32)
          page = f >= unsigned(a.n_free) ? -1 : a.free_blocks ? a.free_blocks[f] : int(f);
          if (p % KV8_BLOCK == 0) *entry = page;
        }
      }
      // (a block that no pool has would give another one's slot)
      if (page < 0 || page > 0x7fffffff / KV8_BLOCK) atomicOr(a.err, DEVERR_INDEX);
      else slot[k] = page * KV8_BLOCK + p % KV8_BLOCK;
    }
    if (base + TAB_SLOTS <= i1 && (reinterpret_cast<uintptr_t>(a.slots + base) & 15) == 0) {
      *reinterpret_cast<int4*>(a.slots + base) = make_int4(slot[0], slot[1], slot[2], slot[3]);
    } else {
#pragma unroll
      for (int k = 0; k < TAB_SLOTS; ++k)
        if (base + k < i1) a.slots[base + k] = slot[k];
    }
  }
}

// ------------------------------------------------------------------ store
// A run is the rows of one block, next to one another in the list but for
// skipped rows, within 64 rows of it.  A warp takes, for one head of the keys or
// of the values, the runs that start among its `chunk` rows: a row is PIECES lanes
// of eight channels, so the warp reads a run once, keeps it in registers while the
// largest magnitude is found, and writes it as codes; nothing is shared between
// warps, so no two of them may have rows of one block.  (A run that does not fit
// the registers is read again, from L2.)  With CTAs of four
// heads that met at barriers, 4 x 831 rows of 16 heads of 72 took 23.9 us, now
// 9.5 (latency: a run's rows, their largest magnitude, its codes); eight fills of
// 4096 tokens, 226 MB, 36.8 (6.1 TB/s).  Six CTAs an SM leave a thread 80 registers
// and nothing is spilled (the compiler's own choice of 64 to 80 spilled up to 24
// bytes: heads of 64 8.4 us, with 80 7.7; five CTAs: the fills 41.1).
constexpr int ST_WARPS = 4, ST_CHUNK = 24, ST_CTAS = 6;

template <class T, int DH, bool WIDE>
__global__ void __launch_bounds__(32 * ST_WARPS, ST_CTAS)
store_kernel(const __grid_constant__ Kv8Pool pool, const T* __restrict__ kx,
             const T* __restrict__ vx, int ldx, const int* __restrict__ slots, int n_bound,
             const int* __restrict__ count, int append, int chunk, unsigned* __restrict__ err) {
  constexpr int PIECES = DH / 8, AT_ONCE = 32 / PIECES;  // lanes of a row, rows of the warp
  constexpr int KEEP = sizeof(T) == 2 ? 8 : 4;           // passes held in registers
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31, unit = blockIdx.y * ST_WARPS + (threadIdx.x >> 5);
  const int head = unit >> 1, side = unit & 1;
  if (head >= pool.heads) return;
  const bool speaks = unit == 0;  // reports what every unit sees
  const int n = live_count(count, n_bound, speaks && lane == 0 ? err : nullptr);
  const int c0 = blockIdx.x * chunk;
  if (c0 >= n) return;
  // slots of the rows from the one before the chunk, 32 apart; -1 for none
  const long long beyond = (long long)pool.blocks * KV8_BLOCK;
  const auto slot_at = [&](long long r) {
    const int s = r >= 0 && r < n ? slots[r] : -1;
    return s >= beyond ? -2 : max(s, -1);
  };
  int slot[3];
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    const long long r = (long long)c0 - 1 + 32 * i + lane;
    slot[i] = slot_at(r);
    if (slot[i] == -2 && speaks && r >= c0 && r < c0 + chunk) atomicOr(err, DEVERR_INDEX);
  }
  // A run begins at a row (below 32 here) whose block is not that of the last row
  // with a slot, or that has none among the 63 before it.
  unsigned todo = __ballot_sync(0xffffffffu, slot[0] >= 0);
  {
    const unsigned below = todo & ((1u << lane) - 1);
    int prev = __shfl_sync(0xffffffffu, slot[0], below ? 31 - __clz(below) : 0);
    if (!(todo & 1) && c0 > 1 && (todo & ((2u << chunk) - 2u))) {
      // (the row before the chunk is skipped: those before it)
      const long long r = (long long)c0 - 2 - lane;  // lane + 1 rows before the one of lane 0
      const int s0 = slot_at(r), s1 = slot_at(r - 32);
      const unsigned some0 = __ballot_sync(0xffffffffu, s0 >= 0);
      const unsigned some1 = __ballot_sync(0xffffffffu, s1 >= 0);
      const int at = some0 ? __ffs(some0) - 1 : some1 ? __ffs(some1) - 1 : 0;
      const int far = __shfl_sync(0xffffffffu, some0 ? s0 : s1, at);
      const int rows = at + 1 + (some0 ? 0 : 32) + lane;  // from there to this one
      if (!below) prev = rows < KV8_BLOCK ? far : -1;
    } else if (!below) {
      prev = -1;
    }
    todo = __ballot_sync(0xffffffffu,
                         slot[0] >= 0 && (prev < 0 || slot[0] / KV8_BLOCK != prev / KV8_BLOCK)) &
           ((2u << chunk) - 2u);
  }
  const auto slot_of = [&](int i) {  // (i < 96, the same or not in each lane)
    const int a = __shfl_sync(0xffffffffu, slot[0], i & 31);
    const int b = __shfl_sync(0xffffffffu, slot[1], i & 31);
    const int c = __shfl_sync(0xffffffffu, slot[2], i & 31);
    return i < 32 ? a : i < 64 ? b : c;
  };
  const int sub = lane / PIECES, piece = lane - sub * PIECES;
  const bool on = sub < AT_ONCE;
  const T* src = (side ? vx : kx) + head * DH + piece * 8;

  while (todo) {
    const int start = __ffs(todo) - 1;
    todo &= todo - 1;
    const int block = __shfl_sync(0xffffffffu, slot[0], start) / KV8_BLOCK;
    // the run's rows among the 64 from here on: those with a slot, ahead of another
    // block's first
    const int s0 = slot_of(start + lane), s1 = slot_of(start + 32 + lane);
    unsigned rows_in[2];
    {
      const unsigned stop0 = __ballot_sync(0xffffffffu, s0 >= 0 && s0 / KV8_BLOCK != block);
      const unsigned stop1 = __ballot_sync(0xffffffffu, s1 >= 0 && s1 / KV8_BLOCK != block);
      rows_in[0] = __ballot_sync(0xffffffffu, s0 >= 0) & (stop0 ? (stop0 & -stop0) - 1 : ~0u);
      rows_in[1] = __ballot_sync(0xffffffffu, s1 >= 0) &
                   (stop0 ? 0u : stop1 ? (stop1 & -stop1) - 1 : ~0u);
      // more rows than places, or a place twice: the first row of a place counts
      if (!stop0 && !stop1) {
        const int next = slot_of(start + KV8_BLOCK);
        if (speaks && lane == 0 && next >= 0 && next / KV8_BLOCK == block)
          atomicOr(err, DEVERR_INDEX);
      }
    }
    const int len = rows_in[1] ? 64 - __clz(rows_in[1]) : 32 - __clz(rows_in[0]);
    const auto takes = [&](int k) {  // row k of the run's 64 (k < 64)
      return ((k < 32 ? rows_in[0] : rows_in[1]) >> (k & 31) & 1) != 0;
    };
    const int off0 = s0 & (KV8_BLOCK - 1), off1 = s1 & (KV8_BLOCK - 1);
    const bool in0 = takes(lane), in1 = takes(lane + 32);
    unsigned fill[2];  // places filled
    fill[0] = __reduce_or_sync(0xffffffffu, (in0 && off0 < 32 ? 1u << off0 : 0u) |
                                                (in1 && off1 < 32 ? 1u << off1 : 0u));
    fill[1] = __reduce_or_sync(0xffffffffu, (in0 && off0 >= 32 ? 1u << (off0 - 32) : 0u) |
                                                (in1 && off1 >= 32 ? 1u << (off1 - 32) : 0u));
    const bool twice =
        __popc(fill[0]) + __popc(fill[1]) != __popc(rows_in[0]) + __popc(rows_in[1]);
    if (twice && speaks && lane == 0) atomicOr(err, DEVERR_INDEX);
    const bool odd = twice || __popc(rows_in[0]) + __popc(rows_in[1]) != len;
    const bool fresh = append && (fill[0] & 1);
    const auto place = [&](int k) {  // of such a row (every lane takes part)
      const int a = __shfl_sync(0xffffffffu, off0, k & 31);
      const int b = __shfl_sync(0xffffffffu, off1, k & 31);
      return k < 32 ? a : b;
    };
    const auto counts = [&](int k) {  // (k < len) it has a slot, and is the first of its place
      bool first = takes(k);
      if (twice) {
        const int s = place(k);
        for (int j = 0; j < len; ++j) {
          const bool same = place(j) == s;
          first &= !(same && takes(j) && j < k);
        }
      }
      return first;
    };
    uint8_t* sc = pool.scale[side] + (long long)block * pool.heads + head;
    const int old = fresh ? 0 : *sc;

    Eight<T> v[KEEP];
    unsigned top = 0;
    const int passes = (len + AT_ONCE - 1) / AT_ONCE;
    const T* rows = src + ((long long)c0 + start - 1 + sub) * ldx;
    const auto fetch_from = [&](int p0) {
      const T* p = rows + (long long)p0 * AT_ONCE * ldx;
#pragma unroll
      for (int i = 0; i < KEEP; ++i, p += (long long)AT_ONCE * ldx) {
        const int k = (p0 + i) * AT_ONCE + sub;
        if (on && k < len) {
          if (WIDE) v[i].load(p);
          else v[i].load_some(p, 8);
        } else {
          v[i].zero();
        }
        if (odd && !counts(min(k, len - 1))) v[i].zero();
      }
    };
    for (int p0 = 0; p0 < passes; p0 += KEEP) {
      fetch_from(p0);
#pragma unroll
      for (int p = 0; p < KEEP; ++p) top = max(top, v[p].top());
    }
    const int b = max(old, scale_byte(__reduce_max_sync(0xffffffffu, top)));
    const float inv = scale_inverse(b);
    uint8_t* base =
        pool.code[side] + ((long long)block * pool.heads + head) * (KV8_BLOCK * DH) + piece * 8;
    for (int p0 = 0; p0 < passes; p0 += KEEP) {
      if (passes > KEEP) fetch_from(p0);
#pragma unroll
      for (int p = 0; p < KEEP; ++p) {
        if (p0 + p >= passes) break;
        const int k = (p0 + p) * AT_ONCE + sub;
        const int off = place(k & 63);
        const bool stays = !odd || counts(min(k, len - 1));
        if (on && k < len && stays) *reinterpret_cast<uint2*>(base + off * DH) = v[p].codes(inv);
      }
    }
    if (b > old && !fresh && on) {
      // the other tokens' codes move to the raised scale (2^(old - b); below
      // 2^-126 every code becomes zero)
      const float f =
          b == 255 ? scale_value(255) : __uint_as_float(uint32_t(max(127 + old - b, 1)) << 23);
      for (int off = sub; off < KV8_BLOCK; off += AT_ONCE) {
        if ((off < 32 ? fill[0] : fill[1]) >> (off & 31) & 1) continue;
        uint2* p = reinterpret_cast<uint2*>(base + off * DH);
        uint2 q = *p;
        uint32_t* w = reinterpret_cast<uint32_t*>(&q);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const float2 lo = e4m3x2_f32(w[i] & 0xffffu), hi = e4m3x2_f32(w[i] >> 16);
          w[i] = e4m3x2(lo.x * f, lo.y * f) | e4m3x2(hi.x * f, hi.y * f) << 16;
        }
        *p = q;
      }
    }
    if (lane == 0 && (b != old || fresh)) *sc = uint8_t(b);
    __syncwarp();
  }
}

template <class T, int DH>
cudaError_t store(const Kv8Pool& pool, const T* k, const T* v, int ld, bool wide, const int* slots,
                  int n, const int* count, bool append, unsigned* err, cudaStream_t st) {
  // rows of a warp: a decode step's rows are a run each, and want a warp each;
  // past 20 warps an SM a run's rows share one
  const long long units = 2LL * pool.heads, c = (long long)n * units / (SMS * 20);
  const int chunk = c < 1 ? 1 : c > ST_CHUNK ? ST_CHUNK : int(c);
  const dim3 grid(unsigned((n + (long long)chunk - 1) / chunk),
                  unsigned((units + ST_WARPS - 1) / ST_WARPS));
  count_launches(1);
  if (wide)
    return launch_k(store_kernel<T, DH, true>, grid, dim3(32 * ST_WARPS), 0, st, pool, k, v, ld,
                    slots, n, count, append ? 1 : 0, chunk, err);
  return launch_k(store_kernel<T, DH, false>, grid, dim3(32 * ST_WARPS), 0, st, pool, k, v, ld,
                  slots, n, count, append ? 1 : 0, chunk, err);
}

}  // namespace

cudaError_t launch_kv8_tables(const Kv8TablesArgs& a, cudaStream_t st) {
  // at most two CTAs an SM: each sums the requests itself
  constexpr int LEAST = TAB_THREADS * TAB_SLOTS;
  long long per = ((long long)a.n_slots + 2 * SMS - 1) / (2 * SMS);
  per = per < LEAST ? LEAST : (per + TAB_SLOTS - 1) / TAB_SLOTS * TAB_SLOTS;
  const long long ctas = ((long long)a.n_slots + per - 1) / per;
  const size_t smem = size_t(3 * a.n + 1) * sizeof(int);
  // (beside the static part.  The attribute is the device's, not the call's: always
  // the most that any call takes, so that none lowers it under another thread's launch)
  constexpr int MOST = (3 * KV8_MAX_REQUESTS + 1) * int(sizeof(int));
  if (smem > 40 * 1024)
    RC_TRY(cudaFuncSetAttribute(tables_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, MOST));
  count_launches(1);
  return launch_k(tables_kernel, dim3(unsigned(ctas < 1 ? 1 : ctas)), dim3(TAB_THREADS), smem, st,
                  a, int(per));
}

cudaError_t launch_kv8_store(const Kv8Pool& pool, const void* k, const void* v, int ld, bool f32,
                             const int* slots, int n, const int* count, bool append,
                             unsigned* err, cudaStream_t st) {
  const uintptr_t bits = reinterpret_cast<uintptr_t>(k) | reinterpret_cast<uintptr_t>(v) |
                         (n > 1 ? uintptr_t(ld) * (f32 ? 4 : 2) : 0);
  const bool wide = (bits & 15u) == 0;
  const auto go = [&](auto* kk, auto* vv) {
    switch (pool.dh) {
      case 64: return store<std::remove_const_t<std::remove_pointer_t<decltype(kk)>>, 64>(
          pool, kk, vv, ld, wide, slots, n, count, append, err, st);
      case 72: return store<std::remove_const_t<std::remove_pointer_t<decltype(kk)>>, 72>(
          pool, kk, vv, ld, wide, slots, n, count, append, err, st);
      default: return store<std::remove_const_t<std::remove_pointer_t<decltype(kk)>>, 128>(
          pool, kk, vv, ld, wide, slots, n, count, append, err, st);
    }
  };
  if (f32) return go(static_cast<const float*>(k), static_cast<const float*>(v));
  return go(static_cast<const bf16*>(k), static_cast<const bf16*>(v));
}

}  // namespace rc
