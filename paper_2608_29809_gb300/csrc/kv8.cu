// Paged eight-bit cache (rc_kv8): block tables and slot maps, and the store.
#include "common.cuh"
#include "fp8.cuh"
#include "kernels.h"

namespace rc {

namespace {

// ------------------------------------------------------- tables and slots
// One launch: every CTA sums the requests' rows and new blocks itself (at most
// KV8_MAX_REQUESTS of them, four a thread) and then writes its own part of the
// slot map.  The rows of a new block include the block's first token, so the
// thread that maps that row also writes the block's table entry, and no CTA
// reads what another one writes.
constexpr int TAB_THREADS = 1024;
constexpr int TAB_PER = KV8_MAX_REQUESTS / TAB_THREADS;  // requests of a thread

struct Request {
  int len, cnt, held, fresh;  // tokens, rows, blocks before, new blocks
};
__device__ __forceinline__ Request request(const Kv8TablesArgs& a, int r, bool report) {
  Request q{0, 0, 0, 0};
  if (r >= a.n) return q;
  const int len = a.lengths[r], cnt = a.counts ? a.counts[r] : len;
  if (len < 0 || cnt < 0 || cnt > len || len > (long long)a.ld_table * KV8_BLOCK) {
    if (report) atomicOr(a.err, DEVERR_COUNT);
    return q;
  }
  const int blocks = (len + KV8_BLOCK - 1) / KV8_BLOCK;
  q.len = len;
  q.cnt = cnt;
  q.held = a.positions ? blocks : (len - cnt + KV8_BLOCK - 1) / KV8_BLOCK;
  q.fresh = blocks - q.held;
  return q;
}

__global__ void __launch_bounds__(TAB_THREADS)
tables_kernel(const __grid_constant__ Kv8TablesArgs a, int rows_per_cta) {
  pdl_wait();
  pdl_trigger();
  // first row and first free block of each request (and behind the last)
  __shared__ int s_row[KV8_MAX_REQUESTS + 1], s_free[KV8_MAX_REQUESTS];
  __shared__ unsigned long long s_warp[32];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const bool first = blockIdx.x == 0;
  // rows in the high and blocks in the low half of one 64-bit sum
  unsigned long long mine[TAB_PER], sum = 0;
#pragma unroll
  for (int i = 0; i < TAB_PER; ++i) {
    const Request q = request(a, tid * TAB_PER + i, first);
    mine[i] = (unsigned long long)(unsigned)q.cnt << 32 | unsigned(q.fresh);
    sum += mine[i];
  }
  unsigned long long incl = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const unsigned long long v = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += v;
  }
  if (lane == 31) s_warp[warp] = incl;
  __syncthreads();
  unsigned long long at = incl - sum;
  for (int i = 0; i < warp; ++i) at += s_warp[i];
#pragma unroll
  for (int i = 0; i < TAB_PER; ++i) {
    const int r = tid * TAB_PER + i;
    s_row[r] = int(min(at >> 32, 0x7fffffffull));
    s_free[r] = int(at & 0xffffffffull);
    if (first && r < a.n) a.offsets[r] = s_row[r];
    at += mine[i];
  }
  if (tid == TAB_THREADS - 1) {
    const int total = int(min(at >> 32, 0x7fffffffull)), taken = int(at & 0xffffffffull);
    s_row[KV8_MAX_REQUESTS] = total;
    if (first) {
      a.offsets[a.n] = total;
      *a.used = taken;
      if (total > a.n_slots || taken > a.n_free) atomicOr(a.err, DEVERR_COUNT);
    }
  }
  __syncthreads();
  const int total = min(s_row[KV8_MAX_REQUESTS], a.n_slots);
  const int i0 = blockIdx.x * rows_per_cta, i1 = min(i0 + rows_per_cta, a.n_slots);
  for (int i = i0 + tid; i < i1; i += TAB_THREADS) {
    int slot = -1;
    if (i < total) {
      int lo = 0, hi = a.n;  // the request with s_row[r] <= i < s_row[r + 1]
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (s_row[mid] <= i) lo = mid;
        else hi = mid;
      }
      const Request q = request(a, lo, false);
      const int p = a.positions ? a.positions[i] : q.len - q.cnt + (i - s_row[lo]);
      if (p < 0 || p >= q.len) {
        atomicOr(a.err, DEVERR_INDEX);
      } else {
        const int blk = p / KV8_BLOCK;
        int* entry = a.table + (long long)lo * a.ld_table + blk;
        int page;
        if (blk < q.held) {
          page = *entry;
        } else {
          const int f = s_free[lo] + blk - q.held;
          page = f >= a.n_free ? -1 : a.free_blocks ? a.free_blocks[f] : f;
          if (p % KV8_BLOCK == 0) *entry = page;
        }
        if (page < 0) atomicOr(a.err, DEVERR_INDEX);
        else slot = page * KV8_BLOCK + p % KV8_BLOCK;
      }
    }
    a.slots[i] = slot;
  }
}

// ------------------------------------------------------------------ store
// A run is the rows of one block, next to one another in the list.  A CTA
// takes the runs that start among its `chunk` rows, four heads of the keys or
// of the values; the threads stand as row lanes x (heads x pieces of eight
// channels), so that a block's rows are read once, stay in registers while
// their largest magnitude is found, and leave as codes.
constexpr int ST_THREADS = 256, ST_HEADS = 4, ST_CHUNK = 16;

template <class T, int DH, bool WIDE>
__global__ void __launch_bounds__(ST_THREADS)
store_kernel(const __grid_constant__ Kv8Pool pool, const T* __restrict__ kx,
             const T* __restrict__ vx, int ldx, const int* __restrict__ slots, int n_bound,
             const int* __restrict__ count, int append, int chunk, unsigned* __restrict__ err) {
  constexpr int PIECES = DH / 8, COLS = ST_HEADS * PIECES;
  constexpr int LANES = ST_THREADS / COLS;               // row lanes
  constexpr int PER = (KV8_BLOCK + LANES - 1) / LANES;   // rows of a lane
  __shared__ int s_slot[ST_CHUNK + KV8_BLOCK + 2];       // from the row before the chunk
  __shared__ unsigned s_top[ST_HEADS];
  __shared__ int s_own[KV8_BLOCK];                       // the row of each place of the block
  pdl_wait();
  pdl_trigger();
  const int tid = threadIdx.x, c0 = blockIdx.x * chunk;
  const int n = live_count(count, n_bound, tid == 0 ? err : nullptr);
  if (c0 >= n) return;
  const long long top_slot = (long long)pool.blocks * KV8_BLOCK;
  for (int i = tid; i < chunk + KV8_BLOCK + 2; i += ST_THREADS) {
    const int r = c0 - 1 + i;
    int s = r >= 0 && r < n ? slots[r] : -1;
    if (s >= top_slot) {
      if (i > 0 && i <= chunk) atomicOr(err, DEVERR_INDEX);
      s = -1;
    }
    s_slot[i] = s < 0 ? -1 : s;
  }
  const int side = blockIdx.z;
  const int lane = tid / COLS, col = tid - lane * COLS;
  const int hl = col / PIECES, piece = col - hl * PIECES, head = blockIdx.y * ST_HEADS + hl;
  const bool on = lane < LANES && head < pool.heads;
  const T* src = (side ? vx : kx) + head * DH + piece * 8;
  __syncthreads();
  for (int start = 1; start <= chunk; ++start) {  // (uniform: every thread sees the same runs)
    const int slot0 = s_slot[start];
    if (slot0 < 0) continue;
    const int block = slot0 / KV8_BLOCK;
    if (s_slot[start - 1] >= 0 && s_slot[start - 1] / KV8_BLOCK == block) continue;
    int len = 1;
    while (len <= KV8_BLOCK && s_slot[start + len] >= 0 &&
           s_slot[start + len] / KV8_BLOCK == block)
      ++len;
    // (more rows than the block has tokens: some slot came twice)
    if (len > KV8_BLOCK) {
      len = KV8_BLOCK;
      if (tid == 0) atomicOr(err, DEVERR_INDEX);
    }
    __syncthreads();  // the run before has been read
    if (tid < KV8_BLOCK) s_own[tid] = KV8_BLOCK;
    if (tid < ST_HEADS) s_top[tid] = 0;
    __syncthreads();
    // the first row of a place fills it
    bool begins = false;
    if (tid < len) {
      const int off = s_slot[start + tid] % KV8_BLOCK;
      begins = off == 0;
      if (atomicMin(&s_own[off], tid) != KV8_BLOCK) atomicOr(err, DEVERR_INDEX);
    }
    const bool fresh = __syncthreads_or(begins) && append;
    Eight<T> v[PER];
    unsigned top = 0;
    bool live[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int k = lane + i * LANES;
      live[i] = on && k < len && s_own[s_slot[start + k] % KV8_BLOCK] == k;
      if (live[i]) {
        const T* p = src + (long long)(c0 + start - 1 + k) * ldx;
        if (WIDE) v[i].load(p);
        else v[i].load_some(p, 8);
      } else {
        v[i].zero();
      }
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) top = max(top, v[i].top());
    if (on) atomicMax(&s_top[hl], top);
    uint8_t* sc = pool.scale[side] + (long long)block * pool.heads + head;
    const int old = on && !fresh ? *sc : 0;
    __syncthreads();
    if (!on) continue;
    const int b = max(old, scale_byte(s_top[hl]));
    uint8_t* base =
        pool.code[side] + ((long long)block * pool.heads + head) * (KV8_BLOCK * DH) + piece * 8;
    const float inv = scale_inverse(b);
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      if (!live[i]) continue;
      const int off = s_slot[start + lane + i * LANES] % KV8_BLOCK;
      *reinterpret_cast<uint2*>(base + off * DH) = v[i].codes(inv);
    }
    if (b > old && !fresh) {
      // the other tokens' codes move to the raised scale (2^(old - b); below
      // 2^-126 every code becomes zero)
      const float f =
          b == 255 ? scale_value(255) : __uint_as_float(uint32_t(max(127 + old - b, 1)) << 23);
      for (int off = lane; off < KV8_BLOCK; off += LANES) {
        if (s_own[off] != KV8_BLOCK) continue;
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
    if (lane == 0 && piece == 0 && (b != old || fresh)) *sc = uint8_t(b);
  }
}

template <class T, int DH>
cudaError_t store(const Kv8Pool& pool, const T* k, const T* v, int ld, bool wide, const int* slots,
                  int n, const int* count, bool append, unsigned* err, cudaStream_t st) {
  // rows of a CTA: a decode step's rows are a run each, and want a CTA each;
  // past eight CTAs an SM a run's rows share one
  const int parts = 2 * ((pool.heads + ST_HEADS - 1) / ST_HEADS);
  const long long c = (long long)n * parts / (152 * 8);
  const int chunk = c < 1 ? 1 : c > ST_CHUNK ? ST_CHUNK : int(c);
  const dim3 grid(unsigned((n + chunk - 1) / chunk), unsigned(parts / 2), 2);
  count_launches(1);
  if (wide)
    return launch_k(store_kernel<T, DH, true>, grid, dim3(ST_THREADS), 0, st, pool, k, v, ld,
                    slots, n, count, append ? 1 : 0, chunk, err);
  return launch_k(store_kernel<T, DH, false>, grid, dim3(ST_THREADS), 0, st, pool, k, v, ld, slots,
                  n, count, append ? 1 : 0, chunk, err);
}

}  // namespace

cudaError_t launch_kv8_tables(const Kv8TablesArgs& a, cudaStream_t st) {
  int per = 4 * TAB_THREADS;
  const long long ctas = ((long long)a.n_slots + per - 1) / per;
  count_launches(1);
  return launch_k(tables_kernel, dim3(unsigned(ctas < 1 ? 1 : ctas)), dim3(TAB_THREADS), 0, st, a,
                  per);
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
