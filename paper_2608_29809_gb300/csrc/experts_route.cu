// The experts of each row and the order of the rows by expert
// (rc_experts_route, rc_experts_sort).
#include <float.h>

#include "../../include/regioncache.h"
#include "block.h"
#include "common.cuh"
#include "tc_common.cuh"

namespace rc {

namespace {

// ------------------------------------------------------------------- routing
// A warp takes a row; lane l holds experts l * PER .. l * PER + PER - 1.  Values
// are compared as unsigned keys of the same order (0: no such expert), so that a
// warp's largest is one reduction and the lowest lane and slot that hold it are
// the lowest index.
__device__ __forceinline__ uint32_t key_of(float v) {
  const uint32_t u = __float_as_uint(v + 0.f);  // (-0 as 0)
  return u >> 31 ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ uint64_t key_of(double v) {
  const uint64_t u = uint64_t(__double_as_longlong(v + 0.0));
  return u >> 63 ? ~u : u | (uint64_t(1) << 63);
}
__device__ __forceinline__ float of_key(uint32_t k) {
  return __uint_as_float(k >> 31 ? k & 0x7fffffffu : ~k);
}
__device__ __forceinline__ double of_key(uint64_t k) {
  return __longlong_as_double((long long)(k >> 63 ? k & ~(uint64_t(1) << 63) : ~k));
}
__device__ __forceinline__ uint32_t warp_max(uint32_t k) { return __reduce_max_sync(~0u, k); }
__device__ __forceinline__ uint64_t warp_max(uint64_t k) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) k = max(k, uint64_t(__shfl_xor_sync(~0u, k, o)));
  return k;
}
__device__ __forceinline__ float warp_maxf(float v) { return of_key(warp_max(key_of(v))); }

// f32 scores are off by at most `score_error(s)`: a sigmoid by 2.3 * 2^-23 (ex2
// good to 2 + |z| steps where s (1 - s) |z| < 0.23, reciprocal and sum); a softmax
// with |z - m| roundings in each exponential, whose mean is at most log(experts)
// = 7, and 37 additions.  A score plus a bias is off by half a step more.
__device__ __forceinline__ float score_error(int score, float s) {
  return score == RC_SCORE_SIGMOID ? 0x1p-21f : 0x1p-18f * s + 0x1p-23f;
}

// Keys of the groups that are not among the best `top_groups` become 0.  `scratch`:
// the warp's, a key an expert.  Returns how far apart (f32 keys) the least value
// of a chosen group and the largest of another are (infinity: no choice).
template <class K, int PER>
__device__ __forceinline__ float keep_groups(K (&key)[PER], const RoutingArgs& a, int lane,
                                             K* scratch) {
  const int size = a.experts / a.groups;
  int per = 32;  // lanes a group, a power of two
  while (per * a.groups > 32) per >>= 1;
#pragma unroll
  for (int i = 0; i < PER; ++i)
    if (lane * PER + i < a.experts) scratch[lane * PER + i] = key[i];
  __syncwarp();
  K one = 0, two = 0;
  const int g = lane / per;
  if (g < a.groups)
    for (int i = lane % per; i < size; i += per) {
      const K k = scratch[g * size + i];
      two = max(two, min(one, k));
      one = max(one, k);
    }
  for (int o = per >> 1; o > 0; o >>= 1) {
    const K k = __shfl_xor_sync(~0u, one, o), l = __shfl_xor_sync(~0u, two, o);
    two = max(min(one, k), max(two, l));
    one = max(one, k);
  }
  if (a.group_best == 2 && two != 0) one = key_of(of_key(one) + of_key(two));
  // lane g: its group's value and rank
  K mine = __shfl_sync(~0u, one, min(lane * per, 31));
  if (lane >= a.groups) mine = 0;
  int rank = 0;
  for (int h = 0; h < a.groups; ++h) {
    const K k = __shfl_sync(~0u, mine, h);
    rank += k > mine || (k == mine && h < lane);
  }
  const bool kept = mine != 0 && rank < a.top_groups;
  const uint32_t mask = __ballot_sync(~0u, kept);
  const K most = warp_max(kept ? K(0) : mine), least = ~warp_max(kept ? K(~mine) : K(0));
  int at = (lane * PER) / size, rest = lane * PER - at * size;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    if (at >= 32 || !(mask >> at & 1)) key[i] = 0;
    if (++rest == size) rest = 0, ++at;
  }
  __syncwarp();
  return most == 0 || mask == 0 ? FLT_MAX : float(of_key(least) - of_key(most));
}

// The `n` largest keys, best first: lane j gets the j-th's expert (-1: none) and key.
template <class K, int PER>
__device__ __forceinline__ void pick(K (&key)[PER], int lane, int n, int& id, K& value) {
  K best = key[0];
#pragma unroll
  for (int i = 1; i < PER; ++i) best = max(best, key[i]);
  id = -1, value = 0;
  for (int j = 0; j < n; ++j) {
    const K top = warp_max(best);
    if (top == 0) break;
    const int from = __ffs(int(__ballot_sync(~0u, best == top))) - 1;
    int slot = 0;
    if (lane == from) {
      best = 0;
#pragma unroll
      for (int i = PER - 1; i >= 0; --i)
        if (key[i] == top) slot = i;
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        if (i == slot) key[i] = 0;
        best = max(best, key[i]);
      }
    }
    slot = __shfl_sync(~0u, slot, from);
    if (lane == j) id = from * PER + slot, value = top;
  }
}

// The choice with scores in f64 (rows whose f32 values are too close).
template <int PER>
__device__ __noinline__ int choose_f64(const float (&z)[PER], const RoutingArgs& a, int lane,
                                       float m, uint64_t* scratch) {
  double s[PER], sum = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    s[i] = 0;
    if (z[i] == -INFINITY) continue;
    s[i] = a.score == RC_SCORE_SOFTMAX ? exp(double(z[i]) - double(m))
                                       : 1 / (1 + exp(-double(z[i])));
    sum += s[i];
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(~0u, sum, o);
  uint64_t key[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const double b = a.bias && z[i] != -INFINITY ? double(fminf(a.bias[lane * PER + i], FLT_MAX))
                                                 : 0;
    key[i] = z[i] == -INFINITY
                 ? 0 : key_of((a.score == RC_SCORE_SOFTMAX ? s[i] / sum : s[i]) + b);
  }
  if (a.top_groups < a.groups) keep_groups(key, a, lane, scratch);
  int id;
  uint64_t value;
  pick(key, lane, a.top_k, id, value);
  return id;
}

__device__ __forceinline__ float logit(const void* p, bool f32, long long i) {
  const float z = f32 ? static_cast<const float*>(p)[i] : bf2f(static_cast<const bf16*>(p)[i]);
  return z != z ? -INFINITY : fminf(z, FLT_MAX);
}

constexpr int ROUTE_WARPS = 4;

template <class T, int PER>
__global__ void __launch_bounds__(32 * ROUTE_WARPS)
route_kernel(const __grid_constant__ RoutingArgs a) {
  __shared__ uint64_t s_scratch[ROUTE_WARPS][PER * 32];
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31;
  const long long row = (long long)blockIdx.x * ROUTE_WARPS + (threadIdx.x >> 5);
  if (row >= a.rows) return;
  const int rows = live_count(a.count, a.rows, row == 0 && lane == 0 ? a.err : nullptr);
  if (row >= rows) {
    if (lane < a.top_k) a.ids[row * a.top_k + lane] = -1, a.weights[row * a.top_k + lane] = 0.f;
    return;
  }
  uint64_t* scratch = s_scratch[threadIdx.x >> 5];
  const long long base = row * a.ld;
  float z[PER], m = -INFINITY;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int e = lane * PER + i;
    z[i] = e < a.experts ? logit(a.logits, sizeof(T) == 4, base + e) : -INFINITY;
    if (a.bias && e < a.experts && !(a.bias[e] > -INFINITY)) z[i] = -INFINITY;
    m = fmaxf(m, z[i]);
  }
  const bool softmax = a.score == RC_SCORE_SOFTMAX, grouped = a.top_groups < a.groups;
  // (without a bias larger logits have larger scores)
  const bool by_logits = !a.bias && (!grouped || a.group_best == 1);
  float sum = 0.f;
  if (!by_logits || (softmax && !a.renormalise)) m = warp_maxf(m);
  uint32_t key[PER];
  if (by_logits) {
#pragma unroll
    for (int i = 0; i < PER; ++i) key[i] = z[i] == -INFINITY ? 0u : key_of(z[i]);
  } else {
    float s[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      s[i] = softmax ? __expf(z[i] - m) : __fdividef(1.f, 1.f + __expf(-z[i]));
      if (z[i] == -INFINITY) s[i] = 0.f;
      sum += s[i];
    }
    const float r = softmax ? 1.f / warp_sum(sum) : 1.f;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int e = lane * PER + i;
      const float b = a.bias && e < a.experts ? fminf(a.bias[e], FLT_MAX) : 0.f;
      key[i] = z[i] == -INFINITY ? 0u : key_of(fmaf(s[i], r, b));
    }
  }
  bool close = false;
  if (grouped) {
    const float gap = keep_groups(key, a, lane, reinterpret_cast<uint32_t*>(scratch));
    // (sums of two values: at most twice their errors; values of any size)
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < PER; ++i)
      if (key[i]) top = fmaxf(top, fabsf(of_key(key[i])));
    if (!by_logits)
      close = !(gap > 4.f * score_error(a.score, 1.f) + 0x1p-20f * warp_maxf(top));
  }
  int id;
  uint32_t value;
  pick(key, lane, by_logits ? a.top_k : a.top_k + 1, id, value);
  if (!by_logits) {
    // neighbours in the order that f32 does not tell apart (but for equal ones)
    const float zi = id < 0 ? 0.f : logit(a.logits, sizeof(T) == 4, base + id);
    const float bi = a.bias && id >= 0 ? a.bias[id] : 0.f, v = id < 0 ? 0.f : of_key(value);
    const int next = __shfl_down_sync(~0u, id, 1);
    const float zn = __shfl_down_sync(~0u, zi, 1), bn = __shfl_down_sync(~0u, bi, 1);
    const float vn = __shfl_down_sync(~0u, v, 1);
    if (lane < a.top_k && id >= 0 && next >= 0 && !(zi == zn && bi == bn)) {
      const float s = fminf(1.f, fmaxf(fabsf(v - bi), fabsf(vn - bn)) + 0x1p-22f);
      close |= v - vn <= 2.f * score_error(a.score, s) + 0x1p-22f * fmaxf(fabsf(v), fabsf(vn));
    }
    if (__any_sync(~0u, close)) id = choose_f64(z, a, lane, m, scratch);
  }
  // lane j: the weight of the j-th.  (With their sum divided out, exponentials are
  // taken from the largest of the chosen, so that no range of scores is lost.)
  if (lane >= a.top_k) id = -1;
  const float zi = id < 0 ? -INFINITY : logit(a.logits, sizeof(T) == 4, base + id);
  const float mc = warp_maxf(zi);
  float w = 0.f;
  if (softmax) {
    if (a.renormalise) {
      w = id < 0 || (!by_logits && mc - m < -745.f) ? 0.f : expf(zi - mc);
    } else {
      float all = 0.f;
#pragma unroll
      for (int i = 0; i < PER; ++i) all += z[i] == -INFINITY ? 0.f : expf(z[i] - m);
      all = warp_sum(all);
      w = id < 0 ? 0.f : expf(zi - m) / all;
    }
  } else if (id >= 0) {
    const float from = a.renormalise ? fminf(mc, 0.f) : 0.f;
    w = zi > 0.f ? 1.f / (1.f + expf(-zi)) : expf(zi - from) / (1.f + expf(zi));
    if (from < -745.f) w = 0.f;
  }
  if (a.renormalise) {
    const float all = warp_sum(w);
    w = all > 0.f ? w / all : 0.f;
  }
  if (lane < a.top_k) {
    a.ids[row * a.top_k + lane] = id;
    a.weights[row * a.top_k + lane] = w * a.scale;
  }
}

template <class T>
cudaError_t route(const RoutingArgs& a, cudaStream_t st) {
  const dim3 grid(unsigned((a.rows + ROUTE_WARPS - 1LL) / ROUTE_WARPS)), block(32 * ROUTE_WARPS);
  count_launches(1);
  if (a.experts <= 32) return launch_k(route_kernel<T, 1>, grid, block, 0, st, a);
  if (a.experts <= 64) return launch_k(route_kernel<T, 2>, grid, block, 0, st, a);
  if (a.experts <= 128) return launch_k(route_kernel<T, 4>, grid, block, 0, st, a);
  if (a.experts <= 256) return launch_k(route_kernel<T, 8>, grid, block, 0, st, a);
  if (a.experts <= 512) return launch_k(route_kernel<T, 16>, grid, block, 0, st, a);
  return launch_k(route_kernel<T, 32>, grid, block, 0, st, a);
}

// ------------------------------------------------------------------- sorting
// A stable counting sort by one cluster.  Each warp owns a run of consecutive
// pairs and counts its experts in a row of its own; the counts become first places
// by a scan over warps, CTAs (through their shared memory) and experts; then the
// warp deals its run out, 32 pairs at a time, equal experts of the 32 in order.
constexpr int SORT_WARPS = 32, SORT_CTAS = 8;

__global__ void __launch_bounds__(32 * SORT_WARPS, 1)
sort_kernel(const __grid_constant__ SortArgs a) {
  extern __shared__ int counts[];  // [SORT_WARPS][experts], then sums and bases [experts]
  __shared__ int parts[32];
  const int E = a.experts, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  int* sums = counts + SORT_WARPS * E;
  int* bases = sums + E;
  const int ctas = int(gridDim.x), cta = int(tc::cluster_ctarank());
  for (int i = tid; i < SORT_WARPS * E; i += blockDim.x) counts[i] = 0;
  pdl_wait();
  pdl_trigger();
  const int all = a.rows * a.top_k;
  const int n = live_count(a.count, a.rows, cta == 0 && tid == 0 ? a.err : nullptr) * a.top_k;
  // (a run is a multiple of 32)
  const int warps = ctas * SORT_WARPS, run = ((n + 31) / 32 + warps - 1) / warps * 32;
  const int from = int(min((long long)(cta * SORT_WARPS + warp) * run, (long long)n));
  const int to = int(min((long long)from + run, (long long)n));
  int* own = counts + warp * E;
  __syncthreads();
  bool bad = false;
  for (int i = from + lane; i < to; i += 32) {
    const int e = a.ids[i];
    bad |= e >= E;
    if (e >= 0 && e < E) atomicAdd(own + e, 1);
  }
  if (bad) atomicOr(a.err, DEVERR_INDEX);
  __syncthreads();
  for (int e = tid; e < E; e += blockDim.x) {
    int c[SORT_WARPS], sum = 0;
#pragma unroll
    for (int w = 0; w < SORT_WARPS; ++w) c[w] = counts[w * E + e];
#pragma unroll
    for (int w = 0; w < SORT_WARPS; ++w) {
      counts[w * E + e] = sum;
      sum += c[w];
    }
    sums[e] = sum;
  }
  tc::cluster_sync();
  // thread e: its expert's first place, and this CTA's (experts <= the block's threads)
  int total = 0, before = 0;
  if (tid < E) {
    const uint32_t at = tc::saddr(sums + tid);
    for (int c = 0; c < ctas; ++c) {
      int v;
      asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(v)
                   : "r"(tc::mapa_shared(at, uint32_t(c))));
      if (c < cta) before += v;
      total += v;
    }
  }
  int scan = total;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int v = __shfl_up_sync(~0u, scan, o);
    if (lane >= o) scan += v;
  }
  if (lane == 31) parts[warp] = scan;
  __syncthreads();
  if (warp == 0) {
    int p = parts[lane];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int v = __shfl_up_sync(~0u, p, o);
      if (lane >= o) p += v;
    }
    parts[lane] = p;
  }
  __syncthreads();
  if (warp > 0) scan += parts[warp - 1];
  if (tid < E) {
    bases[tid] = scan - total + before;
    if (cta == 0) a.offsets[tid] = scan - total;
    if (cta == 0 && tid == E - 1) a.offsets[E] = scan;
  }
  __syncthreads();
  for (int i0 = from; i0 < to; i0 += 32) {
    const int i = i0 + lane;
    int e = i < to ? a.ids[i] : -1;
    if (e < 0 || e >= E) e = -1;
    const uint32_t same = __match_any_sync(~0u, e);
    int place = -1;
    if (e >= 0) place = bases[e] + own[e] + __popc(same & ((1u << lane) - 1));
    __syncwarp();
    if (e >= 0 && lane == __ffs(int(same)) - 1) own[e] += __popc(same);
    __syncwarp();
    if (i < to) {
      a.places[i] = place;
      if (place >= 0) a.source[place] = i / a.top_k;
    }
  }
  for (int i = n + cta * int(blockDim.x) + tid; i < all; i += ctas * int(blockDim.x))
    a.places[i] = -1;
  tc::cluster_sync();  // (no CTA leaves while another may read its sums)
}

}  // namespace

cudaError_t launch_experts_route(const RoutingArgs& a, cudaStream_t st) {
  return a.f32 ? route<float>(a, st) : route<bf16>(a, st);
}

cudaError_t launch_experts_sort(const SortArgs& a, cudaStream_t st) {
  const size_t smem = size_t(SORT_WARPS + 2) * a.experts * sizeof(int);
  // (an attribute of the current device, so set for each call)
  RC_TRY(cudaFuncSetAttribute(sort_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                              int(size_t(SORT_WARPS + 2) * RC_EXPERTS_MAX * sizeof(int))));
  count_launches(1);
  const int ctas = (long long)a.rows * a.top_k > 32 * SORT_WARPS ? SORT_CTAS : 1;
  return launch_k_cluster(sort_kernel, dim3(unsigned(ctas)), dim3(32 * SORT_WARPS), smem, ctas,
                          st, a);
}

}  // namespace rc
