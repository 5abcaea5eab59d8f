// The experts of each row and the order of the rows by expert
// (rc_experts_route, rc_experts_sort).
#include <float.h>

#include "../../include/regioncache.h"
#include "block.h"
#include "common.cuh"
#include "per_device.h"
#include "tc_common.cuh"

namespace rc {

namespace {

// ------------------------------------------------------------------- routing
// A warp takes a row; lane l holds experts l * PER .. l * PER + PER - 1.  Values
// are compared as unsigned keys of the same order (0: no such expert), so that a
// warp's largest is one reduction and the lowest lane and slot that hold it are
// the lowest index.
__device__ __forceinline__ uint32_t order_of(float v) {
  const uint32_t u = __float_as_uint(v);
  return u ^ (uint32_t(int(u) >> 31) | 0x80000000u);
}
__device__ __forceinline__ uint32_t key_of(float v) { return order_of(v + 0.f); }  // (-0 as 0)
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
  return score == RC_SCORE_SIGMOID ? 0x1p-21f : 0x1p-17f * s + 0x1p-22f;
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
__device__ __forceinline__ int choose_f64(const float (&z)[PER], const RoutingArgs& a, int lane,
                                       float m, uint64_t* scratch) {
  double s[PER], sum = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {  // (no branches: the exponentials run side by side)
    const bool softmax = a.score == RC_SCORE_SOFTMAX;
    const double p = exp(softmax ? double(z[i]) - double(fmaxf(m, -FLT_MAX)) : -double(z[i]));
    s[i] = softmax ? p : 1 / (1 + p);  // (0 for -inf)
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

// The score of a logit, m the row's largest (a softmax's without its sum).
__device__ __forceinline__ float score_of(bool softmax, float z, float m) {
  const float l = 1.4426950408889634f;  // log2 e
  return softmax ? ex2_ftz((z - m) * l) : rcp_ftz(1.f + ex2_ftz(-z * l));
}
__device__ __forceinline__ float logit(const void* p, bool f32, long long i) {
  const float z = f32 ? static_cast<const float*>(p)[i] : bf2f(static_cast<const bf16*>(p)[i]);
  return z != z ? -INFINITY : fminf(z, FLT_MAX);
}

// Lane j: the expert `id` of the row's j-th choice (-1: none) and its weight, with the
// row's logits z (a lane's) and their largest m (where `with_m`).  With their sum
// divided out, exponentials are taken from the largest of the chosen, so that no range
// of scores is lost.
template <class T, int PER>
__device__ __forceinline__ void write_choice(const RoutingArgs& a, long long row, int lane, int id,
                                             const float (&z)[PER], float m, bool with_m) {
  const bool softmax = a.score == RC_SCORE_SOFTMAX;
  if (lane >= a.top_k) id = -1;
  const float zi = id < 0 ? -INFINITY : logit(a.logits, sizeof(T) == 4, row * a.ld + id);
  const float mc = warp_maxf(zi);
  float w = 0.f;
  if (softmax) {
    if (a.renormalise) {
      w = id < 0 || (with_m && mc - m < -745.f) ? 0.f : expf(zi - mc);
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

// A row with all that can be asked for.
template <class T, int PER>
__device__ __forceinline__ void route_row(const RoutingArgs& a, long long row, int lane,
                                       uint64_t* scratch) {
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
  m = warp_maxf(m);
  uint32_t key[PER];
  if (by_logits) {
#pragma unroll
    for (int i = 0; i < PER; ++i) key[i] = z[i] == -INFINITY ? 0u : key_of(z[i]);
  } else {
    float s[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      s[i] = z[i] == -INFINITY ? 0.f : score_of(softmax, z[i], m);
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
    const auto near = [&](float vn, float bn) {
      const float s = fminf(1.f, fmaxf(fabsf(v - bi), fabsf(vn - bn)) + 0x1p-22f);
      return v - vn <= 2.f * score_error(a.score, s) + 0x1p-22f * fmaxf(fabsf(v), fabsf(vn));
    };
    const int next = __shfl_down_sync(~0u, id, 1);
    const float zn = __shfl_down_sync(~0u, zi, 1), bn = __shfl_down_sync(~0u, bi, 1);
    const float vn = __shfl_down_sync(~0u, v, 1);
    const bool asked = lane < a.top_k && id >= 0 && next >= 0, equal = zi == zn && bi == bn;
    close |= asked && !equal && near(vn, bn);
    // where the last choice's neighbour is its equal, the first one behind that is not
    bool tied = asked && equal && lane == a.top_k - 1;
    while (__any_sync(~0u, tied && !close)) {
      int other;
      uint32_t v0;
      pick(key, lane, 1, other, v0);
      other = __shfl_sync(~0u, other, 0), v0 = __shfl_sync(~0u, v0, 0);
      if (other < 0) break;
      const float zo = logit(a.logits, sizeof(T) == 4, base + other);
      const float bo = a.bias ? a.bias[other] : 0.f;
      if (tied && !(zi == zo && bi == bo)) {
        close |= near(of_key(v0), bo);
        tied = false;
      }
    }
    if (__any_sync(~0u, close)) id = choose_f64(z, a, lane, m, scratch);
  }
  write_choice<T>(a, row, lane, id, z, m, true);
}

// Keys of a lane in descending order (Batcher's merges of sorted halves).
template <int N, int STRIDE, int AT, int PER>
__device__ __forceinline__ void merge_halves(uint32_t (&k)[PER]) {
  const auto order = [&](int i, int j) {
    const uint32_t hi = max(k[i], k[j]), lo = min(k[i], k[j]);
    k[i] = hi, k[j] = lo;
  };
  if constexpr (2 * STRIDE < N) {
    merge_halves<N, 2 * STRIDE, AT>(k);
    merge_halves<N, 2 * STRIDE, AT + STRIDE>(k);
#pragma unroll
    for (int i = AT + STRIDE; i + STRIDE < AT + N; i += 2 * STRIDE) order(i, i + STRIDE);
  } else {
    order(AT, AT + STRIDE);
  }
}
template <int N, int AT, int PER>
__device__ __forceinline__ void sort_keys(uint32_t (&k)[PER]) {
  if constexpr (N > 1) {
    sort_keys<N / 2, AT>(k);
    sort_keys<N / 2, AT + N / 2>(k);
    merge_halves<N, 1, AT>(k);
  }
}

constexpr int ROUTE_WARPS = 4;
// Choices that are looked at behind the last one where the order is not clear.
constexpr int MORE = 4;

// The experts `id` of the lanes (-1: none) in the order of their logits or sigmoid
// scores with bias, as of f64: lane j gets the j-th.
__device__ __forceinline__ int in_order(const RoutingArgs& a, bool f32, long long row, int lane,
                                     int id) {
  uint64_t mine = 0;
  if (id >= 0) {
    const double z = logit(a.logits, f32, row * a.ld + id);
    const double v = a.bias ? 1 / (1 + exp(-z)) + double(fminf(a.bias[id], FLT_MAX))
                            : a.top_groups < a.groups && a.group_best > 1 ? 1 / (1 + exp(-z)) : z;
    mine = key_of(v);
  }
  int rank = 0;
  for (int j = 0; j < RC_EXPERTS_MAX_TOP_K + 1 + MORE; ++j) {
    const uint64_t k = __shfl_sync(~0u, mine, j);
    const int other = __shfl_sync(~0u, id, j);
    rank += other >= 0 && (k > mine || (k == mine && other < id));
  }
  int out = -1;
  for (int j = 0; j < RC_EXPERTS_MAX_TOP_K + 1 + MORE; ++j) {
    const int r = __shfl_sync(~0u, id >= 0 ? rank : -1, j), other = __shfl_sync(~0u, id, j);
    if (r == lane) out = other;
  }
  return out;
}

// Whether the lane's group (of `lanes` lanes) is among the best by sigmoid scores with bias
// as of f64.  c: the scores in f32, two: the second best of the group, of which what may be
// among the best two in f64 is no farther than both scores may be off.
template <int PER>
__device__ __forceinline__ bool keep_group_f64(const RoutingArgs& a, bool f32, long long row,
                                               int lane, int lanes, int group,
                                               const float (&c)[PER], float two32) {
  const float least = two32 - (0x1p-19f + 0x1p-21f * fabsf(two32));
  uint32_t left = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) left |= uint32_t(c[i] > -INFINITY && !(c[i] < least)) << i;
  double one = -INFINITY, two = -INFINITY;
  while (__any_sync(~0u, left)) {
    if (!left) continue;
    const int e = lane * PER + __ffs(int(left)) - 1;
    left &= left - 1;
    const double z = logit(a.logits, f32, row * a.ld + e);
    const double v = 1 / (1 + exp(-z)) + (a.bias ? double(fminf(a.bias[e], FLT_MAX)) : 0);
    two = fmax(two, fmin(one, v));
    one = fmax(one, v);
  }
  for (int o = 1; o < lanes; o <<= 1) {
    const double k = __shfl_xor_sync(~0u, one, o), l = __shfl_xor_sync(~0u, two, o);
    two = fmax(fmin(one, k), fmax(two, l));
    one = fmax(one, k);
  }
  const double mine = a.group_best == 2 && two > -INFINITY ? one + two : one;
  int rank = 0;
  for (int h = 0; h < a.groups; ++h) {
    const double v = __shfl_sync(~0u, mine, h * lanes);
    rank += v > mine || (v == mine && h < group);
  }
  return group < a.groups && mine > -INFINITY && rank < a.top_groups;
}

// Any routing, a row for each warp.
template <class T, int PER>
__global__ void __launch_bounds__(32 * ROUTE_WARPS)
route_any_kernel(const __grid_constant__ RoutingArgs a) {
  __shared__ uint64_t scratch[ROUTE_WARPS][PER * 32];
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31;
  const long long row = (long long)blockIdx.x * ROUTE_WARPS + (threadIdx.x >> 5);
  if (row >= a.rows) return;
  const int rows = live_count(a.count, a.rows, row == 0 && lane == 0 ? a.err : nullptr);
  if (row < rows) {
    route_row<T, PER>(a, row, lane, scratch[threadIdx.x >> 5]);
  } else if (lane < a.top_k) {
    a.ids[row * a.top_k + lane] = -1, a.weights[row * a.top_k + lane] = 0.f;
  }
}

// The same where a lane's experts are of one group (a group then is 1, 2, 4 .. lanes),
// for the rows whose choice can be told from shortened keys: the value's upper bits,
// and below them the expert's number, lower numbers larger.  Keys are sorted in their
// lanes once, and a choice is then the largest head.  Neighbours closer than what a
// shortened key may be off are put in order by f64, and so are a sigmoid's groups; a
// softmax's that are that close, and rows where more values than MORE behind the last
// choice are, are left to route_row when the others are done (f64 of all experts: 12 us
// for one row).  A warp keeps the bias and takes several rows, the next one's logits
// under way.  (All rows as route_row does them: 16384 rows of 256, sigmoid, groups, 8
// each, 48 us, 1700 instructions a row; now 22.1, 970.)
template <int PER>
constexpr int ROUTE_CTAS = PER <= 4 ? 8 : PER == 8 ? 6 : PER == 16 ? 4 : 2;  // of an SM
template <class T, int PER>
__global__ void __launch_bounds__(32 * ROUTE_WARPS, ROUTE_CTAS<PER>)
route_kernel(const __grid_constant__ RoutingArgs a) {
  __shared__ uint64_t scratch[ROUTE_WARPS][PER * 32];
  const int lane = threadIdx.x & 31, e0 = lane * PER;
  const bool softmax = a.score == RC_SCORE_SOFTMAX, grouped = a.top_groups < a.groups;
  const bool by_logits = !a.bias && (!grouped || a.group_best == 1);
  constexpr uint32_t LOW = 32 * PER - 1;  // where a key has the expert
  const bool wide = ((reinterpret_cast<uintptr_t>(a.logits) | uintptr_t(a.ld * sizeof(T))) &
                     (PER * sizeof(T) < 16 ? PER * sizeof(T) - 1 : 15)) == 0 &&
                    e0 + PER <= a.experts;
  const int size = a.experts / a.groups, lanes = size / PER, group = grouped ? lane / lanes : 0;
  pdl_wait();
  pdl_trigger();
  const int rows =
      live_count(a.count, a.rows, blockIdx.x == 0 && threadIdx.x == 0 ? a.err : nullptr);
  float b[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    b[i] = a.bias && e0 + i < a.experts ? a.bias[e0 + i] : 0.f;
    b[i] = b[i] > -INFINITY ? fminf(b[i], FLT_MAX) : -INFINITY;  // (NaN: none)
  }
  constexpr int BYTES = PER * int(sizeof(T)), WORDS = BYTES < 4 ? 1 : BYTES / 4;
  uint32_t raw[WORDS];  // the lane's logits as they are
  const auto fetch = [&](long long row) {
    const T* p = static_cast<const T*>(a.logits) + row * a.ld + e0;
    if (wide) {
      if constexpr (BYTES >= 16) {
#pragma unroll
        for (int k = 0; k < WORDS; k += 4) {
          const uint4 u = reinterpret_cast<const uint4*>(p)[k / 4];
          raw[k] = u.x, raw[k + 1] = u.y, raw[k + 2] = u.z, raw[k + 3] = u.w;
        }
      } else if constexpr (BYTES == 8) {
        const uint2 u = *reinterpret_cast<const uint2*>(p);
        raw[0] = u.x, raw[1] = u.y;
      } else if constexpr (BYTES == 4) {
        raw[0] = *reinterpret_cast<const uint32_t*>(p);
      } else {
        raw[0] = *reinterpret_cast<const uint16_t*>(p);
      }
    } else if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < PER; ++i)
        raw[i] = e0 + i < a.experts ? reinterpret_cast<const uint32_t*>(p)[i]
                                    : 0xff800000u;  // -inf
    } else {
#pragma unroll
      for (int k = 0; k < WORDS; ++k) raw[k] = 0xff80ff80u;
#pragma unroll
      for (int i = 0; i < PER; ++i)
        if (e0 + i < a.experts) {
          const uint32_t u = reinterpret_cast<const uint16_t*>(p)[i];
          raw[i / 2] = i & 1 ? (raw[i / 2] & 0xffffu) | u << 16 : (raw[i / 2] & 0xffff0000u) | u;
        }
    }
  };
  const int step = gridDim.x * ROUTE_WARPS;
  uint32_t again = 0;  // of the warp's rows (32 at most), those for route_row
  int turn = 0;
  const long long first = blockIdx.x * ROUTE_WARPS + (threadIdx.x >> 5);
  long long row = first;
  if (row < rows) fetch(row);
  for (; row < rows; row += step) {
    float z[PER], m = -INFINITY;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const uint32_t u = sizeof(T) == 4 ? raw[i % WORDS]
                         : i & 1 ? raw[i / 2] & 0xffff0000u : raw[i / 2] << 16;
      z[i] = fminf(fmaxf(__uint_as_float(u), -INFINITY), FLT_MAX);  // (NaN: none)
    }
    if (softmax && a.bias) {
#pragma unroll
      for (int i = 0; i < PER; ++i)
        if (b[i] == -INFINITY) z[i] = -INFINITY;
    }
    if (row + step < rows) fetch(row + step);
    const bool with_m = softmax && (!by_logits || !a.renormalise);
    if (with_m) {
#pragma unroll
      for (int i = 0; i < PER; ++i) m = fmaxf(m, z[i]);
      m = warp_maxf(m);
    }
    float c[PER];  // what experts are chosen by
    float most = 1.f;  // of a score
    if (by_logits) {
#pragma unroll
      for (int i = 0; i < PER; ++i) c[i] = z[i] + 0.f;  // (-0 as 0)
    } else if (softmax) {
      float sum = 0.f;
      m = fmaxf(m, -FLT_MAX);
#pragma unroll
      for (int i = 0; i < PER; ++i) sum += c[i] = score_of(true, z[i], m);
      const float r = 1.f / warp_sum(sum);
      most = fminf(most, r);
#pragma unroll
      for (int i = 0; i < PER; ++i) c[i] = z[i] == -INFINITY ? -INFINITY : fmaf(c[i], r, b[i]);
    } else {
#pragma unroll
      for (int i = 0; i < PER; ++i)
        c[i] = z[i] == -INFINITY ? -INFINITY : score_of(false, z[i], 0.f) + b[i];
    }
    bool close = false;
    if (grouped) {
      float one = -INFINITY, two = -INFINITY;
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        two = fmaxf(two, fminf(one, c[i]));
        one = fmaxf(one, c[i]);
      }
      for (int o = 1; o < lanes; o <<= 1) {
        const float k = __shfl_xor_sync(~0u, one, o), l = __shfl_xor_sync(~0u, two, o);
        two = fmaxf(fminf(one, k), fmaxf(two, l));
        one = fmaxf(one, k);
      }
      // (a sum of two of the lowest biases is beyond f32: the group is there all the same, and
      // as close to another such as can be)
      const float mine = one == -INFINITY ? one
                         : fmaxf(a.group_best == 2 && two > -INFINITY ? one + two : one, -FLT_MAX);
      int rank = 0;
      for (int h = 0; h < a.groups; ++h) {
        const float v = __shfl_sync(~0u, mine, h * lanes);
        rank += v > mine || (v == mine && h < group);
      }
      bool kept = group < a.groups && mine > -INFINITY && rank < a.top_groups;
      if (!by_logits) {
        const uint32_t k = group < a.groups ? key_of(mine) : 0u;
        const float other = of_key(max(warp_max(kept ? 0u : k), key_of(-FLT_MAX)));
        const float least = of_key(~warp_max(kept ? ~k : 0u));
        // (sums of two values: at most twice their errors; a lane without a group, or of a masked
        // one, has nothing to add)
        const float largest = fmaxf(one > -INFINITY ? fabsf(one) : 0.f,
                                    two > -INFINITY ? fabsf(two) : 0.f);
        close = __any_sync(~0u, kept) &&
                !(least - other > 4.f * score_error(a.score, most) + 0x1p-20f * largest +
                                      0x1p-20f * fmaxf(fabsf(least), fabsf(other)));
        if (!softmax && __any_sync(~0u, close)) {
          kept = keep_group_f64(a, sizeof(T) == 4, row, lane, lanes, group, c, two);
          close = false;
        }
      }
      if (!kept)
#pragma unroll
        for (int i = 0; i < PER; ++i) c[i] = -INFINITY;
    }
    uint32_t k[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) k[i] = (order_of(c[i]) & ~LOW) | (LOW - uint32_t(e0 + i));
    sort_keys<PER, 0>(k);
    uint32_t value = 0;  // lane j: the j-th largest
    const auto pick_more = [&](int from, int to) {
#pragma unroll 1
      for (int j = from; j < to; ++j) {
        const uint32_t top = warp_max(k[0]);
        if (k[0] == top) {
#pragma unroll
          for (int i = 0; i + 1 < PER; ++i) k[i] = k[i + 1];
          k[PER - 1] = 0;
        }
        if (lane == j && top >= (key_of(-FLT_MAX) & ~LOW)) value = top;  // (others: -inf)
      }
    };
    // whether lane j's choice may not come before lane j + 1's (asked by all lanes)
    const auto near = [&] {
      const uint32_t next = __shfl_down_sync(~0u, value, 1);
      // (of bf16 the lower half of a key is free: equal logits are in order)
      if (by_logits) return next && sizeof(T) == 4 && ((value ^ next) & ~LOW) == 0;
      const float v = of_key(value & ~LOW), w = of_key(next & ~LOW);
      return next && !(v - w > 2.f * score_error(a.score, most) +
                                   (LOW + 5) * 0x1p-23f * fmaxf(fabsf(v), fabsf(w)) + 0x1p-100f);
    };
    pick_more(0, a.top_k + 1);
    int id = value ? int(LOW - (value & LOW)) : -1;
    const bool unclear = near();
    if (__any_sync(~0u, lane < a.top_k && unclear)) {
      // a few more, up to the first behind the last choice that is clear of the next
      pick_more(a.top_k + 1, a.top_k + 1 + MORE);
      id = value ? int(LOW - (value & LOW)) : -1;
      const bool apart = !near();
      const uint32_t ends = __ballot_sync(~0u, apart && lane >= a.top_k - 1 &&
                                                   lane < a.top_k + MORE);
      if (!ends || (softmax && !by_logits)) close = true;
      else id = in_order(a, sizeof(T) == 4, row, lane, lane < __ffs(int(ends)) ? id : -1);
    }
    if (__any_sync(~0u, close))
      again |= 1u << turn;
    else
      write_choice<T>(a, row, lane, id, z, m, with_m);
    ++turn;
  }
  // (here, where nothing else is alive)
  for (; again; again &= again - 1)
    route_row<T, PER>(a, first + (__ffs(int(again)) - 1) * (long long)step, lane,
                      scratch[threadIdx.x >> 5]);
  for (row = rows + blockIdx.x * ROUTE_WARPS + (threadIdx.x >> 5); row < a.rows; row += step)
    if (lane < a.top_k) a.ids[row * a.top_k + lane] = -1, a.weights[row * a.top_k + lane] = 0.f;
}

template <class T, int PER>
cudaError_t route_of(const RoutingArgs& a, cudaStream_t st) {
  const int size = a.experts / a.groups, lanes = size / PER;
  const bool whole = a.top_groups == a.groups ||
                     (size % PER == 0 && (lanes & (lanes - 1)) == 0);
  const long long ctas = (a.rows + ROUTE_WARPS - 1LL) / ROUTE_WARPS;
  const dim3 block(32 * ROUTE_WARPS);
  if (!whole) return launch_k(route_any_kernel<T, PER>, dim3(unsigned(ctas)), block, 0, st, a);
  // (as many CTAs as the SMs hold at once, or more: a warp takes 32 rows at most)
  const long long held = 152 * ROUTE_CTAS<PER>, least = (ctas + 31) / 32;
  const long long grid = ctas < held ? ctas : least > held ? least : held;
  return launch_k(route_kernel<T, PER>, dim3(unsigned(grid)), block, 0, st, a);
}

template <class T>
cudaError_t route(const RoutingArgs& a, cudaStream_t st) {
  count_launches(1);
  if (a.experts <= 32) return route_of<T, 1>(a, st);
  if (a.experts <= 64) return route_of<T, 2>(a, st);
  if (a.experts <= 128) return route_of<T, 4>(a, st);
  if (a.experts <= 256) return route_of<T, 8>(a, st);
  if (a.experts <= 512) return route_of<T, 16>(a, st);
  return route_of<T, 32>(a, st);
}

// ------------------------------------------------------------------- sorting
// A stable counting sort by one cluster.  Each warp owns a run of consecutive pairs and
// counts its experts in a row of its own, 32 pairs at a time; a pair's place among its
// warp's is what the count was, and its number among equal ones of the 32.  The counts
// become first places by a scan over warps, CTAs (through their shared memory) and
// experts.  The pairs and their places in the run stay in registers in between where a
// run has KEEP or fewer of the 32s.
constexpr int SORT_WARPS = 32, KEEP = 8;

__global__ void __launch_bounds__(32 * SORT_WARPS, 1)
sort_kernel(const __grid_constant__ SortArgs a) {
  extern __shared__ int counts[];  // [warps][experts], then sums and bases [experts]
  __shared__ int parts[32];
  const int E = a.experts, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int ctas = int(gridDim.x), cta = int(tc::cluster_ctarank());
  pdl_wait();
  pdl_trigger();
  const int all = a.rows * a.top_k;
  const int n = live_count(a.count, a.rows, cta == 0 && tid == 0 ? a.err : nullptr) * a.top_k;
  // (a run is a multiple of 32; where there is one CTA, a warp each 32)
  const int warps = ctas * SORT_WARPS, run = ((n + 31) / 32 + warps - 1) / warps * 32;
  const int used = ctas > 1 ? SORT_WARPS : min(SORT_WARPS, (n + 31) / 32);  // warps with pairs
  int* sums = counts + SORT_WARPS * E;
  int* bases = sums + E;
  const int from = int(min((long long)(cta * SORT_WARPS + warp) * run, (long long)n));
  const int to = int(min((long long)from + run, (long long)n));
  int* own = counts + warp * E;
  int e[KEEP], at[KEEP];
#pragma unroll
  for (int k = 0; k < KEEP; ++k) {
    const int i = from + 32 * k + lane;
    e[k] = i < to ? a.ids[i] : -1;
  }
  for (int i = tid; i < used * E; i += blockDim.x) counts[i] = 0;
  __syncthreads();
  bool bad = false;
  const auto count = [&](int& id) {
    bad |= id >= E;
    if (id < 0 || id >= E) id = -1;
    // the lanes of the same expert, by its bits
    uint32_t same = __ballot_sync(~0u, id >= 0);
    if (id < 0) same = ~same;
    for (int b = 1; b < E; b <<= 1) {
      const uint32_t set = __ballot_sync(~0u, id & b);
      same &= id & b ? set : ~set;
    }
    int place = 0;
    if (id >= 0) place = own[id] + __popc(same & ((1u << lane) - 1));
    __syncwarp();
    if (id >= 0 && lane == 31 - __clz(int(same))) own[id] = place + 1;
    __syncwarp();
    return place;
  };
#pragma unroll
  for (int k = 0; k < KEEP; ++k)
    if (from + 32 * k < to) at[k] = count(e[k]);
  for (int i0 = from + 32 * KEEP; i0 < to; i0 += 32) {
    int id = i0 + lane < to ? a.ids[i0 + lane] : -1;
    const int place = count(id);
    if (i0 + lane < to) a.places[i0 + lane] = place;  // (for now)
  }
  if (bad) atomicOr(a.err, DEVERR_INDEX);
  __syncthreads();
  int total = 0, before = 0;  // of expert `tid` (experts <= the block's threads)
  if (tid < E) {
    int sum = 0;
#pragma unroll 8
    for (int w = 0; w < used; ++w) {
      const int c = counts[w * E + tid];
      counts[w * E + tid] = sum;
      sum += c;
    }
    sums[tid] = total = sum;
  }
  if (ctas > 1) {
    tc::cluster_sync();
    if (tid < E) {
      const uint32_t mine = tc::saddr(sums + tid);
      total = 0;
      for (int c = 0; c < ctas; ++c) {
        int v;
        asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(v)
                     : "r"(tc::mapa_shared(mine, uint32_t(c))));
        if (c < cta) before += v;
        total += v;
      }
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
  // (every warp sums up the parts before it)
  int p = lane < warp ? parts[lane] : 0;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) p += __shfl_xor_sync(~0u, p, o);
  scan += p;
  if (tid < E) {
    bases[tid] = scan - total + before;
    if (cta == 0) a.offsets[tid] = scan - total;
    if (cta == 0 && tid == E - 1) a.offsets[E] = scan;
  }
  __syncthreads();
  const auto write = [&](int i, int id, int place) {
    if (id >= 0) {
      place += bases[id] + own[id];
      a.source[place] = i / a.top_k;
    }
    a.places[i] = id >= 0 ? place : -1;
  };
#pragma unroll
  for (int k = 0; k < KEEP; ++k)
    if (from + 32 * k + lane < to) write(from + 32 * k + lane, e[k], at[k]);
  for (int i = from + 32 * KEEP + lane; i < to; i += 32) {
    const int id = a.ids[i];
    write(i, id >= E ? -1 : id, a.places[i]);
  }
  for (int i = n + cta * int(blockDim.x) + tid; i < all; i += ctas * int(blockDim.x))
    a.places[i] = -1;
  if (ctas > 1) tc::cluster_sync();  // (no CTA leaves while another may read its sums)
}

// Whether the device places a cluster of sixteen CTAs (more than any device has to).
bool sixteen_fit(size_t smem) {
  static PerDevice<1> known;
  int device = -1;
  if (cudaGetDevice(&device) != cudaSuccess) return false;
  return known.get(device, 0, [&] {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(16);
    cfg.blockDim = dim3(32 * SORT_WARPS);
    cfg.dynamicSmemBytes = smem;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = 16, attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    int clusters = 0;
    if (cudaOccupancyMaxActiveClusters(&clusters, sort_kernel, &cfg) != cudaSuccess) {
      cudaGetLastError();
      return 0;
    }
    return clusters > 0 ? 1 : 0;
  }) > 0;
}

}  // namespace

cudaError_t launch_experts_route(const RoutingArgs& a, cudaStream_t st) {
  return a.f32 ? route<float>(a, st) : route<bf16>(a, st);
}

cudaError_t launch_experts_sort(const SortArgs& a, cudaStream_t st) {
  const size_t smem = size_t(SORT_WARPS + 2) * a.experts * sizeof(int);
  constexpr size_t most = size_t(SORT_WARPS + 2) * RC_EXPERTS_MAX * sizeof(int);
  // One CTA where it has a warp for each 32 pairs; sixteen where the places' writes are
  // what counts (131072 pairs: a CTA's 32 scattered writes take an SM as many cycles).
  const long long pairs = (long long)a.rows * a.top_k;
  // (attributes of the current device, so set for each call that needs them)
  if (pairs > 16384)
    RC_TRY(cudaFuncSetAttribute(sort_kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
  if (pairs > 16384 || smem > 40 * 1024)  // (up to 48 KB a launch has without asking)
    RC_TRY(cudaFuncSetAttribute(sort_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                int(most)));
  count_launches(1);
  const int ctas = pairs <= 32 * SORT_WARPS ? 1 : pairs > 16384 && sixteen_fit(most) ? 16 : 8;
  return launch_k_cluster(sort_kernel, dim3(unsigned(ctas)), dim3(32 * SORT_WARPS), smem, ctas,
                          st, a);
}

}  // namespace rc
