// The row work between two products (rc_norm_residual): the weighted sum of
// expert rows, norm, gate and residual of a block's output, and the norm and
// modulation before the next block, in one pass.
#include "../../include/regioncache.h"
#include "block.h"
#include "common.cuh"
#include "fp8.cuh"

#include <type_traits>

namespace rc {

namespace {

// A row is dealt in vectors of eight columns to a CTA's threads, which hold them from
// the first load to the last store, so x and h are read once; the sums of a norm go
// through the registers that hold the row (its variance is that of the differences
// from the mean, two passes there).  A mean m is as good as its sum, so the differences d
// may be off by some 2^-24 m, which is nothing to them while |m| is at most their root mean
// square.  Rows with a larger mean go through both passes once more (a constant row of
// 321.55563 gave 0.03 of a root of 1e-3 without).  The mean of d taken off every row, beside
// the squares, cost 16 % (16384 x 4608 bf16, layer norm alone, 74 us; now 66).  Sixteen neighbouring threads hold the 128 columns of a scale.
__device__ __forceinline__ void unpack(const Eight<bf16>& e, float* v) {
  const uint32_t w[4] = {e.u.x, e.u.y, e.u.z, e.u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(w[i] << 16);
    v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void unpack(const Eight<float>& e, float* v) {
  v[0] = e.a.x, v[1] = e.a.y, v[2] = e.a.z, v[3] = e.a.w;
  v[4] = e.b.x, v[5] = e.b.y, v[6] = e.b.z, v[7] = e.b.w;
}
template <class T>
__device__ __forceinline__ void load(Eight<T>& e, const T* p, int n, bool wide) {
  if (wide && n >= 8) e.load(p);
  else if (n > 0) e.load_some(p, n);
  else e.zero();
}
// Eight (n) of a vector of f32 parameters, `rest` where there are none.
__device__ __forceinline__ void parameters(const float* p, int c, int n, float rest, float* v) {
  if (p && n >= 8 && (reinterpret_cast<uintptr_t>(p) & 15) == 0) {
    const float4 a = __ldg(reinterpret_cast<const float4*>(p + c));
    const float4 b = __ldg(reinterpret_cast<const float4*>(p + c) + 1);
    v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w;
    v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = p && k < n ? __ldg(p + c + k) : rest;
  }
}
__device__ __forceinline__ void store(bf16* p, const float* v, int n, bool wide) {
  if (wide && n >= 8) {
    *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]),
                                              pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (k < n) p[k] = f2bf(v[k]);
  }
}
__device__ __forceinline__ void store(float* p, const float* v, int n, bool wide) {
  if (wide && n >= 8) {
    reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (k < n) p[k] = v[k];
  }
}

// Sum over the row's threads; `slots` of the CTA's warps, used in turn so that one
// barrier a sum is enough.
template <int TPR>
__device__ __forceinline__ float row_sum(float v, float (*slots)[16], int& turn) {
  v = warp_sum(v);
  const int warp = threadIdx.x >> 5;
  if ((threadIdx.x & 31) == 0) slots[turn][warp] = v;
  __syncthreads();
  v = 0.f;
#pragma unroll
  for (int w = 0; w < TPR / 32; ++w) v += slots[turn][w];
  turn ^= 1;
  return v;
}

// Whether the row's mean is large against what is left of it (the same for all threads).
__device__ __forceinline__ bool far_from_zero(float mean, float root) {
  return fabsf(mean) * root > 1.f;
}

template <int TPR, int NV>
__device__ __forceinline__ void normalise(const NormOf& o, float (*v)[8], int t, int cols,
                                          float (*slots)[16], int& turn) {
  if (o.kind == RC_NORM_NONE) return;
  float r;
#pragma unroll 1
  for (bool again = o.kind == RC_NORM_LAYER, first = true;; first = false) {
    float mean = 0.f, sum = 0.f;
    if (again) {
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int k = 0; k < 8; ++k) sum += v[i][k];
      mean = row_sum<TPR>(sum, slots, turn) / float(cols);
      sum = 0.f;
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int n = cols - (t + i * TPR) * 8;
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        v[i][k] = k < n ? v[i][k] - mean : 0.f;
        sum = fmaf(v[i][k], v[i][k], sum);
      }
    }
    r = 1.f / sqrtf(row_sum<TPR>(sum, slots, turn) / float(cols) + o.eps);
    again = again && first && far_from_zero(mean, r);
    if (!again) break;
  }
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = (t + i * TPR) * 8, n = cols - c;
    if (n <= 0) continue;
    float w[8], b[8];
    parameters(o.weight, c, n, 1.f, w);
    parameters(o.bias, c, n, 0.f, b);
#pragma unroll
    for (int k = 0; k < 8; ++k) v[i][k] = fmaf(v[i][k] * r, w[k], b[k]);
  }
}

// The item that owns `row` (-1 for none) and the first row behind it that may have
// another, by the whole warp: the last offset that is not above the row, a
// thirty-second of the list at a time.
__device__ __forceinline__ int item_of(const int* offsets, int n_items, int rows, int row,
                                       int& end) {
  const int lane = threadIdx.x & 31;
  int lo = 0, len = n_items;
  end = row + 1;
  if (n_items < 32) {  // (all of it with one load)
    const int v = lane <= n_items ? offsets[lane] : 0;
    const int last = 31 - __clz(int(__ballot_sync(0xffffffffu, lane < n_items && v <= row)));
    const int first = __shfl_sync(0xffffffffu, v, max(last, 0));
    const int behind = __shfl_sync(0xffffffffu, v, max(last, 0) + 1);
    if (last < 0 || first < 0 || row >= behind || behind > rows) return -1;
    end = behind;
    return last;
  }
  while (len > 1) {
    const int step = (len - 1) / 32 + 1;
    const long long at = (long long)lane * step;
    const bool under = at < len && offsets[lo + int(at)] <= row;
    const int last = 31 - __clz(int(__ballot_sync(0xffffffffu, under)));
    if (last < 0) return -1;
    lo += last * step;
    len = min(step, len - last * step);
  }
  const int first = offsets[lo], behind = offsets[lo + 1];
  if (first < 0 || first > row || row >= behind || behind > rows) return -1;
  end = behind;
  return lo;
}
// Offsets that are not in order are reported (one CTA).
__device__ __forceinline__ void check_offsets(const ResidualArgs& a) {
  for (long long i = threadIdx.x; i < a.n_items; i += blockDim.x)
    if (a.row_offsets[i] < 0 || a.row_offsets[i] > a.row_offsets[i + 1] ||
        a.row_offsets[i + 1] > a.rows)
      atomicOr(a.err, DEVERR_COUNT);
}
template <class T>
__device__ __forceinline__ bool wide_rows(const T* p, long long ld) {
  return ((reinterpret_cast<uintptr_t>(p) | uintptr_t(ld * sizeof(T))) & 15) == 0;
}
// Eight (n) outputs of a row as codes; sixteen neighbouring threads hold the columns
// of a scale (n <= 0: a thread without columns).
__device__ __forceinline__ void store_codes(const Fp8Mat& y, long long row, int c, int n,
                                            const float* v) {
  Eight<float> e;
  e.a = make_float4(v[0], v[1], v[2], v[3]);
  e.b = make_float4(v[4], v[5], v[6], v[7]);
  if (n <= 0) e.zero();
  uint32_t top = e.top();
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
  const int b = scale_byte(top);
  const uint2 q = e.codes(scale_inverse(b));
  uint8_t* dst = y.codes + row * y.ld + c;
  if (n >= 8) {
    *reinterpret_cast<uint2*>(dst) = q;
  } else {
    for (int k = 0; k < n; ++k) dst[k] = uint8_t((k < 4 ? q.x : q.y) >> (8 * (k & 3)));
  }
  if (n > 0 && (c & 127) == 0) y.scales[(long long)(c / 128) * y.lds + row] = uint8_t(b);
}
__device__ __forceinline__ void store_y(const ResidualArgs& a, long long row, int c, int n,
                                        const float* v) {
  if (a.y8.codes) {
    store_codes(a.y8, row, c, n, v);
  } else if (n > 0 && a.y_f32) {
    float* y = static_cast<float*>(a.y);
    store(y + row * a.ldy + c, v, n, wide_rows(y, a.ldy));
  } else if (n > 0) {
    bf16* y = static_cast<bf16*>(a.y);
    store(y + row * a.ldy + c, v, n, wide_rows(y, a.ldy));
  }
}

// Rows of up to 8 columns a thread of the CTA (cols <= 5120).  A CTA takes neighbouring
// rows, two at a time: their sums share barriers and shuffles, the next two are on
// their way into shared memory meanwhile, and what the columns' values are multiplied
// with and added to (weights, biases and the item's modulation, folded into one factor
// and one term for each of the two norms) stays in registers until the item changes.
// Two columns an instruction throughout.  Bound by memory where rows are many (16384 x
// 4608 bf16 94 us, 6.4 TB/s; two instructions in three were tests and scalar
// arithmetic before: 219 us, and a row for each 128 threads with its parameters
// read anew 237), and by the first rows' way where a CTA has ten (4128 x 1152
// f32 14.3 us for 8.4 of traffic; it was 27.4).
constexpr int ROWS = 2;
// Sums of both rows over the CTA's threads: the lower sixteen lanes end up with the
// first row's, the upper ones with the second's, of the warp and then of all warps.
__device__ __forceinline__ void sums(float (&v)[2], float (*slots)[2][32], int& turn) {
  const int lane = threadIdx.x & 31, half = lane >> 4, l = lane & 15;
  float s = half ? v[1] : v[0];
  s += __shfl_xor_sync(0xffffffffu, half ? v[0] : v[1], 16);
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if (l == 0) slots[turn][half][threadIdx.x >> 5] = s;
  __syncthreads();
  // (slots of warps that there are not hold zeros)
  s = slots[turn][half][l] + slots[turn][half][l + 16];
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  const float other = __shfl_xor_sync(0xffffffffu, s, 16);
  v[0] = half ? other : s, v[1] = half ? s : other;
  turn ^= 1;
}
// v - mean of the rows' columns, and 1 / root of each row; part = 1 / cols.  n of the
// thread's columns are in the row and the others hold zeros; they do again (where vectors
// are WHOLE, all or none are in the row).
template <bool WHOLE>
__device__ __forceinline__ void standardise(const NormOf& o, float2 (&v)[2][4], float (&root)[2],
                                            int n, float cols, float part,
                                            float (*slots)[2][32], int& turn) {
  root[0] = root[1] = 1.f;
  if (o.kind == RC_NORM_NONE) return;
  float s[2];
  const auto roots = [&] {
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      float2 t = f2_mul(v[r][0], v[r][0]);
#pragma unroll
      for (int k = 1; k < 4; ++k) t = f2_fma(v[r][k], v[r][k], t);
      s[r] = t.x + t.y;
    }
    sums(s, slots, turn);
#pragma unroll
    for (int r = 0; r < 2; ++r) root[r] = rsqrtf(fmaf(s[r], part, o.eps));
  };
  if (o.kind == RC_NORM_RMS) {
    roots();
    return;
  }
  bool far[2] = {true, true};
#pragma unroll 1
  for (bool first = true;; first = false) {
    float m[2];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      const float2 t = f2_add(f2_add(v[r][0], v[r][1]), f2_add(v[r][2], v[r][3]));
      s[r] = t.x + t.y;
    }
    sums(s, slots, turn);
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      m[r] = s[r] * part;
      m[r] = fmaf(fmaf(-m[r], cols, s[r]), part, m[r]);  // (the quotient s / cols)
      // (a large mean times a large root is no finite number; a row does not hang on its
      // neighbour, which may be none)
      const float of = (WHOLE && n <= 0) || !far[r] ? 0.f : m[r];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float2 d = f2_add(v[r][k], f2_of(-of));
        v[r][k] = WHOLE ? d : make_float2(2 * k < n ? d.x : 0.f, 2 * k + 1 < n ? d.y : 0.f);
      }
    }
    roots();
#pragma unroll
    for (int r = 0; r < 2; ++r) far[r] = first && far_from_zero(m[r], root[r]);
    if (!far[0] && !far[1]) return;
  }
}
// A thread's eight (n) columns of a row into its place in shared memory: under way,
// or there where the row is not aligned or too short for that.
template <class T>
__device__ __forceinline__ void stage(Eight<T>* to, const T* p, int n, bool wide) {
  if (wide && n >= 8) {
#pragma unroll
    for (int k = 0; k < int(sizeof(T)) / 2; ++k)
      copy_16(reinterpret_cast<uint4*>(to) + k, reinterpret_cast<const uint4*>(p) + k);
  } else {
    Eight<T> e;
    load(e, p, n, false);
    *to = e;
  }
}
// Batches of rows of a CTA under way or in use (4128 x 1152 f32 14.3 us; with three 15.2,
// with four 16.1, as many CTAs on an SM: the first batch waits for all that is asked for).
constexpr int DEPTH = 2;
__device__ __forceinline__ void pairs_of(const float* u, float2* v) {
#pragma unroll
  for (int k = 0; k < 4; ++k) v[k] = make_float2(u[2 * k], u[2 * k + 1]);
}

// FORM says what there is, with whole, aligned vectors: NEXT x, h (without places), x_out
// and y (of that type, or as codes); ONLY x and y alone; JOIN x, h by places and x_out.
// ANY is everything else (the tests of what there is, for each vector, took half of the
// instructions: 4128 x 1152 bf16 to codes 7.0 us for 10.6, joined with two bf16 rows of
// each by places, looked up once, 7.8 for 12.6; one row to bf16 3.3 for 4.1).
enum Form { ANY, NEXT_BF16, NEXT_F32, NEXT_CODES, ONLY_BF16, ONLY_F32, ONLY_CODES, JOIN };
// Places and weights that a CTA has in shared memory at once; RC_EXPERTS_MAX_TOP_K of a
// row at most.
constexpr int PAIRS = 512;
template <class TX, class TH, Form FORM, int THREADS>
__global__ void __launch_bounds__(THREADS, THREADS <= 256 ? 2 : 1)
norm_rows_kernel(const __grid_constant__ ResidualArgs a) {
  constexpr bool PLAIN = FORM != ANY, MAY_JOIN = FORM == ANY || FORM == JOIN,
                 NEXT = FORM == NEXT_BF16 || FORM == NEXT_F32 || FORM == NEXT_CODES,
                 ONLY = FORM == ONLY_BF16 || FORM == ONLY_F32 || FORM == ONLY_CODES,
                 CODES = FORM == NEXT_CODES || FORM == ONLY_CODES;
  using TY = std::conditional_t<FORM == NEXT_F32 || FORM == ONLY_F32, float, bf16>;
  extern __shared__ uint4 staged[];  // [DEPTH][ROWS][threads] of x, then of h
  __shared__ float slots[2][2][32];
  __shared__ int place_of[MAY_JOIN ? PAIRS : 1];
  __shared__ float weight_of[MAY_JOIN ? PAIRS : 1];
  for (int i = threadIdx.x; i < 128; i += blockDim.x) (&slots[0][0][0])[i] = 0.f;
  __syncthreads();
  pdl_wait();
  pdl_trigger();
  if (a.row_offsets && blockIdx.x == 0) check_offsets(a);
  const int c = threadIdx.x * 8, n = a.cols - c;
  const TX* x = static_cast<const TX*>(a.x);
  const TH* h = static_cast<const TH*>(a.h);
  TX* x_out = static_cast<TX*>(a.x_out);
  const bool wide_x = wide_rows(x, a.ldx), wide_h = wide_rows(h, a.ldh),
             wide_out = wide_rows(x_out, a.ldx_out);
  const int last = int((long long)(blockIdx.x + 1) * a.rows / gridDim.x);
  int row = int((long long)blockIdx.x * a.rows / gridDim.x), end = row, item = -1, turn = 0;
  Eight<TX>* sx = reinterpret_cast<Eight<TX>*>(staged) + threadIdx.x;
  Eight<TH>* sh = reinterpret_cast<Eight<TH>*>(reinterpret_cast<Eight<TX>*>(staged) +
                                               DEPTH * ROWS * blockDim.x) + threadIdx.x;
  const int top_k = MAY_JOIN ? a.top_k : 0;
  const bool own_h = FORM == ANY ? h && top_k == 0 : NEXT;
  // rows are staged in order, a group of copies for each (`left` of them are still to come;
  // below 0: asked for behind the last, where there are none); `to` and `at` are the places
  // of the next to be staged and to be read (in rows of the CTA's threads)
  const int step = blockDim.x, places = DEPTH * ROWS * step;
  int left = last - row, to = 0, at = 0;
  const TX* px = x + (long long)row * a.ldx + c;
  const TH* ph = h + (long long)row * a.ldh + c;
  const auto fetch = [&] {
    if (left > 0 && n > 0) {
      if (PLAIN) {
        stage(sx + to, px, 8, true);
        if (NEXT) stage(sh + to, ph, 8, true);
      } else {
        if (x) stage(sx + to, px, n, wide_x);
        if (own_h) stage(sh + to, ph, n, wide_h);
      }
    }
    copy_commit();
    --left;
    px += a.ldx, ph += a.ldh;
    to += step;
    if (to == places) to = 0;
  };
  // (threads without columns, and those of what there is not, read zeros)
#pragma unroll 1
  for (int i = 0; i < DEPTH * ROWS; ++i) {
    Eight<TX> zx;
    Eight<TH> zh;
    zx.zero(), zh.zero();
    if (n <= 0 || !x) sx[i * step] = zx;
    if (n <= 0 && own_h) sh[i * step] = zh;
  }
#pragma unroll 1
  for (int i = 0; i < DEPTH * ROWS; ++i) fetch();
  TX* po = x_out + (long long)row * a.ldx_out + c;
  const bool codes = FORM == ANY ? a.y8.codes != nullptr : CODES,
             y_wide = a.y_f32 ? wide_rows(static_cast<float*>(a.y), a.ldy)
                                                  : wide_rows(static_cast<bf16*>(a.y), a.ldy);
  const int y_size = a.y_f32 ? 4 : 2;
  const long long y_step = (long long)a.ldy * y_size;
  uint8_t* py = static_cast<uint8_t*>(a.y) + row * y_step + c * y_size;
  const float cols = float(a.cols), part = 1.f / cols;
  float2 pa[4], pb[4], qa[4], qb[4];  // of the branch and of y; zero outside the row
  int paired = row, pairs_from = row;  // rows whose places are in shared memory (-2: one
                                       // that there is not, of no consequence elsewhere)
  while (row < last) {
    if (MAY_JOIN && top_k > 0 && paired - row < ROWS && paired < last) {
      __syncthreads();
      pairs_from = row, paired = row + min(last - row, PAIRS / max(top_k, 1));
      for (int i = threadIdx.x; i < (paired - row) * top_k; i += step) {
        const long long pair = (long long)row * top_k + i;
        const int place = a.places[pair];
        const bool there = place >= 0 && place < a.h_rows;
        place_of[i] = there ? place : place < 0 ? -1 : -2;
        weight_of[i] = there ? a.weights[pair] : 0.f;
      }
      __syncthreads();
    }
    if (row >= end) {
      // (what does not depend on the item is on its way while that is looked up)
      float t[8], b[8], t2[8], b2[8], u[8], u2[8];
      parameters(a.post.weight, c, n, 1.f, t);
      parameters(a.post.bias, c, n, 0.f, b);
      parameters(a.pre.weight, c, n, 1.f, t2);
      parameters(a.pre.bias, c, n, 0.f, b2);
      if (a.row_offsets) {
        item = item_of(a.row_offsets, a.n_items, a.rows, row, end);
      } else {
        item = 0, end = a.rows;
      }
      const long long mod = (long long)max(item, 0) * a.ld_mod;
      parameters(a.gate ? a.gate + mod : nullptr, c, n, 1.f, u);
      parameters(a.scale ? a.scale + mod : nullptr, c, n, 0.f, u2);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        t[k] = k < n ? t[k] * u[k] : 0.f, b[k] *= u[k];
        t2[k] = k < n ? fmaf(t2[k], u2[k], t2[k]) : 0.f, b2[k] = fmaf(b2[k], u2[k], b2[k]);
      }
      parameters(a.shift ? a.shift + mod : nullptr, c, n, 0.f, u);
#pragma unroll
      for (int k = 0; k < 8; ++k) b2[k] += u[k];
      pairs_of(t, pa), pairs_of(b, pb), pairs_of(t2, qa), pairs_of(b2, qb);
    }
    const int rows = item < 0 ? 0 : min(ROWS, min(last, end) - row);
    float2 v[ROWS][4], b[ROWS][4];
    copy_wait<(DEPTH - 1) * ROWS>();
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      // (behind the last row: of no consequence)
      const int from = at + r * step < places ? at + r * step : at + r * step - places;
      const Eight<TX> ex = sx[from];
      Eight<TH> eh;
      if (own_h) eh = sh[from];
      else eh.zero();
      float u[8];
      unpack(ex, u), pairs_of(u, v[r]);
      unpack(eh, u), pairs_of(u, b[r]);
    }
    // (the thread's own places: what it has read may be staged anew)
    const int done = max(rows, 1);
    if (done == ROWS) {
#pragma unroll
      for (int i = 0; i < ROWS; ++i) fetch();
    } else {
      for (int i = 0; i < done; ++i) fetch();
    }
    at += done * step;
    if (at >= places) at -= places;
    if (rows == 0) {  // (a row of no item)
      row += 1, po += a.ldx_out, py += y_step;
      continue;
    }
    const float2 scale = f2_of(a.residual_scale);
    if (PLAIN ? !ONLY : h != nullptr) {
#pragma unroll 2
      for (int j = 0; j < top_k; ++j) {
        Eight<TH> e[ROWS];
        float w[ROWS];
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
          const int pair = (row - pairs_from + (r < rows ? r : 0)) * top_k + j;
          const int place = place_of[pair];
          w[r] = weight_of[pair];
          if (place == -2 && threadIdx.x == 0) atomicOr(a.err, DEVERR_INDEX);
          load(e[r], h + (long long)place * a.ldh + c, place < 0 || n <= 0 ? 0 : PLAIN ? 8 : n,
               PLAIN || wide_h);
        }
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
          float u[8];
          float2 t[4];
          unpack(e[r], u), pairs_of(u, t);
#pragma unroll
          for (int k = 0; k < 4; ++k) b[r][k] = f2_fma(f2_of(w[r]), t[k], b[r][k]);
        }
      }
      float root[ROWS];
      standardise<PLAIN>(a.post, b, root, n, cols, part, slots, turn);
#pragma unroll
      for (int r = 0; r < ROWS; ++r)
#pragma unroll
        for (int k = 0; k < 4; ++k)
          v[r][k] = f2_fma(v[r][k], scale,
                           f2_fma(f2_mul(b[r][k], f2_of(root[r])), pa[k], pb[k]));
    } else {
#pragma unroll
      for (int r = 0; r < ROWS; ++r)
#pragma unroll
        for (int k = 0; k < 4; ++k) v[r][k] = f2_mul(v[r][k], scale);
    }
    if (PLAIN ? !ONLY : x_out != nullptr) {
#pragma unroll
      for (int r = 0; r < ROWS; ++r)
        if (r < rows && n > 0)
          store(po + (long long)r * a.ldx_out, &v[r][0].x, PLAIN ? 8 : n, PLAIN || wide_out);
    }
    if (PLAIN ? FORM != JOIN : a.y || codes) {
      float root[ROWS];
      standardise<PLAIN>(a.pre, v, root, n, cols, part, slots, turn);
#pragma unroll
      for (int r = 0; r < ROWS; ++r) {
        if (r >= rows) break;
#pragma unroll
        for (int k = 0; k < 4; ++k)
          v[r][k] = f2_fma(f2_mul(v[r][k], f2_of(root[r])), qa[k], qb[k]);
        if constexpr (PLAIN && !CODES) {
          if (n > 0) store(reinterpret_cast<TY*>(py + r * y_step), &v[r][0].x, 8, true);
          continue;
        }
        if (codes) store_codes(a.y8, row + r, c, n, &v[r][0].x);
        else if (n > 0 && a.y_f32)
          store(reinterpret_cast<float*>(py + r * y_step), &v[r][0].x, n, y_wide);
        else if (n > 0)
          store(reinterpret_cast<bf16*>(py + r * y_step), &v[r][0].x, n, y_wide);
      }
    }
    row += done, po += done * (long long)a.ldx_out, py += done * y_step;
  }
  copy_wait<0>();
}

// Wider rows, one for each CTA: thread t of TPR holds vectors t, t + TPR ..  (NV at
// most).
template <class TX, class TH, int TPR, int NV>
__global__ void __launch_bounds__(TPR)
norm_residual_kernel(const __grid_constant__ ResidualArgs a) {
  __shared__ float slots[2][16];
  pdl_wait();
  pdl_trigger();
  const int t = threadIdx.x;
  if (a.row_offsets && blockIdx.x == 0) check_offsets(a);
  const long long row = blockIdx.x;
  const TX* x = static_cast<const TX*>(a.x);
  const TH* h = static_cast<const TH*>(a.h);
  const bool wide_x = wide_rows(x, a.ldx), wide_h = wide_rows(h, a.ldh);
  float v[NV][8], r[NV][8];
  {
    Eight<TX> ex[NV];
    Eight<TH> eh[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (t + i * TPR) * 8;
      load(ex[i], x + row * a.ldx + c, x ? a.cols - c : 0, wide_x);
      load(eh[i], h + row * a.ldh + c, h && a.top_k == 0 ? a.cols - c : 0, wide_h);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) unpack(ex[i], v[i]), unpack(eh[i], r[i]);
  }
  int end;
  const int item = a.row_offsets ? item_of(a.row_offsets, a.n_items, a.rows, int(row), end) : 0;
  if (item < 0) return;  // (the row's threads alike)
  const long long mod = (long long)item * a.ld_mod;

  for (int j = 0; h && j < a.top_k; ++j) {
    const int place = a.places[row * a.top_k + j];
    if (place < 0) continue;
    if (place >= a.h_rows) {
      if (t == 0) atomicOr(a.err, DEVERR_INDEX);
      continue;
    }
    const float w = a.weights[row * a.top_k + j];
    Eight<TH> eh[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (t + i * TPR) * 8;
      load(eh[i], h + (long long)place * a.ldh + c, a.cols - c, wide_h);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      float u[8];
      unpack(eh[i], u);
#pragma unroll
      for (int k = 0; k < 8; ++k) r[i][k] = fmaf(w, u[k], r[i][k]);
    }
  }

  int turn = 0;
  if (h) {
    normalise<TPR, NV>(a.post, r, t, a.cols, slots, turn);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (t + i * TPR) * 8, n = a.cols - c;
      if (n <= 0) continue;
      float g[8];
      parameters(a.gate ? a.gate + mod : nullptr, c, n, 1.f, g);
#pragma unroll
      for (int k = 0; k < 8; ++k)
        v[i][k] = k < n ? fmaf(a.residual_scale, v[i][k], g[k] * r[i][k]) : 0.f;
    }
  } else {
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int k = 0; k < 8; ++k) v[i][k] *= a.residual_scale;
  }
  if (a.x_out) {
    TX* out = static_cast<TX*>(a.x_out);
    const bool wide_out = wide_rows(out, a.ldx_out);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (t + i * TPR) * 8;
      if (c < a.cols) store(out + row * a.ldx_out + c, v[i], a.cols - c, wide_out);
    }
  }
  if (!a.y && !a.y8.codes) return;

  normalise<TPR, NV>(a.pre, v, t, a.cols, slots, turn);
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = (t + i * TPR) * 8, n = a.cols - c;
    if (n > 0) {
      float s[8], b[8];
      parameters(a.scale ? a.scale + mod : nullptr, c, n, 0.f, s);
      parameters(a.shift ? a.shift + mod : nullptr, c, n, 0.f, b);
#pragma unroll
      for (int k = 0; k < 8; ++k) v[i][k] = k < n ? fmaf(v[i][k], 1.f + s[k], b[k]) : 0.f;
    }
    store_y(a, row, c, n, v[i]);
  }
}

constexpr int SMS = 152;
constexpr size_t ANY_SMEM = 40 * 1024;  // that a launch has without asking, beside the slots

template <class TX, class TH, Form FORM, int THREADS>
cudaError_t rows(const ResidualArgs& a, int threads, int ctas, cudaStream_t st) {
  const bool own_h = a.h && a.top_k == 0;
  const size_t smem = size_t(DEPTH) * ROWS * threads * 8 *
                      (sizeof(TX) + (own_h ? sizeof(TH) : 0));
  // (an attribute of the current device, so set for each call that needs it; always to the
  // same, for calls of several threads)
  constexpr int most = DEPTH * ROWS * THREADS * 8 * (sizeof(TX) + sizeof(TH));
  if (smem > ANY_SMEM)
    RC_TRY(cudaFuncSetAttribute(norm_rows_kernel<TX, TH, FORM, THREADS>,
                                cudaFuncAttributeMaxDynamicSharedMemorySize, most));
  return launch_k(norm_rows_kernel<TX, TH, FORM, THREADS>,
                  dim3(unsigned(a.rows < SMS * ctas ? a.rows : SMS * ctas)),
                  dim3(unsigned(threads)), smem, st, a);
}
template <class TX, class TH, Form FORM>
cudaError_t of_form(const ResidualArgs& a, int threads, cudaStream_t st) {
  // (CTAs of an SM: what it holds at once, by their registers, of 160 threads, for 1152
  // columns.  Narrower rows, of a warp or two, could have more and run as few: 524288 x 128
  // bf16, alone, 190 us where 268 MB take 40.)
  constexpr bool ONLY = FORM == ONLY_BF16 || FORM == ONLY_F32 || FORM == ONLY_CODES;
  if (threads <= 256)
    return rows<TX, TH, FORM, 256>(a, threads, threads > 160 ? 2 : ONLY ? 4 : 3, st);
  return rows<TX, TH, FORM, 640>(a, threads, 1, st);
}

template <class TX, class TH>
cudaError_t go(const ResidualArgs& a, cudaStream_t st) {
  count_launches(1);
  const int threads = (a.cols + 255) / 256 * 32;
  if (threads > 640)
    return launch_k(norm_residual_kernel<TX, TH, 512, 4>, dim3(unsigned(a.rows)), dim3(512), 0, st,
                    a);
  const auto wide = [](const void* p, long long ld, int size) {
    return p && ((reinterpret_cast<uintptr_t>(p) | uintptr_t(ld * size)) & 15) == 0;
  };
  const bool x = a.cols % 8 == 0 && wide(a.x, a.ldx, sizeof(TX)),
             h = wide(a.h, a.ldh, sizeof(TH)), out = wide(a.x_out, a.ldx_out, sizeof(TX)),
             y = wide(a.y, a.ldy, a.y_f32 ? 4 : 2);
  if (x && !a.h && !a.x_out && (a.y8.codes || y))  // (h's type is of no consequence)
    return a.y8.codes ? of_form<TX, bf16, ONLY_CODES>(a, threads, st)
           : a.y_f32  ? of_form<TX, bf16, ONLY_F32>(a, threads, st)
                      : of_form<TX, bf16, ONLY_BF16>(a, threads, st);
  if (x && h && out && a.top_k > 0 && !a.y && !a.y8.codes)
    return of_form<TX, TH, JOIN>(a, threads, st);
  if (x && h && out && a.top_k == 0 && (a.y8.codes || y))
    return a.y8.codes ? of_form<TX, TH, NEXT_CODES>(a, threads, st)
           : a.y_f32  ? of_form<TX, TH, NEXT_F32>(a, threads, st)
                      : of_form<TX, TH, NEXT_BF16>(a, threads, st);
  return of_form<TX, TH, ANY>(a, threads, st);
}

}  // namespace

cudaError_t launch_norm_residual(const ResidualArgs& a, cudaStream_t st) {
  if (a.x_f32) return a.h_f32 ? go<float, float>(a, st) : go<float, bf16>(a, st);
  return a.h_f32 ? go<bf16, float>(a, st) : go<bf16, bf16>(a, st);
}

}  // namespace rc
