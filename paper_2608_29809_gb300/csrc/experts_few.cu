// Products of each expert's rows with its quantised matrix (rc_experts_linear) where
// experts have a few rows each and there are few of them: latency is all that counts,
// to which the tensor core of experts_linear.cu, fed by way of shared and tensor
// memory, adds (a block of one token: 9.5 and 10.5 us for its two products of 5 MB
// each; here 8.1 and 6.6, most of them a chain of round trips: offsets, source, x and
// scales, blocks of W, the join).
//
// A CTA's warps take up to ROWS rows of an expert and CW tiles of 16 of its outputs, the
// columns in runs for the rest of its warps.  A warp copies its tile's codes, 16 bytes a
// lane and row, some blocks of 128 columns ahead into shared memory; the same lane takes
// them back, so nothing waits for another warp.  The rows of x and all scales are
// there once for the CTA.  Codes become f16 (exact) and go through the m16n8k16 MMA: a
// product's order of columns is free, so each lane's 16 bytes are four such steps of
// its own.  A block's sums, f32, are scaled and added up; runs and the activation are
// joined in shared memory.  A scale is kept as two powers of 2 of half the exponent: sums
// times one of x's and of W's, and then times the others, pass the largest f32 on the way
// only where the result does (x of 1e36 and W of 1e-36: either scale alone is too much).
#include "../../include/regioncache.h"
#include "block.h"
#include "common.cuh"
#include "experts_act.cuh"
#include "fp8.cuh"

namespace rc {

namespace {

constexpr int DEPTH = 4, BLOCK = 2048;  // blocks under way, bytes of W in a warp's

struct FewPlan {
  int cw, kw, nt, kb;
};

__device__ __forceinline__ void mma_f16(float* d, uint32_t a0, uint32_t a1, uint32_t a2,
                                        uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, "
      "{%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// The two powers of 2 whose product is a scale (NaN for 255), the larger one first for
// x's and last for W's.
__device__ __forceinline__ float2 scale_halves(int b, bool larger_first) {
  if (b == 255) return make_float2(__uint_as_float(0x7fffffffu), 1.f);
  const int lo = (b - 127) >> 1, hi = b - 127 - lo;
  return make_float2(__uint_as_float(uint32_t(127 + (larger_first ? hi : lo)) << 23),
                     __uint_as_float(uint32_t(127 + (larger_first ? lo : hi)) << 23));
}
// Sixteen codes of which the first `left` are columns into shared memory, zeros behind.
__device__ __forceinline__ void copy_some(uint4* to, const uint8_t* from, int left) {
  uint8_t* b = reinterpret_cast<uint8_t*>(to);
#pragma unroll 1
  for (int i = 0; i < 16; ++i) b[i] = i < left ? from[i] : uint8_t(0);
}

template <ExpertsOut OUT, int NT, int WARPS>
__global__ void __launch_bounds__(32 * WARPS, 16 / WARPS)
experts_few_kernel(const __grid_constant__ ExpertsArgs a, const __grid_constant__ FewPlan pl) {
  constexpr int ROWS = 8 * NT, THREADS = 32 * WARPS;
  extern __shared__ uint4 smem[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  pdl_wait();
  pdl_trigger();
  // the chunk of rows: the q-th, of ROWS each, of all experts'
  const int q = blockIdx.x / pl.nt, tile_n = blockIdx.x - q * pl.nt;
  int expert = -1, place = 0, rows = 0;
  for (int e0 = 0, before = 0; e0 < a.experts; e0 += 32) {
    const int e = e0 + lane;
    int lo = 0, hi = 0;
    if (e < a.experts) lo = a.offsets[e], hi = a.offsets[e + 1];
    if (lo < 0 || lo > hi || hi > a.pairs) {
      if (blockIdx.x == 0 && warp == 0) atomicOr(a.err, DEVERR_COUNT);
      lo = hi = 0;
    }
    const int mine = (hi - lo + ROWS - 1) / ROWS;
    int sum = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int v = __shfl_up_sync(~0u, sum, o);
      if (lane >= o) sum += v;
    }
    const uint32_t behind = __ballot_sync(~0u, before + sum > q);
    if (behind && expert < 0) {
      const int from = __ffs(int(behind)) - 1;
      expert = e0 + from;
      place = lo + (q - (before + sum - mine)) * ROWS;
      rows = min(ROWS, hi - place);
      place = __shfl_sync(~0u, place, from);
      rows = __shfl_sync(~0u, rows, from);
      if (blockIdx.x != 0) break;  // (one CTA looks at all offsets)
    }
    before = __shfl_sync(~0u, before + sum, 31);
  }
  if (expert < 0) return;

  const bool gated = a.act == RC_ACT_GATED_SILU;
  const int cw = warp % pl.cw, ks = warp / pl.cw;  // (cw * kw = WARPS)
  const int e_rows = a.w.rows / a.experts, N = gated ? 2 * a.n : a.n;
  const int c0 = tile_n * pl.cw * 16;  // the CTA's outputs
  const int kb0 = ks * pl.kb / pl.kw, kb1 = (ks + 1) * pl.kb / pl.kw;
  const int cols = a.x.cols, full = min(kb1, cols / 128);  // (blocks before that are whole)
  const int parts = gated ? 2 : 1, out_cols = pl.cw * 16;
  // shared memory: the warps' rings, the rows of x (a block of each, 128 bytes, after
  // another), their scales [block][row], W's [part][first, second 128 rows][block], sums
  uint4* ring = smem + warp * (DEPTH * BLOCK / 16) + lane;
  uint8_t* xs = reinterpret_cast<uint8_t*>(smem + WARPS * (DEPTH * BLOCK / 16));
  float2* sx = reinterpret_cast<float2*>(xs + pl.kb * ROWS * 128);
  float2* sw = sx + pl.kb * ROWS;
  float* sums = reinterpret_cast<float*>(sw + 4 * pl.kb);

  // (outputs behind the last read rows of the expert that are never written; its
  // matrix has them up to a multiple of 128)
  const auto w_row = [&](int part, int i) {
    return (long long)expert * e_rows + min(min(part * a.n + c0, e_rows - 1) + i, e_rows - 1);
  };
  const uint8_t* pw[2];
  int staged = kb0, to = 0;  // the next block to be staged, and where
  const auto fetch = [&] {
    uint4* at = ring + to * (BLOCK / 16);
    if (staged < full) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        copy_16(at + (2 * h) * 32, pw[0] + 64 * h);
        copy_16(at + (2 * h + 1) * 32, pw[1] + 64 * h);
      }
    } else if (staged < kb1) {  // (the last columns)
#pragma unroll 1
      for (int h = 0; h < 2; ++h) {
        const int left = cols - staged * 128 - 64 * h - 16 * t;
        copy_some(at + (2 * h) * 32, pw[0] + 64 * h, left);
        copy_some(at + (2 * h + 1) * 32, pw[1] + 64 * h, left);
      }
    }
    copy_commit();
    ++staged;
    pw[0] += 128, pw[1] += 128;
    if (++to == DEPTH) to = 0;
  };
#pragma unroll 1
  for (int part = 0; part < parts; ++part) {
    const int r0 = cw * 16 + g;
    pw[0] = a.w.codes + w_row(part, r0) * a.w.ld + kb0 * 128LL + 16 * t;
    pw[1] = a.w.codes + w_row(part, r0 + 8) * a.w.ld + kb0 * 128LL + 16 * t;
    staged = kb0, to = 0;
#pragma unroll 1
    for (int i = 0; i < DEPTH - 1; ++i) fetch();
    if (part == 0) {
      // the rows of x, a warp's a row (rows that there are not: any), and the scales
      for (int r = warp; r < ROWS; r += WARPS) {
        int row = place + min(r, rows - 1);
        if (a.source) {
          row = a.source[row];
          if (row < 0 || row >= a.x.rows) {
            if (lane == 0) atomicOr(a.err, DEVERR_INDEX);
            row = 0;
          }
        }
        const uint8_t* from = a.x.codes + (long long)row * a.x.ld;
        for (int c = 16 * lane; c < pl.kb * 128; c += 512) {
          uint4* at = reinterpret_cast<uint4*>(xs + (c / 128 * ROWS + r) * 128 + c % 128);
          if (c + 16 <= cols) *at = *reinterpret_cast<const uint4*>(from + c);
          else copy_some(at, from + c, cols - c);
        }
        for (int k = lane; k < pl.kb; k += 32)
          sx[k * ROWS + r] = scale_halves(a.x.scales[(long long)k * a.x.lds + row], true);
      }
      for (int i = threadIdx.x; i < 2 * parts * pl.kb; i += THREADS) {
        const int k = i % pl.kb, which = i / pl.kb;  // [part][first, second]
        sw[i] = scale_halves(a.w.scales[(long long)k * a.w.lds +
                                        w_row(which >> 1, which & 1 ? out_cols - 1 : 0) / 128],
                             false);
      }
      __syncthreads();
    }
    const long long block0 = w_row(part, 0) / 128;
    const float2* f_of[2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
      f_of[i] = sw + (2 * part + (w_row(part, r0 + 8 * i) / 128 != block0 ? 1 : 0)) * pl.kb;
    float total[NT][4] = {};
    int slot = 0;
#pragma unroll 1
    for (int kb = kb0; kb < kb1; ++kb) {
      copy_wait<DEPTH - 2>();
      // (of W's only what the lane itself has put there)
      const uint4* from = ring + slot * (BLOCK / 16);
      const uint4* xf = reinterpret_cast<const uint4*>(xs + (kb * ROWS + g) * 128) + t;
      float block[NT][2][4] = {};  // (two chains of MMAs)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint4 wa = from[(2 * h) * 32], wb = from[(2 * h + 1) * 32];
        const uint32_t qa[4] = {wa.x, wa.y, wa.z, wa.w}, qb[4] = {wb.x, wb.y, wb.z, wb.w};
        uint4 xv[NT];
#pragma unroll
        for (int j = 0; j < NT; ++j) xv[j] = xf[j * 64 + h * 4];
#pragma unroll
        for (int m = 0; m < 4; ++m) {
          uint32_t fa[2], fb[2];
          e4m3x4_f16(qa[m], fa[0], fa[1]);
          e4m3x4_f16(qb[m], fb[0], fb[1]);
#pragma unroll
          for (int j = 0; j < NT; ++j) {
            const uint32_t qx[4] = {xv[j].x, xv[j].y, xv[j].z, xv[j].w};
            uint32_t b0, b1;
            e4m3x4_f16(qx[m], b0, b1);
            mma_f16(block[j][m & 1], fa[0], fb[0], fa[1], fb[1], b0, b1);
          }
        }
      }
      fetch();
      if (++slot == DEPTH) slot = 0;
      const float2 f[2] = {f_of[0][kb], f_of[1][kb]};
#pragma unroll
      for (int j = 0; j < NT; ++j) {  // (the lane's rows 2 t, 2 t + 1 of each eight)
        const float4 two = *reinterpret_cast<const float4*>(sx + kb * ROWS + 8 * j + 2 * t);
        const float2 x[2] = {make_float2(two.x, two.y), make_float2(two.z, two.w)};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float sum = block[j][0][i] + block[j][1][i];
          total[j][i] = fmaf(sum * (x[i & 1].x * f[i >> 1].x), x[i & 1].y * f[i >> 1].y,
                             total[j][i]);
        }
      }
    }
    copy_wait<0>();
    // [part][run][row][output]
    float* mine = sums + ((part * pl.kw + ks) * ROWS) * out_cols + cw * 16;
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        mine[(8 * j + 2 * t + (i & 1)) * out_cols + g + 8 * (i >> 1)] = total[j][i];
  }
  __syncthreads();
  // a row and 32 outputs for each warp (128 with codes)
  constexpr int LANES = OUT == OUT_CODES ? 4 : 1;
  const int per_row = (out_cols + 32 * LANES - 1) / (32 * LANES);
  for (int u = warp; u < rows * per_row; u += WARPS) {
    const int row = u / per_row, ch = u - row * per_row;
    float v[LANES];
#pragma unroll
    for (int i = 0; i < LANES; ++i) {
      const int o = (ch * LANES + i) * 32 + lane, c = c0 + o;
      v[i] = 0.f;
      if (o >= out_cols || c >= a.n) continue;
      float s[2] = {0.f, 0.f};
      for (int part = 0; part < parts; ++part) {
        for (int k = 0; k < pl.kw; ++k)
          s[part] += sums[((part * pl.kw + k) * ROWS + row) * out_cols + o];
        if (a.bias) s[part] += __ldg(a.bias + (long long)expert * N + part * a.n + c);
      }
      v[i] = gated ? act_of(RC_ACT_SILU, s[0]) * s[1] : act_of(a.act, s[0]);
    }
    const long long at = place + row;
    if constexpr (OUT == OUT_CODES) {
      const int c = c0 + ch * 128;
      uint32_t top = 0;
#pragma unroll
      for (int i = 0; i < LANES; ++i) top = max(top, __float_as_uint(v[i]) & 0x7fffffffu);
      top = __reduce_max_sync(~0u, top);
      const int b = scale_byte(top);
      const float inv = scale_inverse(b);
#pragma unroll
      for (int i = 0; i < LANES; ++i)
        if (c + i * 32 + lane < a.n)
          a.y8.codes[at * a.y8.ld + c + i * 32 + lane] = uint8_t(e4m3x2(v[i] * inv, 0.f));
      if (lane == 0 && c < a.n) a.y8.scales[(long long)(c / 128) * a.y8.lds + at] = uint8_t(b);
    } else {
      const int o = ch * 32 + lane, c = c0 + o;
      if (o < out_cols && c < a.n) {
        if constexpr (OUT == OUT_F32) static_cast<float*>(a.y)[at * a.ldy + c] = v[0];
        else static_cast<bf16*>(a.y)[at * a.ldy + c] = f2bf(v[0]);
      }
    }
  }
}

constexpr int SMS = 152;
constexpr size_t MOST_SMEM = 227 * 1024;

size_t smem_of(const ExpertsArgs& a, int rows, int warps) {
  const size_t kb = size_t(a.x.cols - 1) / 128 + 1, parts = a.act == RC_ACT_GATED_SILU ? 2 : 1;
  return size_t(warps) * DEPTH * BLOCK + kb * (rows * 136 + 32) +
         parts * warps * 16 * rows * sizeof(float);
}
// (codes are made 128 outputs at a time: the CTAs are fewer, and have more warps)
int warps_of(const ExpertsArgs& a) { return a.y8.codes && a.x.cols > 128 ? 16 : 8; }
long long chunks_of(const ExpertsArgs& a, int rows) {
  const long long used = a.pairs < a.experts ? a.pairs : a.experts;
  return used + (a.pairs - used) / rows;
}

template <ExpertsOut OUT, int NT, int WARPS>
cudaError_t go(const ExpertsArgs& a, cudaStream_t st) {
  constexpr int ROWS = 8 * NT;
  const long long chunks = chunks_of(a, ROWS);
  FewPlan pl;
  pl.kb = (a.x.cols - 1) / 128 + 1;
  // as many tiles in a CTA as leave a CTA for each half of an SM, and a run of columns
  // for each warp
  pl.cw = 8;
  while (OUT != OUT_CODES && pl.cw > 1 && chunks * ((a.n - 1) / (16 * pl.cw) + 1) < 2 * SMS &&
         2 * (WARPS / pl.cw) <= pl.kb)
    pl.cw /= 2;
  pl.kw = WARPS / pl.cw;
  pl.nt = (a.n - 1) / (16 * pl.cw) + 1;
  const size_t smem = smem_of(a, ROWS, WARPS);
  // (an attribute of the current device, so set for each call; always to the same, for
  // calls of several threads)
  RC_TRY(cudaFuncSetAttribute(experts_few_kernel<OUT, NT, WARPS>,
                              cudaFuncAttributeMaxDynamicSharedMemorySize, int(MOST_SMEM)));
  count_launches(1);
  return launch_k(experts_few_kernel<OUT, NT, WARPS>, dim3(unsigned(chunks * pl.nt)),
                  dim3(32 * WARPS), smem, st, a, pl);
}

// Rows of a chunk: eight where experts have two or fewer on average.
int rows_of(const ExpertsArgs& a) { return a.pairs <= 2LL * a.experts ? 8 : 16; }

template <ExpertsOut OUT, int NT>
cudaError_t of_rows(const ExpertsArgs& a, cudaStream_t st) {
  if constexpr (OUT == OUT_CODES)
    if (warps_of(a) == 16) return go<OUT, NT, 16>(a, st);
  return go<OUT, NT, 8>(a, st);
}
template <ExpertsOut OUT>
cudaError_t few(const ExpertsArgs& a, cudaStream_t st) {
  return rows_of(a) == 8 ? of_rows<OUT, 1>(a, st) : of_rows<OUT, 2>(a, st);
}

}  // namespace

bool experts_few(const ExpertsArgs& a) {
  // few rows of each expert that can have one, a CTA or less for each SM, rows of x that
  // shared memory holds (48 rows by 6 of 64 experts, 1152 x 1152, 576 CTAs: 28 us,
  // where experts_linear.cu takes 18)
  const long long used = a.pairs < a.experts ? a.pairs : a.experts;
  return a.pairs <= 8 * used && chunks_of(a, rows_of(a)) * ((a.n - 1) / 128 + 1) <= SMS &&
         smem_of(a, rows_of(a), warps_of(a)) <= MOST_SMEM;
}

cudaError_t launch_experts_few(const ExpertsArgs& a, cudaStream_t st) {
  if (a.y8.codes) return few<OUT_CODES>(a, st);
  return a.f32 ? few<OUT_F32>(a, st) : few<OUT_BF16>(a, st);
}

}  // namespace rc
