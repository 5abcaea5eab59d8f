// Internal launchers of a block's row work, rotary positions and experts
// (rc_norm_residual, rc_rotary_*, rc_experts_*).  Every launcher queues one
// kernel on `st` and returns the cudaError_t of the launch.
#pragma once
#include "../../include/regioncache.h"
#include "eight_bit.h"

namespace rc {

struct NormOf {
  int kind;  // RC_NORM_*
  float eps;
  const float *weight, *bias;
};
// As rc_residual; y8.codes null for none.
struct ResidualArgs {
  int rows, cols, n_items, top_k;
  const int* row_offsets;
  const void* x;
  void* x_out;
  const void* h;
  const int* places;
  const float *weights, *gate, *scale, *shift;
  void* y;
  Fp8Mat y8;
  bool x_f32, h_f32, y_f32;
  int ldx, ldx_out, ldh, h_rows, ld_mod, ldy;
  float residual_scale;
  NormOf post, pre;
  unsigned* err;
};
cudaError_t launch_norm_residual(const ResidualArgs& a, cudaStream_t st);

struct RotaryArgs {
  ::rc_rotary plan;
  const void* x;
  void* y;
  int ldx, ldy, rows, heads, head_dim;
  bool f32;
  const int *positions, *count;
  int inverse, per;  // per: rows of a CTA, set by the launcher
  unsigned* err;
};
cudaError_t launch_rotary(const RotaryArgs& a, cudaStream_t st);

struct RoutingArgs {
  const void* logits;
  bool f32;
  int ld, rows, experts, top_k, score, groups, top_groups, group_best, renormalise;
  float scale;
  const float* bias;
  const int* count;
  int* ids;
  float* weights;
  unsigned* err;
};
cudaError_t launch_experts_route(const RoutingArgs& a, cudaStream_t st);
struct SortArgs {
  const int* ids;
  int rows, top_k, experts;
  const int* count;
  int *offsets, *source, *places;
  unsigned* err;
};
cudaError_t launch_experts_sort(const SortArgs& a, cudaStream_t st);
// w: the experts' matrices one below the other; y8.codes null for none.
struct ExpertsArgs {
  Fp8Mat x, w;
  const float* bias;
  int experts, n;
  const int *offsets, *source;
  int pairs, act;
  void* y;
  int ldy;
  bool f32, tma;  // tma: y's rows are 16-byte aligned, set by the launcher
  Fp8Mat y8;
  unsigned* err;
};
cudaError_t launch_experts_linear(const ExpertsArgs& a, cudaStream_t st);
// The same for few experts of a few rows each, and whether a call is of those.
bool experts_few(const ExpertsArgs& a);
cudaError_t launch_experts_few(const ExpertsArgs& a, cudaStream_t st);

}  // namespace rc
