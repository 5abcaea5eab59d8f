// C ABI of the rest of a block (see include/regioncache.h, rc_norm_residual,
// rc_rotary_*, rc_experts_*): host-side validation, the rotary plan and the
// launches.
#include "block.h"

#include <math.h>

#include "abi_checks.h"

using namespace rc::abi;

namespace {

bool is_finite(double v) { return v - v == 0; }

rc_status check_norm(const rc_norm& n, const char* fn, const char* name, rc::NormOf* out) {
  if (n.kind < RC_NORM_NONE || n.kind > RC_NORM_RMS)
    return fail(RC_ERR_INVALID_ARG, "%s: %s.kind %d", fn, name, n.kind);
  if (n.kind == RC_NORM_NONE) {
    if (n.weight || n.bias)
      return fail(RC_ERR_INVALID_ARG, "%s: %s has a weight or bias without a norm", fn, name);
  } else if (!(n.eps >= 0) || !is_finite(n.eps)) {
    return fail(RC_ERR_INVALID_ARG, "%s: %s.eps %g", fn, name, double(n.eps));
  }
  if (!aligned(n.weight, 4) || !aligned(n.bias, 4))
    return fail(RC_ERR_INVALID_ARG, "%s: %s has a pointer that is not 4-B aligned", fn, name);
  *out = rc::NormOf{n.kind, n.eps, n.weight, n.bias};
  return RC_OK;
}

// A matrix of rows of `cols` values: there, aligned to its type, rows apart.
rc_status check_rows(const void* p, int type, int ld, int cols, const char* fn, const char* name) {
  RC_CHECK(check_type(type, fn));
  if (ld < cols) return fail(RC_ERR_SHAPE, "%s: ld of %s %d below %d", fn, name, ld, cols);
  if (!aligned(p, type == RC_F32 ? 4 : 2))
    return fail(RC_ERR_INVALID_ARG, "%s: %s is not aligned to its type", fn, name);
  return RC_OK;
}

rc_status check_plan(const rc_rotary* p, const char* fn) {
  if (p->rot < 2 || p->rot > RC_ROTARY_MAX || p->rot % 2 || p->axes < 1 || p->axes > 3)
    return fail(RC_ERR_SHAPE, "%s: %d channels turned (even, 2 .. %d), %d axes (1 .. 3)", fn,
                p->rot, RC_ROTARY_MAX, p->axes);
  long long sum = 0;
  for (int a = 0; a < p->axes; ++a) {
    if (p->pairs[a] < 1) return fail(RC_ERR_SHAPE, "%s: axis %d has %d pairs", fn, a, p->pairs[a]);
    sum += p->pairs[a];
  }
  if (sum != p->rot / 2)
    return fail(RC_ERR_SHAPE, "%s: the axes have %lld pairs of %d", fn, sum, p->rot / 2);
  if (p->first < 0 || p->first > RC_ROTARY_MAX_HEAD - p->rot)
    return fail(RC_ERR_SHAPE, "%s: %d channels from %d on", fn, p->rot, p->first);
  if (p->layout != RC_ROTARY_HALF && p->layout != RC_ROTARY_PAIRS)
    return fail(RC_ERR_INVALID_ARG, "%s: layout %d", fn, p->layout);
  if (!is_finite(p->amplitude)) return fail(RC_ERR_INVALID_ARG, "%s: amplitude is not finite", fn);
  return RC_OK;
}

}  // namespace

extern "C" {

rc_status rc_norm_residual(rc_ctx* c, const rc_residual* op, rc_stream stream) {
  const char* fn = "rc_norm_residual";
  if (!c || !op) return fail(RC_ERR_INVALID_ARG, "%s: null argument", fn);
  if (op->rows < 0 || op->cols < 1 || op->cols > RC_NORM_MAX_COLS || op->n_items < 1 ||
      op->top_k < 0 || op->top_k > RC_EXPERTS_MAX_TOP_K)
    return fail(RC_ERR_SHAPE, "%s: %d rows of %d (at most %d), %d items, top_k %d (at most %d)", fn,
                op->rows, op->cols, RC_NORM_MAX_COLS, op->n_items, op->top_k,
                RC_EXPERTS_MAX_TOP_K);
  rc::ResidualArgs a = {};
  RC_CHECK(check_norm(op->post, fn, "post", &a.post));
  RC_CHECK(check_norm(op->pre, fn, "pre", &a.pre));
  if (!op->row_offsets && op->n_items != 1)
    return fail(RC_ERR_INVALID_ARG, "%s: %d items without row_offsets", fn, op->n_items);
  if (!op->x_out && !op->y && !op->y8)
    return fail(RC_ERR_INVALID_ARG, "%s: nothing to write", fn);
  if (op->y && op->y8) return fail(RC_ERR_INVALID_ARG, "%s: both y and y8", fn);
  if (op->x || op->x_out) RC_CHECK(check_type(op->x_type, fn));
  if (op->x) RC_CHECK(check_rows(op->x, op->x_type, op->ldx, op->cols, fn, "x"));
  if (op->x_out) RC_CHECK(check_rows(op->x_out, op->x_type, op->ldx_out, op->cols, fn, "x_out"));
  if (op->x_out && op->x_out == op->x && op->ldx_out != op->ldx)
    return fail(RC_ERR_SHAPE, "%s: x_out is x with another stride", fn);
  if (op->h) {
    RC_CHECK(check_rows(op->h, op->h_type, op->ldh, op->cols, fn, "h"));
    if (op->top_k > 0 && (!op->places || !op->weights))
      return fail(RC_ERR_INVALID_ARG, "%s: top_k %d without places or weights", fn, op->top_k);
    if (op->top_k > 0 && op->h_rows < 0)
      return fail(RC_ERR_SHAPE, "%s: h has %d rows", fn, op->h_rows);
  } else if (op->top_k > 0 || op->post.kind != RC_NORM_NONE || op->gate) {
    return fail(RC_ERR_INVALID_ARG, "%s: top_k, post or gate without h", fn);
  }
  if (op->y) RC_CHECK(check_rows(op->y, op->y_type, op->ldy, op->cols, fn, "y"));
  if (op->y8) {
    RC_CHECK(check_matrix(op->y8, fn, "y8", &a.y8));
    if (op->y8->group != 1 || op->y8->cols != op->cols || op->y8->rows < op->rows)
      return fail(RC_ERR_SHAPE, "%s: y8 is %d x %d in groups of %d for %d x %d", fn, op->y8->rows,
                  op->y8->cols, op->y8->group, op->rows, op->cols);
  }
  if ((op->gate || op->scale || op->shift) && op->n_items > 1 && op->ld_mod < op->cols)
    return fail(RC_ERR_SHAPE, "%s: ld_mod %d below %d", fn, op->ld_mod, op->cols);
  const void* words[] = {op->gate, op->scale, op->shift, op->row_offsets, op->places, op->weights};
  for (const void* p : words)
    if (!aligned(p, 4)) return fail(RC_ERR_INVALID_ARG, "%s: a pointer is not 4-B aligned", fn);
  if (!is_finite(op->residual_scale))
    return fail(RC_ERR_INVALID_ARG, "%s: residual_scale is not finite", fn);
  if (op->rows == 0) return RC_OK;
  RC_CHECK(check_device(c, fn));
  a.rows = op->rows, a.cols = op->cols, a.n_items = op->n_items, a.top_k = op->top_k;
  a.row_offsets = op->row_offsets;
  a.x = op->x, a.x_out = op->x_out, a.h = op->h;
  a.places = op->places, a.weights = op->weights;
  a.gate = op->gate, a.scale = op->scale, a.shift = op->shift;
  a.y = op->y;
  a.x_f32 = op->x_type == RC_F32, a.h_f32 = op->h_type == RC_F32, a.y_f32 = op->y_type == RC_F32;
  a.ldx = op->ldx, a.ldx_out = op->ldx_out, a.ldh = op->ldh, a.h_rows = op->h_rows;
  a.ld_mod = op->ld_mod, a.ldy = op->ldy;
  a.residual_scale = op->residual_scale;
  a.err = rc::ctx_error_word(c);
  return launched(rc::launch_norm_residual(a, static_cast<cudaStream_t>(stream)), fn);
}

rc_status rc_rotary_plan(const rc_rotary_spec* s, rc_rotary* out) {
  const char* fn = "rc_rotary_plan";
  if (!s || !out) return fail(RC_ERR_INVALID_ARG, "%s: null argument", fn);
  rc_rotary p = {};
  p.rot = s->rot, p.first = s->first, p.layout = s->layout, p.axes = s->axes;
  for (int a = 0; a < 3 && a < s->axes; ++a) p.pairs[a] = s->pairs[a];
  p.amplitude = float(s->amplitude);
  RC_CHECK(check_plan(&p, fn));
  if (s->scaling < RC_ROTARY_PLAIN || s->scaling > RC_ROTARY_RAMP)
    return fail(RC_ERR_INVALID_ARG, "%s: scaling %d", fn, s->scaling);
  if (!(s->theta > 0) || !is_finite(s->theta))
    return fail(RC_ERR_INVALID_ARG, "%s: theta %g", fn, s->theta);
  if (s->scaling != RC_ROTARY_PLAIN && (!(s->factor >= 1) || !is_finite(s->factor)))
    return fail(RC_ERR_INVALID_ARG, "%s: factor %g", fn, s->factor);
  const bool bands = s->scaling == RC_ROTARY_BANDS, ramp = s->scaling == RC_ROTARY_RAMP;
  if ((bands || ramp) && (!(s->native_length > 0) || !is_finite(s->native_length) ||
                          !(s->slow > 0) || !(s->fast > s->slow) || !is_finite(s->fast)))
    return fail(RC_ERR_INVALID_ARG, "%s: native_length %g, fast %g, slow %g", fn, s->native_length,
                s->fast, s->slow);
  if (ramp && !(s->theta > 1))
    return fail(RC_ERR_INVALID_ARG, "%s: theta %g (RC_ROTARY_RAMP: above 1)", fn, s->theta);
  const double two_pi = 6.283185307179586;
  int at = 0;
  for (int a = 0; a < p.axes; ++a) {
    const int n = p.pairs[a];
    const double theta = s->scaling == RC_ROTARY_BASE && n > 1
                             ? s->theta * pow(s->factor, double(n) / (n - 1)) : s->theta;
    double lo = 0, hi = 0;
    if (ramp) {
      lo = floor(n * log(s->native_length / (s->fast * two_pi)) / log(theta));
      hi = ceil(n * log(s->native_length / (s->slow * two_pi)) / log(theta));
      lo = fmax(lo, 0);
      // (of one axis as YaRN's ramp, which may run out behind the last pair; an axis of several,
      // for which there is no published ramp, ends with its own last pair)
      hi = fmin(hi, p.axes == 1 ? p.rot - 1 : n - 1);
    }
    for (int i = 0; i < n; ++i) {
      double f = pow(theta, -double(i) / n), k = 1;
      if (s->scaling == RC_ROTARY_LINEAR) k = 0;
      if (bands) k = (s->native_length * f / two_pi - s->slow) / (s->fast - s->slow);
      if (ramp) k = 1 - (i - lo) / fmax(hi - lo, 0.001);
      k = fmin(fmax(k, 0), 1);
      if (k < 1) f = k * f + (1 - k) * f / s->factor;
      const double turns = f / two_pi;
      if (!is_finite(turns))
        return fail(RC_ERR_INVALID_ARG, "%s: theta %g makes an infinite frequency", fn, s->theta);
      p.turns[at++] = uint64_t(ldexp(turns - floor(turns), 64));
    }
  }
  *out = p;
  return RC_OK;
}

rc_status rc_rotary_apply(rc_ctx* c, const rc_rotary* plan, const void* x, int ldx, int type,
                          int rows, int heads, int head_dim, const int32_t* positions,
                          const int32_t* count, int inverse, void* y, int ldy, rc_stream stream) {
  const char* fn = "rc_rotary_apply";
  if (!c || !plan) return fail(RC_ERR_INVALID_ARG, "%s: null argument", fn);
  RC_CHECK(check_plan(plan, fn));
  RC_CHECK(check_type(type, fn));
  if (rows < 0 || heads < 0 || head_dim < plan->first + plan->rot ||
      head_dim > RC_ROTARY_MAX_HEAD || (long long)heads * head_dim > 0x7fffffff)
    return fail(RC_ERR_SHAPE, "%s: %d rows, %d heads of %d (%d .. %d)", fn, rows, heads, head_dim,
                plan->first + plan->rot, RC_ROTARY_MAX_HEAD);
  if (rows == 0 || heads == 0) return RC_OK;
  if (!x || !y) return fail(RC_ERR_INVALID_ARG, "%s: null argument", fn);
  RC_CHECK(check_rows(x, type, ldx, heads * head_dim, fn, "x"));
  RC_CHECK(check_rows(y, type, ldy, heads * head_dim, fn, "y"));
  if (x == y && ldx != ldy) return fail(RC_ERR_SHAPE, "%s: y is x with another stride", fn);
  if (!aligned(positions, 4) || !aligned(count, 4))
    return fail(RC_ERR_INVALID_ARG, "%s: a pointer is not 4-B aligned", fn);
  RC_CHECK(check_device(c, fn));
  rc::RotaryArgs a = {};
  a.plan = *plan;
  for (int i = plan->axes; i < 3; ++i) a.plan.pairs[i] = 0;  // (whatever a caller left there)
  a.x = x, a.y = y, a.ldx = ldx, a.ldy = ldy;
  a.rows = rows, a.heads = heads, a.head_dim = head_dim, a.f32 = type == RC_F32;
  a.positions = positions, a.count = count, a.inverse = inverse != 0;
  a.err = rc::ctx_error_word(c);
  return launched(rc::launch_rotary(a, static_cast<cudaStream_t>(stream)), fn);
}

rc_status rc_experts_route(rc_ctx* c, const rc_routing* r, const void* logits, int ld, int type,
                           int rows, const int32_t* count, int32_t* ids, float* weights,
                           rc_stream stream) {
  const char* fn = "rc_experts_route";
  if (!c || !r) return fail(RC_ERR_INVALID_ARG, "%s: null argument", fn);
  RC_CHECK(check_type(type, fn));
  if (rows < 0 || r->experts < 1 || r->experts > RC_EXPERTS_MAX || r->top_k < 1 ||
      r->top_k > RC_EXPERTS_MAX_TOP_K || ld < r->experts)
    return fail(RC_ERR_SHAPE, "%s: %d rows, %d experts (at most %d), top_k %d (at most %d), ld %d",
                fn, rows, r->experts, RC_EXPERTS_MAX, r->top_k, RC_EXPERTS_MAX_TOP_K, ld);
  if (r->groups < 1 || r->groups > 32 || r->experts % r->groups || r->top_groups < 1 ||
      r->top_groups > r->groups)
    return fail(RC_ERR_SHAPE, "%s: %d of %d groups (at most 32) of %d experts", fn, r->top_groups,
                r->groups, r->experts);
  if (r->group_best != 1 && r->group_best != 2)
    return fail(RC_ERR_INVALID_ARG, "%s: group_best %d is not 1 or 2", fn, r->group_best);
  if (r->score != RC_SCORE_SOFTMAX && r->score != RC_SCORE_SIGMOID)
    return fail(RC_ERR_INVALID_ARG, "%s: score %d", fn, r->score);
  if (!is_finite(r->scale)) return fail(RC_ERR_INVALID_ARG, "%s: scale is not finite", fn);
  if (!aligned(logits, type == RC_F32 ? 4 : 2) || !aligned(r->bias, 4) || !aligned(count, 4) ||
      !aligned(ids, 4) || !aligned(weights, 4))
    return fail(RC_ERR_INVALID_ARG, "%s: a pointer is not aligned to its type", fn);
  if (rows == 0) return RC_OK;
  if (!logits || !ids || !weights) return fail(RC_ERR_INVALID_ARG, "%s: null argument", fn);
  RC_CHECK(check_device(c, fn));
  const rc::RoutingArgs a{logits, type == RC_F32, ld, rows, r->experts, r->top_k, r->score,
                          r->groups, r->top_groups, r->group_best, r->renormalise != 0, r->scale,
                          r->bias, count, ids, weights, rc::ctx_error_word(c)};
  return launched(rc::launch_experts_route(a, static_cast<cudaStream_t>(stream)), fn);
}

rc_status rc_experts_sort(rc_ctx* c, const int32_t* ids, int rows, int top_k, int experts,
                          const int32_t* count, int32_t* offsets, int32_t* source, int32_t* places,
                          rc_stream stream) {
  const char* fn = "rc_experts_sort";
  if (!c || !offsets) return fail(RC_ERR_INVALID_ARG, "%s: null argument", fn);
  if (rows < 0 || top_k < 1 || top_k > RC_EXPERTS_MAX_TOP_K || experts < 1 ||
      experts > RC_EXPERTS_MAX || (long long)rows * top_k > RC_EXPERTS_MAX_PAIRS)
    return fail(RC_ERR_SHAPE, "%s: %d rows of %d (at most %d) of %d experts (at most %d)", fn, rows,
                top_k, RC_EXPERTS_MAX_TOP_K, experts, RC_EXPERTS_MAX);
  if (rows > 0 && (!ids || !source || !places))
    return fail(RC_ERR_INVALID_ARG, "%s: null argument", fn);
  const void* ints[] = {ids, count, offsets, source, places};
  for (const void* p : ints)
    if (!aligned(p, 4)) return fail(RC_ERR_INVALID_ARG, "%s: a pointer is not 4-B aligned", fn);
  RC_CHECK(check_device(c, fn));
  const rc::SortArgs a{ids, rows, top_k, experts, count, offsets, source, places,
                       rc::ctx_error_word(c)};
  return launched(rc::launch_experts_sort(a, static_cast<cudaStream_t>(stream)), fn);
}

rc_status rc_experts_linear(rc_ctx* c, const rc_fp8* x, const rc_fp8* W, const float* b,
                            int experts, int n, const int32_t* offsets, const int32_t* source,
                            int pairs, int act, void* y, int ldy, int type, const rc_fp8* y8,
                            rc_stream stream) {
  const char* fn = "rc_experts_linear";
  if (!c || !x || !W) return fail(RC_ERR_INVALID_ARG, "%s: null argument", fn);
  rc::ExpertsArgs a = {};
  RC_CHECK(check_matrix(x, fn, "x", &a.x));
  RC_CHECK(check_matrix(W, fn, "W", &a.w));
  if (x->group != 1 || W->group != 128)
    return fail(RC_ERR_INVALID_ARG, "%s: groups of x and W are %d and %d (1 and 128)", fn, x->group,
                W->group);
  if (act < RC_ACT_NONE || act > RC_ACT_GATED_SILU)
    return fail(RC_ERR_INVALID_ARG, "%s: act %d", fn, act);
  if (experts < 1 || experts > RC_EXPERTS_MAX || n < 1 || pairs < 0 ||
      pairs > RC_EXPERTS_MAX_PAIRS ||
      (pairs / 128LL + experts) * (n / 32LL + 1) >= 0x7fffffffLL - 152)
    return fail(RC_ERR_SHAPE, "%s: %d experts (at most %d) of %d outputs, %d pairs", fn, experts,
                RC_EXPERTS_MAX, n, pairs);
  const long long wide = act == RC_ACT_GATED_SILU ? 2LL * n : n;
  if (x->cols != W->cols || W->rows < 1 || W->rows % (experts * 128) || W->rows / experts < wide)
    return fail(RC_ERR_SHAPE,
                "%s: x has %d columns, W is %d x %d for %d experts of %lld rows (in 128s each)", fn,
                x->cols, W->rows, W->cols, experts, wide);
  if (pairs > 0 && x->rows < (source ? 1 : pairs))
    return fail(RC_ERR_SHAPE, "%s: x has %d rows for %d pairs", fn, x->rows, pairs);
  if (y && y8) return fail(RC_ERR_INVALID_ARG, "%s: both y and y8", fn);
  if (y8) {
    RC_CHECK(check_matrix(y8, fn, "y8", &a.y8));
    if (y8->group != 1 || y8->cols != n || y8->rows < pairs)
      return fail(RC_ERR_SHAPE, "%s: y8 is %d x %d in groups of %d for %d x %d", fn, y8->rows,
                  y8->cols, y8->group, pairs, n);
  } else {
    RC_CHECK(check_rows(y, type, ldy, n, fn, "y"));
  }
  if (pairs == 0) return RC_OK;
  if (!offsets || (!y && !y8)) return fail(RC_ERR_INVALID_ARG, "%s: null argument", fn);
  if (!aligned(b, 4) || !aligned(offsets, 4) || !aligned(source, 4))
    return fail(RC_ERR_INVALID_ARG, "%s: a pointer is not 4-B aligned", fn);
  RC_CHECK(check_device(c, fn));
  a.bias = b;
  a.experts = experts, a.n = n, a.offsets = offsets, a.source = source, a.pairs = pairs;
  a.act = act;
  a.y = y, a.ldy = ldy, a.f32 = type == RC_F32;
  a.err = rc::ctx_error_word(c);
  return launched(rc::launch_experts_linear(a, static_cast<cudaStream_t>(stream)), fn);
}

}  // extern "C"
