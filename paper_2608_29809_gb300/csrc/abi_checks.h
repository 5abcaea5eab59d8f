// What the entry points of the C ABI share: the error message, checks of
// arguments, the outcome of a launch (host code).
#pragma once
#include <stdarg.h>
#include <stdio.h>

#include "../../include/regioncache.h"
#include "eight_bit.h"

namespace rc {
namespace abi {

inline rc_status fail(rc_status s, const char* fmt, ...) {
  char buf[256];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof(buf), fmt, ap);
  va_end(ap);
  rc::set_last_error(buf);
  return s;
}

inline bool aligned(const void* p, unsigned n) {
  return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0;
}

// RC_OK, or the failure of a launch.
inline rc_status launched(cudaError_t e, const char* what) {
  if (e == cudaSuccess) return RC_OK;
  cudaGetLastError();  // (not left for a later call)
  return fail(RC_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e));
}

inline rc_status check_device(const rc_ctx* c, const char* fn) {
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess) {
    cudaGetLastError();
    return fail(RC_ERR_CUDA, "%s: no current device", fn);
  }
  if (dev != rc::ctx_device(c))
    return fail(RC_ERR_INVALID_ARG, "%s: device %d is current, the context's is %d", fn, dev,
                rc::ctx_device(c));
  return RC_OK;
}

// A quantised matrix as a kernel argument.
inline rc_status check_matrix(const rc_fp8* m, const char* fn, const char* name, rc::Fp8Mat* out) {
  if (m->rows < 0 || m->rows > RC_FP8_MAX_ROWS || m->cols < 1 || m->cols > RC_FP8_MAX_COLS)
    return fail(RC_ERR_SHAPE, "%s: %s is %d x %d (at most %d x %d)", fn, name, m->rows, m->cols,
                RC_FP8_MAX_ROWS, RC_FP8_MAX_COLS);
  if (m->group != 1 && m->group != 128)
    return fail(RC_ERR_INVALID_ARG, "%s: %s.group %d is not 1 or 128", fn, name, m->group);
  const long long scales = (m->rows + (long long)m->group - 1) / m->group;
  if (m->ld < m->cols || m->ld % 16 || m->lds < scales)
    return fail(RC_ERR_SHAPE, "%s: %s.ld %d (a multiple of 16, >= %d), lds %d (>= %lld)", fn, name,
                m->ld, m->cols, m->lds, scales);
  if (m->rows > 0 && (!m->codes || !m->scales))
    return fail(RC_ERR_INVALID_ARG, "%s: %s has a null pointer", fn, name);
  if (!aligned(m->codes, 16))
    return fail(RC_ERR_INVALID_ARG, "%s: %s.codes must be 16-B aligned", fn, name);
  *out = rc::Fp8Mat{static_cast<uint8_t*>(m->codes), static_cast<uint8_t*>(m->scales), m->rows,
                    m->cols, m->ld, m->lds, m->group};
  return RC_OK;
}

inline rc_status check_type(int type, const char* fn) {
  if (type == RC_BF16 || type == RC_F32) return RC_OK;
  return fail(RC_ERR_INVALID_ARG, "%s: type %d", fn, type);
}

#define RC_CHECK(call)                 \
  do {                                 \
    const rc_status s_ = (call);       \
    if (s_ != RC_OK) return s_;        \
  } while (0)

}  // namespace abi
}  // namespace rc
