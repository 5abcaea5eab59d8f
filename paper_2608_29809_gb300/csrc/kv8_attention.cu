// Attention over the paged eight-bit cache (rc_kv8): the choice of its kernel.
#include "common.cuh"
#include "kernels.h"

namespace rc {

cudaError_t launch_kv8_attention(const Kv8Pool& pool, const Kv8AttnArgs& a, cudaStream_t st) {
  if ((long long)a.max_q * (a.heads / pool.heads) <= 64) return launch_kv8_few(pool, a, st);
  return launch_kv8_many(pool, a, st);
}

}  // namespace rc
