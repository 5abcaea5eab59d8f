// Attention over the paged eight-bit cache (rc_kv8): the choice of its kernel.
#include "common.cuh"
#include "kernels.h"

namespace rc {

cudaError_t launch_kv8_attention(const Kv8Pool& pool, const Kv8AttnArgs& a, cudaStream_t st) {
  // Sixteen rows of a key head read the cache once in the kernel for few rows;
  // more of them only where the GPU is not full with that (16 heads of 72, 4096
  // tokens: 8 requests of 16 rows 28.7 us, of 17 57.5, in the kernel for many
  // 41; one request of 64 rows 16.2 and 15.8)
  const long long rows = (long long)a.max_q * (a.heads / pool.heads);
  const long long units = (rows + 15) / 16 * pool.heads * a.n;
  if (rows <= 16 || (rows <= 64 && units <= 76)) return launch_kv8_few(pool, a, st);
  return launch_kv8_many(pool, a, st);
}

}  // namespace rc
