// Attention over the paged eight-bit cache (rc_kv8): the choice of its kernel.
#include "common.cuh"
#include "eight_bit.h"

namespace rc {

// Sixteen rows (query, head of a key head's group) read the cache once in the
// kernel for few rows; more of them only where the GPU is not full with that
// (16 heads of 72, 4096 tokens: 8 requests of 16 rows 26 us, of 17 57, in the
// kernel for many 40; one request of 64 rows 15.2 and 15.8).  A batch of
// more key heads than two waves of CTAs whose mean request has less than a
// third of the rows that the largest may have is taken for one of many short
// requests and a few long ones, and the short ones get a launch of their own
// (32 requests of 2000 tokens, 24 of one row and 8 of 300: 95 us, in one launch
// 111; 8 of 4096, 7 of one row and one of 831: 82 and 66).
cudaError_t launch_kv8_attention(const Kv8Pool& pool, const Kv8AttnArgs& args, cudaStream_t st) {
  Kv8AttnArgs a = args;
  a.least_rows = 1;
  a.most_rows = 0x7fffffff;
  const int group = a.heads / pool.heads;
  const long long rows = (long long)a.max_q * group;
  const long long units = (rows + 15) / 16 * pool.heads * a.n;
  if (rows <= 16 || (rows <= 64 && units <= 76)) return launch_kv8_few(pool, a, st);
  if ((long long)a.n * pool.heads >= 2 * 152 && 3LL * a.q_rows < (long long)a.n * a.max_q) {
    a.most_rows = 16;
    const cudaError_t e = launch_kv8_few(pool, a, st);
    if (e != cudaSuccess) return e;
    a.least_rows = 17;
    a.most_rows = 0x7fffffff;
  }
  return launch_kv8_many(pool, a, st);
}

}  // namespace rc
