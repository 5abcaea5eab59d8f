// Internal launchers of eight-bit serving (rc_fp8_*, rc_kv8_*).  Every launcher
// queues one kernel on `st` (the attention two, for batches of many short and a few
// long requests) and returns the cudaError_t of the launch.
#pragma once
#include "kernels.h"

namespace rc {

// Of a context, for host code outside regioncache.cu.
unsigned* ctx_error_word(const ::rc_ctx* c);
int ctx_device(const ::rc_ctx* c);

// Quantised matrix (rc_fp8): codes [rows][ld], scales [ceil(cols / 128)][lds].
struct Fp8Mat {
  uint8_t* codes;
  uint8_t* scales;
  int rows, cols, ld, lds, group;
};
cudaError_t launch_fp8_quantize(const void* x, int ldx, bool f32, const Fp8Mat& out,
                                cudaStream_t st);
// y = x w^T + b, y f32 or bf16 [x.rows][ldy].
cudaError_t launch_fp8_linear(const Fp8Mat& x, const Fp8Mat& w, const float* b, void* y, int ldy,
                              bool f32, unsigned* err, cudaStream_t st);

// Paged eight-bit cache (rc_kv8): side 0 the keys, 1 the values.
constexpr int KV8_BLOCK = 64;
constexpr int KV8_MAX_REQUESTS = 4096;
struct Kv8Pool {
  uint8_t* code[2];   // [blocks][heads][KV8_BLOCK][dh]
  uint8_t* scale[2];  // [blocks][heads]
  int blocks, heads, dh;
};
struct Kv8TablesArgs {
  const int *lengths, *counts, *positions, *free_blocks;
  int n, n_free, ld_table, n_slots;
  int *table, *offsets, *slots, *used;
  unsigned* err;
};
cudaError_t launch_kv8_tables(const Kv8TablesArgs& a, cudaStream_t st);
// `rows` [n][ld] of keys and of values to their slots; *count of them (null: n).
cudaError_t launch_kv8_store(const Kv8Pool& pool, const void* k, const void* v, int ld, bool f32,
                             const int* slots, int n, const int* count, bool append,
                             unsigned* err, cudaStream_t st);
struct Kv8AttnArgs {
  const bf16* q;
  bf16* o;
  int ldq, ldo, q_rows, n, max_q, ld_table, heads, causal;
  const int *offsets, *lengths, *table;
  unsigned* err;
  // requests of other numbers of rows (query, head of a key head's group) are
  // left to another launch
  int least_rows, most_rows;
};
cudaError_t launch_kv8_attention(const Kv8Pool& pool, const Kv8AttnArgs& a, cudaStream_t st);
// The same for requests of a few rows each (every sixteen read the cache).
cudaError_t launch_kv8_few(const Kv8Pool& pool, const Kv8AttnArgs& a, cudaStream_t st);
// And for requests of many rows (the tensor memory path).
cudaError_t launch_kv8_many(const Kv8Pool& pool, const Kv8AttnArgs& a, cudaStream_t st);

}  // namespace rc
