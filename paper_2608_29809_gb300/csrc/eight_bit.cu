// C ABI of eight-bit serving (see include/regioncache.h, rc_fp8_* and
// rc_kv8_*): host-side validation and the launches.
#include "abi_checks.h"

static_assert(RC_KV8_BLOCK == rc::KV8_BLOCK && RC_KV8_MAX_REQUESTS == rc::KV8_MAX_REQUESTS,
              "the header's limits are the kernels'");

using namespace rc::abi;

namespace {

rc_status check_pool(const rc_kv8* p, const char* fn, rc::Kv8Pool* out) {
  if (!p->k || !p->v || !p->k_scale || !p->v_scale)
    return fail(RC_ERR_INVALID_ARG, "%s: the pool has a null pointer", fn);
  if (!aligned(p->k, 16) || !aligned(p->v, 16))
    return fail(RC_ERR_INVALID_ARG, "%s: the pool's codes must be 16-B aligned", fn);
  if (p->blocks < 1 || (long long)p->blocks * RC_KV8_BLOCK > 0x7fffffffLL || p->kv_heads < 1 ||
      p->kv_heads > 1024 || (p->head_dim != 64 && p->head_dim != 72 && p->head_dim != 128))
    return fail(RC_ERR_SHAPE, "%s: a pool of %d blocks, %d heads of %d (64, 72 or 128)", fn,
                p->blocks, p->kv_heads, p->head_dim);
  *out = rc::Kv8Pool{{static_cast<uint8_t*>(p->k), static_cast<uint8_t*>(p->v)},
                     {static_cast<uint8_t*>(p->k_scale), static_cast<uint8_t*>(p->v_scale)},
                     p->blocks, p->kv_heads, p->head_dim};
  return RC_OK;
}

}  // namespace

extern "C" {

rc_status rc_fp8_quantize(rc_ctx* c, const void* x, int ldx, int type, const rc_fp8* out,
                          rc_stream stream) {
  const char* fn = "rc_fp8_quantize";
  if (!c || !out) return fail(RC_ERR_INVALID_ARG, "%s: null argument", fn);
  rc::Fp8Mat m;
  RC_CHECK(check_type(type, fn));
  RC_CHECK(check_matrix(out, fn, "out", &m));
  if (ldx < m.cols) return fail(RC_ERR_SHAPE, "%s: ldx %d below %d columns", fn, ldx, m.cols);
  if (m.rows == 0) return RC_OK;
  if (!x) return fail(RC_ERR_INVALID_ARG, "%s: null argument", fn);
  if (!aligned(x, type == RC_F32 ? 4 : 2))
    return fail(RC_ERR_INVALID_ARG, "%s: x is not aligned to its type", fn);
  RC_CHECK(check_device(c, fn));
  return launched(rc::launch_fp8_quantize(x, ldx, type == RC_F32, m,
                                          static_cast<cudaStream_t>(stream)), fn);
}

rc_status rc_fp8_linear(rc_ctx* c, const rc_fp8* x, const rc_fp8* W, const float* b, void* y,
                        int ldy, int type, rc_stream stream) {
  const char* fn = "rc_fp8_linear";
  if (!c || !x || !W) return fail(RC_ERR_INVALID_ARG, "%s: null argument", fn);
  rc::Fp8Mat mx, mw;
  RC_CHECK(check_type(type, fn));
  RC_CHECK(check_matrix(x, fn, "x", &mx));
  RC_CHECK(check_matrix(W, fn, "W", &mw));
  if (mx.cols != mw.cols || mw.rows < 1 || ldy < mw.rows)
    return fail(RC_ERR_SHAPE, "%s: x has %d columns, W is %d x %d, ldy %d", fn, mx.cols, mw.rows,
                mw.cols, ldy);
  if (mx.rows == 0) return RC_OK;
  if (!y) return fail(RC_ERR_INVALID_ARG, "%s: null argument", fn);
  if (!aligned(y, type == RC_F32 ? 4 : 2) || !aligned(b, 4))
    return fail(RC_ERR_INVALID_ARG, "%s: y or b is not aligned to its type", fn);
  RC_CHECK(check_device(c, fn));
  return launched(rc::launch_fp8_linear(mx, mw, b, y, ldy, type == RC_F32,
                                        rc::ctx_error_word(c), static_cast<cudaStream_t>(stream)), fn);
}

rc_status rc_kv8_tables(rc_ctx* c, const int32_t* lengths, const int32_t* counts,
                        const int32_t* positions, int n, const int32_t* free_blocks, int n_free,
                        int32_t* table, int ld_table, int32_t* row_offsets, int32_t* slots,
                        int n_slots, int32_t* used, rc_stream stream) {
  const char* fn = "rc_kv8_tables";
  if (!c || !lengths || !table || !row_offsets || !used || (n_slots > 0 && !slots))
    return fail(RC_ERR_INVALID_ARG, "%s: null argument", fn);
  if (n < 1 || n > RC_KV8_MAX_REQUESTS || n_free < 0 || n_free > 0x7fffffff / RC_KV8_BLOCK ||
      ld_table < 1 || ld_table > 0x7fffffff / RC_KV8_BLOCK || n_slots < 0 || n_slots > 1 << 30)
    return fail(RC_ERR_SHAPE, "%s: %d requests (at most %d), %d free blocks, ld_table %d, %d slots",
                fn, n, RC_KV8_MAX_REQUESTS, n_free, ld_table, n_slots);
  const void* ints[] = {lengths, counts, positions, free_blocks, table, row_offsets, slots, used};
  for (const void* p : ints)
    if (!aligned(p, 4)) return fail(RC_ERR_INVALID_ARG, "%s: pointers must be 4-B aligned", fn);
  RC_CHECK(check_device(c, fn));
  const rc::Kv8TablesArgs a{lengths, counts, positions, free_blocks, n, n_free, ld_table, n_slots,
                            table, row_offsets, slots, used, rc::ctx_error_word(c)};
  return launched(rc::launch_kv8_tables(a, static_cast<cudaStream_t>(stream)), fn);
}

rc_status rc_kv8_store(rc_ctx* c, const rc_kv8* pool, const void* k, const void* v, int ldkv,
                       int type, const int32_t* slots, int n, const int32_t* count, int mode,
                       rc_stream stream) {
  const char* fn = "rc_kv8_store";
  if (!c || !pool) return fail(RC_ERR_INVALID_ARG, "%s: null argument", fn);
  rc::Kv8Pool p;
  RC_CHECK(check_type(type, fn));
  RC_CHECK(check_pool(pool, fn, &p));
  if (mode != RC_KV8_UPDATE && mode != RC_KV8_APPEND)
    return fail(RC_ERR_INVALID_ARG, "%s: mode %d", fn, mode);
  if (n < 0 || ldkv < p.heads * p.dh)
    return fail(RC_ERR_SHAPE, "%s: %d rows, ldkv %d below %d", fn, n, ldkv, p.heads * p.dh);
  if (n == 0) return RC_OK;
  if (!k || !v || !slots) return fail(RC_ERR_INVALID_ARG, "%s: null argument", fn);
  const unsigned size = type == RC_F32 ? 4 : 2;
  if (!aligned(k, size) || !aligned(v, size) || !aligned(slots, 4) || !aligned(count, 4))
    return fail(RC_ERR_INVALID_ARG, "%s: a pointer is not aligned to its type", fn);
  RC_CHECK(check_device(c, fn));
  return launched(rc::launch_kv8_store(p, k, v, ldkv, type == RC_F32, slots, n, count,
                                       mode == RC_KV8_APPEND, rc::ctx_error_word(c),
                                       static_cast<cudaStream_t>(stream)), fn);
}

rc_status rc_kv8_attention(rc_ctx* c, const rc_kv8* pool, const void* Q, int ldq, int q_rows,
                           const int32_t* row_offsets, const int32_t* lengths, int n, int max_q,
                           const int32_t* table, int ld_table, int heads, int causal, void* O,
                           int ldo, rc_stream stream) {
  const char* fn = "rc_kv8_attention";
  if (!c || !pool) return fail(RC_ERR_INVALID_ARG, "%s: null argument", fn);
  rc::Kv8Pool p;
  RC_CHECK(check_pool(pool, fn, &p));
  if (heads < 1 || heads > 1024 || heads % p.heads || heads / p.heads > 16)
    return fail(RC_ERR_SHAPE, "%s: %d heads over %d key heads (at most 16 each)", fn, heads,
                p.heads);
  if (q_rows < 0 || max_q < 0 || n < 0 || n > RC_KV8_MAX_REQUESTS || ld_table < 1 ||
      ld_table > 0x7fffffff / RC_KV8_BLOCK || ldq < heads * p.dh || ldo < heads * p.dh ||
      ldq % 8 || ldo % 8)
    return fail(RC_ERR_SHAPE,
                "%s: %d rows, max_q %d, %d requests (at most %d), ld_table %d, ldq %d, ldo %d "
                "(multiples of 8, >= %d)", fn, q_rows, max_q, n, RC_KV8_MAX_REQUESTS, ld_table,
                ldq, ldo, heads * p.dh);
  if ((long long)q_rows * (heads / p.heads) > 0x7fffffffLL)
    return fail(RC_ERR_SHAPE, "%s: %d rows of %d heads a key head", fn, q_rows, heads / p.heads);
  if (q_rows == 0 || max_q == 0 || n == 0) return RC_OK;
  if (!Q || !O || !row_offsets || !lengths || !table)
    return fail(RC_ERR_INVALID_ARG, "%s: null argument", fn);
  if (!aligned(Q, 16) || !aligned(O, 16) || !aligned(row_offsets, 4) || !aligned(lengths, 4) ||
      !aligned(table, 4))
    return fail(RC_ERR_INVALID_ARG, "%s: Q and O must be 16-B aligned, the rest 4-B", fn);
  RC_CHECK(check_device(c, fn));
  const rc::Kv8AttnArgs a{static_cast<const rc::bf16*>(Q), static_cast<rc::bf16*>(O), ldq, ldo,
                          q_rows, n, max_q < q_rows ? max_q : q_rows, ld_table, heads,
                          causal ? 1 : 0, row_offsets, lengths, table, rc::ctx_error_word(c), 1,
                          0x7fffffff};
  return launched(rc::launch_kv8_attention(p, a, static_cast<cudaStream_t>(stream)), fn);
}

}  // extern "C"
