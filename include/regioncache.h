/*
 * regioncache.h -- C ABI of the GB300 (sm_103a) region-sparse DiT step.
 *
 * The library implements the hot path of RegionCache (semantic-aware region
 * reuse for multi-turn image editing): a cross-attention localisation pass
 * turns the prompt-delta text tokens into a token-level dirty mask
 * (Section 3.2, R_edit); only dirty image tokens are recomputed through each
 * PixArt-alpha-shaped block, their queries attending over every token's
 * keys/values, where clean tokens' K/V and hidden states come from a
 * per-(layer, timestep) cache (Section 3.3, Region-Level Sparse Attention);
 * fresh K/V rows are written straight to their cache rows by the projection
 * GEMM (Section 3.4, Kernel Fusing); a step follows a per-step reuse
 * schedule given as input (Section 3.3, Eq. 2).
 *
 * Conventions for every entry point:
 *   - Return value: rc_status; RC_OK (0) on success.  No C++ exception ever
 *     crosses this boundary.  rc_last_error() gives a thread-local message
 *     for the last failing call on the calling thread.
 *   - Host arguments are validated before anything is launched; a failing
 *     validation launches nothing and changes no memory.
 *   - Pointers named *_host are host memory.  Every other tensor pointer is a
 *     device pointer owned by the caller, who keeps it alive and unmodified
 *     until the work queued on `stream` has finished.  Weights are borrowed
 *     for the lifetime of the rc_ctx.
 *   - Work is queued asynchronously on `stream` (a cudaStream_t; 0 is the
 *     legacy default stream).  Device-side argument errors (an index out of
 *     range, a count above its bound) are recorded in a library-owned error
 *     word and reported by rc_sync().
 *   - Dtypes: "bf16" = bfloat16 (2 bytes), "f32" = IEEE float.  Matrices are
 *     row-major.  Linear weights are [out][in]: y = x W^T + b.
 */
#ifndef REGIONCACHE_H
#define REGIONCACHE_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef int rc_status;
#define RC_OK 0
#define RC_ERR_INVALID_ARG 1   /* null pointer, value out of range           */
#define RC_ERR_SHAPE 2         /* sizes inconsistent with the rc_dims         */
#define RC_ERR_OOM 3           /* device allocation failed                    */
#define RC_ERR_CUDA 4          /* a CUDA runtime call failed                  */
#define RC_ERR_TIMEOUT 5       /* a bounded device wait gave up               */
#define RC_ERR_DEVICE_ASSERT 6 /* a kernel found a bad index / count          */
#define RC_ERR_STATE 7         /* call order violated (e.g. no weights set)   */
#define RC_ERR_IO 8            /* a file could not be opened, read or written */

/* Per-step modes of a reuse schedule (Section 3.3, Eq. 2). */
#define RC_MODE_DENSE 0  /* every token recomputed; cache rows overwritten    */
#define RC_MODE_SPARSE 1 /* only the dirty tokens recomputed                  */
#define RC_MODE_REUSE 2  /* no block runs; the last hidden state is cached    */

typedef void* rc_stream; /* cudaStream_t */

/* Model and problem sizes.  PixArt-alpha: hidden 1152, heads 16 (head_dim
 * 72), mlp 4608, layers 28, patch 2, in_ch 4, out_ch 8, text_len 120,
 * freq_dim 256.  N = grid_h * grid_w image tokens.  max_batch = most items
 * of one rc_step_batched call (1 .. RC_MAX_BATCH; 0 means 1): the context's
 * row scratch is sized for max_batch * N rows. */
#define RC_MAX_BATCH 16
typedef struct rc_dims {
  int hidden, heads, mlp, layers;
  int grid_h, grid_w, patch, in_ch, out_ch;
  int text_len, timesteps, freq_dim;
  int max_batch;
} rc_dims;

/* One block's weights (device pointers, borrowed).  W_* bf16 [out][in];
 * b_* f32 [out]; table f32 [6][hidden] = the adaLN-single scale-shift table
 * whose rows are (shift_msa, scale_msa, gate_msa, shift_mlp, scale_mlp,
 * gate_mlp).  W_qkv's outputs are q | k | v; W_xkv's are k | v. */
typedef struct rc_layer_weights {
  const void* W_qkv; const float* b_qkv;  /* [3h][h], [3h] */
  const void* W_o;   const float* b_o;    /* [h][h],  [h]  */
  const void* W_xq;  const float* b_xq;   /* [h][h],  [h]  */
  const void* W_xkv; const float* b_xkv;  /* [2h][h], [2h] */
  const void* W_xo;  const float* b_xo;   /* [h][h],  [h]  */
  const void* W_1;   const float* b_1;    /* [F][h],  [F]  */
  const void* W_2;   const float* b_2;    /* [h][F],  [h]  */
  const float* table;                     /* [6][h]        */
} rc_layer_weights;

/* Model-level weights (device pointers, borrowed).  W_e: patch embedding as a
 * linear map of the patch vector ordered (channel, py, px), bf16
 * [h][in_ch*p*p]; pos f32 [N][h] fixed positional table; timestep MLP
 * W_t1 [h][freq_dim], W_t2 [h][h]; adaLN-single W_tb [6h][h]; final layer
 * table_f f32 [2][h] (shift, scale), W_f bf16 [p*p*out_ch][h] with outputs
 * ordered (py, px, channel). */
typedef struct rc_global_weights {
  const void* W_e;  const float* b_e;  const float* pos;
  const void* W_t1; const float* b_t1;
  const void* W_t2; const float* b_t2;
  const void* W_tb; const float* b_tb;
  const float* table_f;
  const void* W_f;  const float* b_f;
} rc_global_weights;

typedef struct rc_ctx rc_ctx;     /* model + device scratch, one per stream user */
typedef struct rc_cache rc_cache; /* library-owned per-(session, t, layer) cache */

/* ---------------------------------------------------------------- context */

/* Creates a context on the current CUDA device and allocates its scratch
 * (sized for N tokens).  Errors: RC_ERR_INVALID_ARG (null, a dimension <= 0),
 * RC_ERR_SHAPE (hidden % heads != 0, head_dim not 72 or 64, hidden not a
 * multiple of 128 or above 1536, mlp not a multiple of 128, N > 16384,
 * in_ch * patch^2 > 16, out_ch < in_ch), RC_ERR_OOM.  Validation happens
 * before any CUDA call. */
rc_status rc_create(const rc_dims* dims, rc_ctx** out);
void rc_destroy(rc_ctx* ctx);

/* Registers (borrows) the weights of block `layer` / of the model.  The text
 * keys / values of every session (and the cross-query keys folded from them,
 * see rc_set_text) depend on a layer's W_xkv, b_xkv, W_xq and b_xq:
 * rc_set_layer_weights therefore marks the text of every session of every
 * cache of this context stale, and steps of a session return RC_ERR_STATE
 * until rc_set_text (or rc_cache_import) runs for it again. */
rc_status rc_set_layer_weights(rc_ctx* ctx, int layer, const rc_layer_weights* w);
/* The timestep embedding and t_block modulation of every scheduled timestep
 * depend only on W_t1 .. b_tb and the schedule: they are computed once, at
 * the first step or graph capture after rc_set_global_weights or
 * rc_set_schedule, and reused by every later step.  Weights changed in place
 * therefore need rc_set_global_weights again.  (A step captured by the
 * caller into a graph before they exist computes its own.) */
rc_status rc_set_global_weights(rc_ctx* ctx, const rc_global_weights* w);

/* Sampling schedule, copied: timestep values t_values_host[timesteps] fed to
 * the timestep embedding, and cumulative alphas alpha_bar_host[timesteps+1]
 * (entry timesteps is the value after the last step, normally 1) for the
 * DDIM (eta = 0) update after step t: alpha_bar[t] -> alpha_bar[t+1]. */
rc_status rc_set_schedule(rc_ctx* ctx, const float* t_values_host, const float* alpha_bar_host);

/* Reproducible sums.  By default the three gated-residual projections of a
 * block (x += g (y W^T + b) after attention, cross-attention and the MLP,
 * Section 3.3's region block) may split their reduction over k between
 * CTAs that add their partial products into x with atomic reductions, so a
 * step's result can differ in the last bits from run to run (always within
 * the documented tolerances).  With on != 0 every such GEMM runs on whole
 * output tiles (one reduction per element, k summed in a fixed order), and
 * rc_step, rc_step_batched, rc_step_dense, rc_block_forward_region and the
 * graphs captured from them give bit-identical results for bit-identical
 * inputs on the same GPU and build.  It costs about a tenth of the step
 * rate at 831 dirty tokens of 4096 (fewer CTAs share the residual GEMMs).
 * The score sums of rc_step_capture and rc_localize_scores (over heads, with
 * atomic adds) stay order-dependent either way.  Takes effect at the next
 * launch; graphs keep the schedule they were captured with.  Never fails
 * except on a null context. */
rc_status rc_set_deterministic(rc_ctx* ctx, int on);

/* ------------------------------------------------------------------ cache */

/* Cache pool of Section 3.2 (Hidden-State-Oriented Caching): for every
 * session s, timestep t and layer l, the block output H^{l+1}, keys K^l and
 * values V^l of all N tokens, bf16 [N][hidden] each, plus the per-session
 * text keys/values of every layer.  Library-owned device memory:
 * sessions * timesteps * layers * 3 * N * hidden * 2 bytes (15.85 GB for one
 * PixArt-alpha session at 4096 tokens and 20 steps). */
rc_status rc_cache_create(rc_ctx* ctx, int sessions, rc_cache** out);

/* The same pool in pinned, device-mapped host memory (Section 3.4, Pipelined
 * Execution): for pools larger than HBM.  The text keys/values and two HBM
 * windows of 3 * N * hidden bf16 stay on the device.  rc_step and
 * rc_step_capture on such a cache load each layer's cached K, V (plus H for the
 * last layer) into a window on a library-owned copy stream while the previous
 * layer computes, then write the dirty rows' H, K, V back to host memory; the
 * results equal those of a device-tier cache.  rc_step_batched takes one item
 * and rc_block_forward_region is refused (RC_ERR_INVALID_ARG).  Steps on one
 * host-tier cache must be issued from one host thread.  rc_cache_fill /
 * rc_cache_read work as for a device-tier cache.  Errors: RC_ERR_OOM when the
 * pinned allocation or a window fails. */
rc_status rc_cache_create_host(rc_ctx* ctx, int sessions, rc_cache** out);
void rc_cache_destroy(rc_cache* cache);

/* Copies caller bf16 [N][hidden] device buffers into / out of the (session,
 * layer, t) slot.  Any of H, K, V may be null to skip it. */
rc_status rc_cache_fill(rc_cache* cache, int session, int layer, int t,
                        const void* H, const void* K, const void* V, rc_stream stream);
rc_status rc_cache_read(rc_cache* cache, int session, int layer, int t,
                        void* H, void* K, void* V, rc_stream stream);

/* One session's whole cache to / from a file, so that an editing session
 * outlives the process (the paper keeps the pool in host memory between
 * turns, Section 3.4): every (t, layer) H, K, V slot and the text
 * keys/values, after a header with N, hidden, layers, timesteps and
 * text_len.  Synchronous (the device is synchronised first); the file is
 * raw little-endian bf16, about timesteps * layers * 3 * N * hidden * 2
 * bytes.  Import requires a header equal to the cache's dimensions
 * (RC_ERR_SHAPE otherwise) and marks the session's text as set when the
 * exported session had it; the folded text keys (see rc_set_text) are not
 * in the file but recomputed on import, so a session with text needs every
 * layer's weights set first (RC_ERR_STATE otherwise).  Errors:
 * RC_ERR_INVALID_ARG, RC_ERR_IO (open, short read / write, bad magic),
 * RC_ERR_SHAPE, RC_ERR_STATE, RC_ERR_CUDA.  An import that fails after the
 * header check has overwritten part of the session: its text is then marked
 * unset (steps return RC_ERR_STATE) until rc_set_text or a successful import. */
rc_status rc_cache_export(rc_cache* cache, int session, const char* path);
rc_status rc_cache_import(rc_cache* cache, int session, const char* path);

/* Text conditioning of one session for an editing turn: ctx_bf16 is the
 * text context, bf16 [text_len][hidden].  Computes every layer's
 * cross-attention keys/values (ctx W_xkv^T + b_xkv) into the session's
 * cache, and from them the keys with the cross-query projection folded in
 * (G_h = K_h W_xq,h, kb_h = K_h b_xq,h per head, device memory owned by the
 * cache) that sparse steps use instead of a separate query projection.
 * Must precede rc_step / rc_block_forward_region for the session. */
rc_status rc_set_text(rc_ctx* ctx, rc_cache* cache, int session, const void* ctx_bf16,
                      rc_stream stream);

/* ----------------------------------------------------------- localisation */

/* Bytes of device workspace rc_localize_mask needs for N tokens and
 * n_delta delta tokens. */
size_t rc_localize_workspace_size(int N, int n_delta);

/* Edit region R_edit of Section 3.2 as a dirty mask and a compact list.
 *   xattn        f32 [S][N][M] cross-attention scores (S slices, e.g. heads
 *                x layers, averaged: summed in ascending s, divided by S).
 *   delta_ids_host  int32 [n_delta], the new/modified text tokens, each in
 *                [0, M); 1 <= n_delta <= 64.
 *   threshold    per delta token j the scores are min-max normalised over the
 *                N tokens and token i is in j's region iff the normalised
 *                value is >= threshold; a constant column gives no token,
 *                and so does a column whose averaged scores hold a
 *                non-finite value (NaN, +-Inf), where the normalisation is
 *                undefined.
 *   dilation     the union over j is dilated by a (2r+1)^2 square on the
 *                grid_h x grid_w token grid (r = dilation, 0..8), neighbours
 *                outside the grid ignored.
 *   mask         out, u8 [N] 0/1.
 *   dirty_idx    out, int32 [N] capacity; the first D entries are the dirty
 *                tokens in ascending order.
 *   dirty_count  out, int32 [1] device: D.
 *   workspace    device scratch of rc_localize_workspace_size() bytes.
 * The comparison is taken in f32 with round-to-nearest subtraction and
 * division, so the result is bit-identical to a float32 evaluation of the
 * same definition.  Errors: RC_ERR_INVALID_ARG, RC_ERR_SHAPE
 * (N != grid_h * grid_w, N > 16384, M < 1). */
rc_status rc_localize_mask(const float* xattn, int S, int N, int M, int grid_h, int grid_w,
                           const int32_t* delta_ids_host, int n_delta, float threshold,
                           int dilation, uint8_t* mask, int32_t* dirty_idx,
                           int32_t* dirty_count, void* workspace, size_t workspace_bytes,
                           rc_stream stream);

/* Allocation-free variant of rc_localize_mask.  The paper has no counterpart
 * to this entry point; it exists for callers that cannot allocate device
 * memory where they need a mask: code running inside an inference server's
 * plugin hook that must not call the CUDA allocator, programs whose device
 * memory is wholly owned by another framework's pool, and latency-critical
 * loops that cannot afford cudaMalloc's implicit device-wide synchronisation.
 *
 * It computes exactly what rc_localize_mask computes (same arguments minus
 * the workspace, same bit-exact result) but takes its scratch from a fixed
 * array compiled into the library: RC_NOALLOC_SCRATCH_BYTES (about 1 MiB) of
 * device memory that every GPU which loads the library holds until the
 * process exits.  It calls no cudaMalloc, cudaFree or other allocating
 * routine.
 *   Limits: N <= RC_NOALLOC_MAX_TOKENS and n_delta <= RC_NOALLOC_MAX_DELTA;
 *   larger sizes return RC_ERR_SHAPE with a message naming the limit.
 *   Set-up: the first call on each device (with that device current) looks
 *   up the array's device address once and keeps it for the rest of the
 *   process; make that first call before any stream capture.  The kept
 *   address does not survive cudaDeviceReset (or any destruction of the
 *   device's primary context): do not call this entry point after one.
 *   Sharing: every call on a device uses the same scratch, which keeps the
 *   previous call's contents; no part of it needs to start at zero (each
 *   pass overwrites what the next pass reads).  Calls whose work overlaps on
 *   the GPU (for example issued on two unordered streams) race on the
 *   scratch and can return wrong masks: serialise them on one stream or
 *   order them with events. */
#define RC_NOALLOC_MAX_TOKENS 16384
#define RC_NOALLOC_MAX_DELTA 16
#define RC_NOALLOC_SCRATCH_BYTES 1073408
rc_status rc_localize_mask_noalloc(const float* xattn, int S, int N, int M, int grid_h,
                                   int grid_w, const int32_t* delta_ids_host, int n_delta,
                                   float threshold, int dilation, uint8_t* mask,
                                   int32_t* dirty_idx, int32_t* dirty_count, rc_stream stream);

/* ------------------------------------------------------------ block / step */

/* Region-level sparse forward of block `layer` at timestep slot `t` of
 * `session` (Section 3.3, Region-Level Sparse Attention; Section 3.4, Kernel
 * Fusing).
 *   hidden       f32 [N][hidden], in/out: rows dirty_idx[r] are the dirty
 *                tokens' block inputs and are overwritten with their block
 *                outputs; other rows are neither read nor written.
 *   dirty_idx    int32 device, distinct token indices in [0, N) (any order).
 *   D            number of dirty tokens, 0..N; with dirty_count non-null it
 *                is only an upper bound (-1 = N) and *dirty_count is used.
 *   mod6         f32 [6][hidden] device: this block's adaLN-single vector
 *                (table + timestep projection).
 * Effect on the cache slot (session, layer, t): K and V rows of the dirty
 * tokens are replaced by their fresh projections before the attention (the
 * dirty queries attend over all N keys: cached for clean tokens, fresh for
 * dirty ones); H rows of the dirty tokens are replaced by their block
 * outputs (bf16), so H holds the merged H^{l+1}.  Clean rows are untouched.
 * D = 0 is legal and changes nothing.  Errors: RC_ERR_INVALID_ARG,
 * RC_ERR_STATE (weights or text not set). */
rc_status rc_block_forward_region(rc_ctx* ctx, rc_cache* cache, int session, int layer, int t,
                                  float* hidden, const int32_t* dirty_idx, int D,
                                  const int32_t* dirty_count, const float* mod6,
                                  rc_stream stream);

/* One denoising step t of `session` following the reuse schedule
 * schedule_host[timesteps] (modes RC_MODE_*; Section 3.3, Eq. 2):
 *   DENSE   every token is embedded and pushed through all blocks; every
 *           cache row of (session, *, t) is overwritten.
 *   SPARSE  only the dirty tokens (dirty_idx / D / dirty_count as in
 *           rc_block_forward_region) are embedded and recomputed through all
 *           blocks; clean rows come from the cache.
 *   REUSE   no block runs; the final layer reads the cached H of the last
 *           block.
 * Then the final layer (LayerNorm, modulation by the timestep embedding,
 * linear to p*p*out_ch) gives eps (the first in_ch output channels) for all
 * tokens and the latent is updated in place by DDIM (eta = 0).
 *   latent  f32 [in_ch][grid_h*patch][grid_w*patch], in/out.
 * Errors: RC_ERR_INVALID_ARG, RC_ERR_STATE (weights, schedule or text not
 * set). */
rc_status rc_step(rc_ctx* ctx, rc_cache* cache, int session, float* latent, int t,
                  const uint8_t* schedule_host, const int32_t* dirty_idx, int D,
                  const int32_t* dirty_count, rc_stream stream);

/* One item of a batched step: one session's denoising step.
 *   session      cache session (an item per (session, t) at most per call)
 *   latent       device f32 [in_ch][grid_h*patch][grid_w*patch], in/out
 *   t            timestep index in [0, timesteps)
 *   mode         RC_MODE_DENSE / SPARSE / REUSE for this step
 *   dirty_idx, D, dirty_count   SPARSE only, as in rc_step */
typedef struct rc_batch_item {
  int session;
  float* latent;
  int t;
  int mode;
  const int32_t* dirty_idx;
  int D;
  const int32_t* dirty_count;
} rc_batch_item;

/* Batched serving (no counterpart in the paper, which serves one request at
 * a time): one denoising step for each of n_items sessions, each exactly as
 * rc_step would compute it (Section 3.3 region-level sparse attention per
 * item: an item's dirty queries attend over its own session's cached and
 * fresh keys / values at its own timestep, with its own text context).  The
 * dirty rows of all items are processed together, so every weight matrix is
 * read once per call.  items: host array; 1 <= n_items <= the context's
 * max_batch.  Errors: RC_ERR_INVALID_ARG (bad item, two items on the same
 * (session, t), n_items out of range), RC_ERR_STATE (weights, schedule or a
 * session's text not set). */
rc_status rc_step_batched(rc_ctx* ctx, rc_cache* cache, const rc_batch_item* items, int n_items,
                          rc_stream stream);

/* A DENSE step (as rc_step with mode DENSE) that also produces the
 * localisation scores of Section 3.2 for the next sparse steps: for each of
 * the n_delta (1..8) newly introduced or modified text tokens j in
 * delta_ids_host (host array, values in [0, text_len)), the cross-attention
 * probabilities of j, aggregated (averaged) over the heads and layers of
 * the step:  scores[i][j] = mean_{l,h} softmax_j'(q'_{l,h,i} k_{l,h,j'} /
 * sqrt(head_dim))[j], for every image token i.
 *   scores  device f32 [N][text_len] (caller-owned, 16-B aligned): zeroed,
 *           then the delta columns written; it is the [S = 1][N][M] score map
 *           rc_localize_mask takes.
 * Errors: as rc_step; RC_ERR_INVALID_ARG for bad ids or n_delta. */
rc_status rc_step_capture(rc_ctx* ctx, rc_cache* cache, int session, float* latent, int t,
                          const int32_t* delta_ids_host, int n_delta, float* scores,
                          rc_stream stream);

/* The localisation scores of Section 3.2 for a new editing turn, computed
 * from the cached states of the previous turn instead of a dense step, so
 * that a turn scheduled by Eq. 2 (REUSE steps, then SPARSE steps, no dense
 * step at all) can localise its edit before anything is recomputed.  Call
 * it after rc_set_text with the new prompt.  For each of the n_delta (1..8)
 * new or modified text tokens j in delta_ids_host (host array, values in
 * [0, text_len)):
 *   scores[i][j] = mean over blocks l and heads h of
 *                  softmax_j'(q'_{l,h,i} k_{l,h,j'} / sqrt(head_dim))[j],
 * where the text keys k are the session's current ones and the image
 * queries q' = H^l W_xq^T + b_xq use the hidden state entering block l as
 * the cache holds it at timestep slot t: for l >= 1 the cached output of
 * block l - 1 (bf16), for l = 0 the patch embedding of `latent` (f32
 * [in_ch][grid_h*patch][grid_w*patch], the latent of step t).  The cache is
 * only read.
 *   scores  device f32 [N][text_len] (caller-owned, 16-B aligned): zeroed,
 *           then the delta columns written; it is the [S = 1][N][M] score
 *           map rc_localize_mask takes.
 * Errors: RC_ERR_INVALID_ARG (bad session, t, ids or n_delta, a host-tier
 * cache), RC_ERR_STATE (weights or the session's text not set). */
rc_status rc_localize_scores(rc_ctx* ctx, rc_cache* cache, int session, int t,
                             const float* latent, const int32_t* delta_ids_host, int n_delta,
                             float* scores, rc_stream stream);

/* Semantic-aware adaptive reuse scheduling (Section 3.3), host-only.
 * rc_prompt_similarity: Eq. 1, s = cos(e(tau-), e(tau+)) of two token
 *   embeddings (host arrays of dim floats), accumulated in double.
 * rc_reuse_schedule: Eq. 2, T_reuse = T if s >= tau_s else floor(rho T), and
 *   the per-step modes of an edited region for rc_step: RC_MODE_REUSE for
 *   t < T_reuse, RC_MODE_SPARSE after (modes_out: host array of T).  The
 *   paper sets rho = 0.2.
 * Errors: RC_ERR_INVALID_ARG (null, dim or T <= 0, zero embedding, rho
 * outside [0, 1], NaN). */
rc_status rc_prompt_similarity(const float* e_minus, const float* e_plus, int dim, float* s_out);
rc_status rc_reuse_schedule(float s, float tau_s, float rho, int T, uint8_t* modes_out);

/* CUDA Graph of one rc_step (no counterpart in the paper; serving
 * plumbing): the step's ~255 kernel launches for fixed arguments are
 * recorded once and replayed with one launch call.  The arguments are those
 * of rc_step; the graph keeps the device pointers (latent, dirty_idx,
 * dirty_count, the cache slots of (session, t)) and reads and writes their
 * CONTENTS at each replay, so a new edit region only needs new dirty_idx /
 * dirty_count contents (use D = -1 with a device count whose bound is N).
 * Mode schedule_host[t] and the host bound D are fixed at creation.  The
 * graph reuses the context's scratch: replays of graphs of one context are
 * serialised on one stream, like its steps.  Creation enqueues nothing on
 * the caller's streams; when the per-timestep embedding tables are stale
 * (see rc_set_global_weights) it computes them first, on a private stream
 * that it waits for.  A replay reads those tables but keeps the DDIM
 * coefficients of the schedule at creation: create graphs again after
 * rc_set_schedule or rc_set_global_weights.
 * Errors: as rc_step; RC_ERR_INVALID_ARG for a host-tier cache or while a
 * timing probe is enabled; RC_ERR_CUDA when capture or instantiation fails. */
typedef struct rc_graph rc_graph;
rc_status rc_step_graph_create(rc_ctx* ctx, rc_cache* cache, int session, float* latent, int t,
                               const uint8_t* schedule_host, const int32_t* dirty_idx, int D,
                               const int32_t* dirty_count, rc_graph** out);
/* Replays the graph on `stream`. */
rc_status rc_graph_launch(rc_graph* graph, rc_stream stream);
void rc_graph_destroy(rc_graph* graph);

/* Cross-session serving scheduler (no counterpart in the paper, which serves
 * one request at a time): editing sessions join and leave between steps,
 * and every tick runs ONE rc_step_batched over up to max_items of the turns
 * in progress, each at its own timestep, so that one pass over the weights
 * serves them all.  A turn = the steps t = 0 .. timesteps-1 of one session,
 * in order, each computed exactly as rc_step would compute it.  When more
 * turns are running than a tick takes, the least recently stepped go first
 * (ties: admission order), so every turn advances in round robin.  Host
 * state only; drive a server from one host thread, and let no other call
 * step the sessions it is running.
 *   rc_server_create   max_items in [1, the context's max_batch] (1 for a
 *                      host-tier cache).
 *   rc_server_admit    starts a turn of `session` (not already running):
 *                      latent f32 [in_ch][grid_h*patch][grid_w*patch]
 *                      device, in/out; schedule_host[timesteps] modes
 *                      (copied); dirty_idx / D / dirty_count as in rc_step,
 *                      read at each SPARSE step (borrowed until the turn
 *                      ends).
 *   rc_server_tick     one batched step on `stream`; sessions_out (host,
 *                      max_items entries, may be null) receives the sessions
 *                      stepped, *n_out their number (0 when no turn is
 *                      running).  A turn whose last step ran leaves the
 *                      server.  On an error nothing advances.
 *   rc_server_state    *next_t = the next step of the session's running
 *                      turn, or -1 when it has none.
 *   rc_server_running  number of turns in progress.
 * Errors: RC_ERR_INVALID_ARG, and those of rc_step_batched. */
typedef struct rc_server rc_server;
rc_status rc_server_create(rc_ctx* ctx, rc_cache* cache, int max_items, rc_server** out);
void rc_server_destroy(rc_server* server);
rc_status rc_server_admit(rc_server* server, int session, float* latent,
                          const uint8_t* schedule_host, const int32_t* dirty_idx, int D,
                          const int32_t* dirty_count);
rc_status rc_server_tick(rc_server* server, rc_stream stream, int* sessions_out, int* n_out);
rc_status rc_server_state(const rc_server* server, int session, int* next_t);
int rc_server_running(const rc_server* server);

/* Full-recompute baseline: rc_step with mode DENSE. */
rc_status rc_step_dense(rc_ctx* ctx, rc_cache* cache, int session, float* latent, int t,
                        rc_stream stream);

/* ------------------------------------------------------------- auxiliary */

/* The tensor-core GEMM of the block on its own: y = x W^T + b.
 *   x bf16 [rows][k], W bf16 [n][k], b f32 [n] (may be null), y f32 [rows][n].
 *   k % 64 == 0, n % 64 == 0, rows >= 0.
 * Provided so the GEMM can be checked and timed in isolation. */
rc_status rc_linear(rc_ctx* ctx, const void* x, const void* W, const float* b, float* y,
                    int rows, int n, int k, rc_stream stream);

/* The dirty-query attention of the block on its own (Section 3.3,
 * Region-Level Sparse Attention): for each of the context's heads h,
 * O[r][h*dh..] = softmax(Q_r,h K_h^T / sqrt(dh)) V_h over the Nk keys.
 *   Q bf16 [Nq][ldq], K and V bf16 [Nk][ldkv] (head h in columns h*dh ..
 *   h*dh+dh-1), O bf16 [Nq][ldo].  ldq, ldkv, ldo multiples of 8, >= heads*dh;
 *   pointers 16-byte aligned; Nq, Nk >= 0.
 * Provided so the attention kernel can be checked and timed in isolation. */
rc_status rc_attention(rc_ctx* ctx, const void* Q, int ldq, const void* K, const void* V,
                       int ldkv, int Nq, int Nk, void* O, int ldo, rc_stream stream);

/* ------------------------------------------------------ eight-bit serving */

/* Weights, activations and cached keys / values in eight bits (no counterpart
 * in the paper; serving plumbing).  A value is an e4m3 code (4 exponent, 3
 * mantissa bits, no infinity, largest 448) times its block's scale, a power
 * of two held as one byte: byte b stands for 2^(b - 127), 255 for NaN.  The
 * scale of a block whose largest magnitude is a is the least 2^e, e >= -127,
 * with a <= 448 * 2^e; codes are rounded to nearest, ties to even.  A block
 * that holds a non-finite value has scale 255 and NaN codes (0x7f) throughout,
 * so everything computed from it is NaN.  (A power of two costs e4m3 no
 * relative precision within its 2^15 of normal range, a scale can be raised
 * later without rounding the codes again, and the tensor core applies it.)
 *
 * Entry points below take a context for its error word only (rc_sync), keep
 * no state and no scratch in it, and allocate nothing: calls on different
 * streams may overlap as long as their buffers do not.  The context's device
 * must be current (RC_ERR_INVALID_ARG otherwise).  All of them may be
 * captured into a graph, which keeps the pointers and sizes. */
#define RC_BF16 0
#define RC_F32 1

/* A quantised matrix of `rows` x `cols` values, blocks of `group` rows (1 or
 * 128) by 128 columns.
 *   codes   u8 [rows][ld], 16-B aligned, ld >= cols a multiple of 16; columns
 *           cols .. ld - 1 are neither read nor written.
 *   scales  u8 [ceil(cols / 128)][lds], lds >= ceil(rows / group): the scale
 *           of (r, c) is scales[c / 128][r / group].
 * rows is at most RC_FP8_MAX_ROWS, cols RC_FP8_MAX_COLS. */
#define RC_FP8_MAX_ROWS 1073741824
#define RC_FP8_MAX_COLS 4194304
typedef struct rc_fp8 {
  void* codes;
  void* scales;
  int rows, cols, ld, lds, group;
} rc_fp8;

/* out = x quantised.  x: rows x cols values of `type` (RC_BF16, RC_F32) with
 * row stride ldx >= cols, aligned to its element size (16-B aligned rows are
 * read faster).  out->rows = 0 is legal and does nothing.  Errors:
 * RC_ERR_INVALID_ARG (null, alignment, type, group), RC_ERR_SHAPE. */
rc_status rc_fp8_quantize(rc_ctx* ctx, const void* x, int ldx, int type, const rc_fp8* out,
                          rc_stream stream);

/* rc_linear on quantised operands: y = x W^T + b with f32 accumulation.
 *   x  [rows][k], W [n][k] (x->cols == W->cols), each with either group.
 *   b  f32 [n] or null.
 *   y  `type` (RC_BF16, RC_F32) [rows][ldy], ldy >= n, aligned to its element
 *      size (16-B aligned rows are written faster); columns n .. ldy - 1 are
 *      not written.
 * Any rows >= 0, n >= 1, k >= 1.  Results are bit-identical from call to
 * call.  Errors: RC_ERR_INVALID_ARG, RC_ERR_SHAPE. */
rc_status rc_fp8_linear(rc_ctx* ctx, const rc_fp8* x, const rc_fp8* W, const float* b, void* y,
                        int ldy, int type, rc_stream stream);

/* A paged key / value cache in eight bits: blocks of RC_KV8_BLOCK tokens, one
 * scale for each (block, head) of the keys and of the values.
 *   k, v              u8 codes [blocks][kv_heads][RC_KV8_BLOCK][head_dim],
 *                     16-B aligned; head_dim 64, 72 or 128.
 *   k_scale, v_scale  u8 [blocks][kv_heads].
 * A new pool is filled with zeros by its owner.  A token's slot is
 * block * RC_KV8_BLOCK + its place in the block; blocks * RC_KV8_BLOCK must
 * stay below 2^31. */
#define RC_KV8_BLOCK 64
typedef struct rc_kv8 {
  void* k;
  void* v;
  void* k_scale;
  void* v_scale;
  int blocks, kv_heads, head_dim;
} rc_kv8;

/* Block table and slot map of a step, built on the device from the requests'
 * lengths.  For each of n_requests (1 .. RC_KV8_MAX_REQUESTS) requests r:
 *   lengths      i32: its tokens once this step's rows are stored.
 *   counts       i32: its rows of this step (null: lengths, a first fill),
 *                0 <= counts[r] <= lengths[r].
 *   table        i32 [n_requests][ld_table], in/out: the blocks of its
 *                tokens; ceil(lengths[r] / RC_KV8_BLOCK) <= ld_table.
 *   row_offsets  out, i32 [n_requests + 1]: the rows of all requests one after
 *                another; request r owns rows row_offsets[r] ..
 *   slots        out, i32 [n_slots]: the slot of each row; entries behind the
 *                last row are -1.  The sum of counts <= n_slots <= 2^30.
 * Without positions (null) the rows are the request's last counts[r] tokens.
 * Blocks that no earlier token lies in are taken from free_blocks (i32
 * [n_free], null: 0 .. n_free - 1) in order, request by request, and written
 * to the table; *used (out, i32) is how many were taken.  With positions (i32
 * [n_slots], the token of each row, 0 .. lengths[r] - 1: an edit's dirty
 * tokens) the table is only read and *used is 0.
 * Device checks (RC_ERR_DEVICE_ASSERT at rc_sync): a request with bad counts
 * or too long for its table has no rows; a row whose block is missing (the
 * free blocks have run out, an entry below 0 or of 2^25 on) or whose position is out
 * of range has slot -1; rows beyond n_slots are dropped.
 * Errors: RC_ERR_INVALID_ARG, RC_ERR_SHAPE. */
#define RC_KV8_MAX_REQUESTS 4096
rc_status rc_kv8_tables(rc_ctx* ctx, const int32_t* lengths, const int32_t* counts,
                        const int32_t* positions, int n_requests, const int32_t* free_blocks,
                        int n_free, int32_t* table, int ld_table, int32_t* row_offsets,
                        int32_t* slots, int n_slots, int32_t* used, rc_stream stream);

/* Stores key and value rows into their slots.
 *   k, v    `type` (RC_BF16, RC_F32) [n][ldkv], head h in columns
 *           h * head_dim ..; ldkv >= kv_heads * head_dim; aligned to the
 *           element size (16-B aligned rows are read faster).
 *   slots   i32 [n]; a negative slot skips its row.  Slots are distinct, and
 *           the rows of one block stand next to one another (as
 *           rc_kv8_tables gives them for ascending tokens), with nothing but
 *           skipped rows between them, within RC_KV8_BLOCK rows of the list.
 *   count   i32 on the device, the rows to store (null: n), 0 .. n.
 *   mode    RC_KV8_UPDATE: a block's scale is raised when the new rows need
 *           it (the codes of its other tokens move with it) and never
 *           lowered.  RC_KV8_APPEND: a block whose first token is among the
 *           rows starts anew, its scale set by these rows alone and its other
 *           tokens void; other blocks as in RC_KV8_UPDATE.
 * Device checks: a slot beyond the pool or a slot twice in a block's rows is
 * skipped and reported.  Rows of one block in two places of the list, or
 * farther apart, are not detected: the block's codes and scale may be wrong.
 * Errors: RC_ERR_INVALID_ARG, RC_ERR_SHAPE. */
#define RC_KV8_UPDATE 0
#define RC_KV8_APPEND 1
rc_status rc_kv8_store(rc_ctx* ctx, const rc_kv8* pool, const void* k, const void* v, int ldkv,
                       int type, const int32_t* slots, int n, const int32_t* count, int mode,
                       rc_stream stream);

/* rc_attention over the paged eight-bit cache for several requests at once:
 * for each row i of request r and each of `heads` query heads h,
 *   O = softmax(q K^T / sqrt(head_dim)) V
 * over the cached tokens 0 .. lengths[r] - 1 of r's blocks, with key head
 * h / (heads / kv_heads).  With causal != 0 the rows are the request's last
 * tokens and row i of n sees tokens 0 .. lengths[r] - n + i only.  A row that
 * sees no token gives zeros.
 *   Q            bf16 [q_rows][ldq], O bf16 [q_rows][ldo], 16-B aligned; ldq,
 *                ldo >= heads * head_dim, multiples of 8.
 *   row_offsets  i32 [n_requests + 1], as from rc_kv8_tables: request r owns
 *                rows row_offsets[r] .. row_offsets[r + 1] - 1, at most max_q
 *                of them.  Rows of no request are left as they were.
 *   lengths      i32 [n_requests], 0 .. ld_table * RC_KV8_BLOCK.
 *   table        i32 [n_requests][ld_table].
 * The work is shared out on the host, for requests as long as the table holds
 * and max_q rows at most: values far above the requests' cost time, not results.
 * Keys are exact in the products; sums are f32, the result is rounded to bf16.
 * Softmax weights are bf16 or finer: off by at most 2^-8 of themselves, or 2^-25
 * of their row's largest.  Values more than 2^80 below the largest that a row sees
 * may count as zero.  Results are bit-identical from call to call.
 * Device checks: a request with bad offsets, more than max_q rows or a bad
 * length is left out; a table entry outside the pool hides its tokens.
 * Errors: RC_ERR_INVALID_ARG, RC_ERR_SHAPE (heads not a multiple of kv_heads,
 * heads / kv_heads > 16 or q_rows * heads / kv_heads >= 2^31). */
rc_status rc_kv8_attention(rc_ctx* ctx, const rc_kv8* pool, const void* Q, int ldq, int q_rows,
                           const int32_t* row_offsets, const int32_t* lengths, int n_requests,
                           int max_q, const int32_t* table, int ld_table, int heads, int causal,
                           void* O, int ldo, rc_stream stream);

/* --------------------------------------------------- the rest of a block */

/* What a transformer block needs between its quantised products and the
 * eight-bit cache (no counterpart in the paper; serving plumbing): norms with
 * gate and residual, rotary positions, and feed-forward experts.  As above:
 * the context serves for its error word and device only, nothing is allocated
 * or kept, calls on different streams may overlap as long as their buffers do
 * not, and all calls but rc_rotary_plan (host code) may be captured.  Results
 * are bit-identical from call to call. */

/* A norm over the columns of a row: RC_NORM_LAYER (v - mean) / sqrt(var + eps),
 * RC_NORM_RMS v / sqrt(mean of v^2 + eps), RC_NORM_NONE v itself; then times
 * weight and plus bias (f32 [cols], each null for none; not with RC_NORM_NONE).
 * Sums are f32, the variance is that of the differences from the mean.
 * eps >= 0. */
#define RC_NORM_NONE 0
#define RC_NORM_LAYER 1
#define RC_NORM_RMS 2
typedef struct rc_norm {
  int kind;
  float eps;
  const float* weight;
  const float* bias;
} rc_norm;

/* The row work between two products, in one pass: for each row
 *   r  = post(b)            b: the row of h, or with top_k > 0 the sum over j of
 *                           weights[row][j] * h[places[row][j]]
 *   x' = residual_scale * x + gate * r
 *   y  = pre(x') * (1 + scale) + shift
 * all in f32, rounded once where x' and y are written (y is made of x' before
 * its rounding).
 *   rows, cols   cols 1 .. RC_NORM_MAX_COLS.
 *   x            x_type (RC_BF16, RC_F32) [rows][ldx], or null for zeros.
 *   x_out        x_type [rows][ldx_out], may be x itself, or null: not written.
 *   h            h_type [rows][ldh] ([h_rows][ldh] with top_k > 0), or null: no
 *                branch, x' = residual_scale * x.
 *   places, weights  i32, f32 [rows][top_k], top_k 0 .. RC_EXPERTS_MAX_TOP_K; an
 *                entry below 0 is passed over, and so is its weight.
 *   gate, scale, shift  f32 [n_items][ld_mod], each null for 1, 0 and 0.
 *   row_offsets  i32 [n_items + 1] on the device: item i owns rows
 *                row_offsets[i] .. row_offsets[i + 1] - 1.  Rows of no item are
 *                left as they were.  Null with n_items = 1: all rows.
 *   y            y_type [rows][ldy], or null.
 *   y8           y as codes instead (then y is null): rows x cols or more rows,
 *                group 1; codes and scales as rc_fp8_quantize gives them for the
 *                f32 values.  null: none.
 * One of x_out, y and y8 at least.  Buffers overlap only where x_out is x with
 * the same stride.  Pointers are aligned to their types (rows of 16-B aligned
 * pieces are read and written faster).
 * Device checks: row_offsets that descend or leave 0 .. rows (rows near them may
 * be left out) and a place of h_rows and more (passed over) are reported.
 * Errors: RC_ERR_INVALID_ARG, RC_ERR_SHAPE. */
#define RC_NORM_MAX_COLS 16384
#define RC_EXPERTS_MAX_TOP_K 16
typedef struct rc_residual {
  int rows, cols, n_items, top_k;
  const int32_t* row_offsets;
  const void* x;
  void* x_out;
  const void* h;
  const int32_t* places;
  const float* weights;
  const float* gate;
  const float* scale;
  const float* shift;
  void* y;
  const rc_fp8* y8;
  int x_type, ldx, ldx_out, h_type, ldh, h_rows, ld_mod, y_type, ldy;
  float residual_scale;
  rc_norm post, pre;
} rc_residual;
rc_status rc_norm_residual(rc_ctx* ctx, const rc_residual* op, rc_stream stream);

/* Rotary positions.  A head's channels first .. first + rot - 1 form rot / 2
 * pairs, each turned by its row's position times the pair's frequency:
 *   (a, b) -> amplitude * (a cos - b sin, b cos + a sin).
 * RC_ROTARY_HALF pairs channel i with i + rot / 2, RC_ROTARY_PAIRS 2 i with
 * 2 i + 1.  Up to three axes (a token's place in text, or in an image's rows
 * and columns) take pairs[a] pairs each, one after another; axis a's position
 * is positions[row][a].
 *
 * rc_rotary_plan (host code, no context) fills a plan from its description:
 *   rot        2 .. 256, even; pairs[0 .. axes - 1] positive, summing to rot / 2.
 *   theta      > 0.  Pair i of an axis with p pairs turns f = theta^(-i / p)
 *              radians a position, changed by `scaling` for contexts `factor`
 *              (>= 1) times as long as the native_length the model was made for:
 *     RC_ROTARY_PLAIN   f;
 *     RC_ROTARY_LINEAR  f / factor;
 *     RC_ROTARY_BASE    theta taken times factor^(p / (p - 1)) (p > 1);
 *     RC_ROTARY_BANDS   k f + (1 - k) f / factor with k = (native_length f / 2 pi -
 *                       slow) / (fast - slow), cut to 0 .. 1: pairs that turn often
 *                       stay, slow ones are stretched;
 *     RC_ROTARY_RAMP    the same with k = 1 - (i - lo) / (hi - lo), cut to 0 .. 1,
 *                       where lo (rounded down, at least 0) and hi (up) are the
 *                       indexes of pairs that turn fast and slow times, and
 *                       hi - lo counts as 0.001 at least; theta > 1.  With one
 *                       axis, as YaRN has it, hi is at most rot - 1, so the ramp
 *                       may end behind the last pair; with several, p - 1.
 *              fast > slow > 0 (in turns over native_length > 0) for the last two.
 *   amplitude  finite.
 * A plan holds a pair's turns a position as a fraction of 2^64: a position
 * times it, modulo 2^64, is the exact place within the turn, so far positions
 * lose nothing to range reduction.  A caller may fill turns itself.
 * Errors: RC_ERR_INVALID_ARG, RC_ERR_SHAPE. */
#define RC_ROTARY_HALF 0
#define RC_ROTARY_PAIRS 1
#define RC_ROTARY_PLAIN 0
#define RC_ROTARY_LINEAR 1
#define RC_ROTARY_BASE 2
#define RC_ROTARY_BANDS 3
#define RC_ROTARY_RAMP 4
#define RC_ROTARY_MAX 256
typedef struct rc_rotary_spec {
  int rot, first, layout, axes, pairs[3], scaling;
  double theta, factor, native_length, fast, slow, amplitude;
} rc_rotary_spec;
typedef struct rc_rotary {
  int rot, first, layout, axes, pairs[3];
  float amplitude;
  uint64_t turns[RC_ROTARY_MAX / 2];
} rc_rotary;
rc_status rc_rotary_plan(const rc_rotary_spec* spec, rc_rotary* out);

/* y = x with its heads' pairs turned.
 *   x, y       `type` (RC_BF16, RC_F32) [rows][ldx], [rows][ldy], head h in
 *              columns h * head_dim ..; y may be x itself with the same stride
 *              (no other overlap): the channels outside first .. first + rot - 1
 *              are then left alone, otherwise copied.  Query and key heads that
 *              lie side by side are turned in one call.  rows and heads >= 0;
 *              head_dim up to RC_ROTARY_MAX_HEAD; pointers aligned to the type
 *              (more makes wider accesses).
 *   positions  i32 [rows][axes], any value; null: the row's index, on all axes.
 *   count      i32 on the device: the rows to turn (null: rows), 0 .. rows; the
 *              rest are left as they were.
 *   inverse    != 0: turned back (the transposed map: also the gradient).
 * Device checks: a count out of range is reported and taken as 0.
 * Errors: RC_ERR_INVALID_ARG, RC_ERR_SHAPE. */
#define RC_ROTARY_MAX_HEAD 1024
rc_status rc_rotary_apply(rc_ctx* ctx, const rc_rotary* plan, const void* x, int ldx, int type,
                          int rows, int heads, int head_dim, const int32_t* positions,
                          const int32_t* count, int inverse, void* y, int ldy, rc_stream stream);

/* The experts of each row.  With a row's logits z, its scores are
 * RC_SCORE_SOFTMAX exp(z) / sum of exp(z), or RC_SCORE_SIGMOID 1 / (1 + exp(-z)).
 * An expert counts by score + bias (bias f32 [experts], null for zeros: balances
 * the load and does not enter the weights).  Of `groups` groups of neighbouring
 * experts only the top_groups with the largest value take part, the value being
 * the sum of a group's group_best best experts.  The top_k best experts are
 * chosen, best first; ties go to the lower index, of groups too.  weights are
 * the chosen scores, with `renormalise` divided by their sum (all 0 where that
 * is 0), times `scale`.
 * Which expert is larger is decided as if scores were computed in f64: f32
 * scores closer than they are exact are computed again.  Without bias, and with
 * groups valued by one expert, it is decided by the logits themselves.
 * An expert whose logit or bias is NaN or -inf (a mask) is never chosen and
 * adds nothing to a softmax; a logit or bias of +inf counts as the largest f32.
 * Where fewer than top_k are left, the rest of ids is -1 with weight 0.
 *   experts 1 .. RC_EXPERTS_MAX, a multiple of groups; top_k 1 ..
 *   RC_EXPERTS_MAX_TOP_K; groups 1 .. 32, top_groups 1 .. groups, group_best 1
 *   or 2; scale finite.
 *   logits       `type` (RC_BF16, RC_F32) [rows][ld], ld >= experts.
 *   count        i32 on the device, rows to route (null: rows); the others' ids are
 *                set to -1 and their weights to 0.
 *   ids, weights out, i32 and f32 [rows][top_k].
 * Device checks: a count out of range is reported and taken as 0.
 * Errors: RC_ERR_INVALID_ARG, RC_ERR_SHAPE. */
#define RC_SCORE_SOFTMAX 0
#define RC_SCORE_SIGMOID 1
#define RC_EXPERTS_MAX 1024
typedef struct rc_routing {
  int experts, top_k, score, groups, top_groups, group_best, renormalise;
  float scale;
  const float* bias;
} rc_routing;
rc_status rc_experts_route(rc_ctx* ctx, const rc_routing* routing, const void* logits, int ld,
                           int type, int rows, const int32_t* count, int32_t* ids, float* weights,
                           rc_stream stream);

/* The rows of each expert, one expert after another and in ascending order.
 *   ids      i32 [rows][top_k], as from rc_experts_route (below 0: no expert).
 *            rows * top_k <= RC_EXPERTS_MAX_PAIRS, experts 1 .. RC_EXPERTS_MAX.
 *   count    i32 on the device, rows to sort (null: rows); the others have no
 *            expert.
 *   offsets  out, i32 [experts + 1]: expert e owns places offsets[e] ..
 *            offsets[e + 1] - 1.
 *   source   out, i32 [rows * top_k]: the row of each place; entries from
 *            offsets[experts] on are left as they were.
 *   places   out, i32 [rows][top_k]: the place of each pair, -1 without one.
 * Device checks: an id of `experts` or more is reported and taken as none, a
 * count out of range is reported and taken as 0.
 * Errors: RC_ERR_INVALID_ARG, RC_ERR_SHAPE. */
#define RC_EXPERTS_MAX_PAIRS 1073741824
rc_status rc_experts_sort(rc_ctx* ctx, const int32_t* ids, int rows, int top_k, int experts,
                          const int32_t* count, int32_t* offsets, int32_t* source,
                          int32_t* places, rc_stream stream);

/* rc_fp8_linear for each expert's rows, with its activation: for the places p
 * of expert e,  y[p] = act(x[row] W_e^T + b_e),  row = source[p], or p without
 * source.
 *   x        group 1; without source of `pairs` rows at least.
 *   W        group 128, W->rows a multiple of experts * 128: expert e's matrix
 *            is rows e * W->rows / experts .., of which the first N count:
 *            N = n, or 2 n with a gated activation.  x->cols == W->cols.
 *   b        f32 [experts][N] or null.
 *   offsets  i32 [experts + 1] as from rc_experts_sort, 0 .. pairs.
 *   source   i32, the row of x of each place, or null.
 *   act      of the f32 sums: RC_ACT_NONE; RC_ACT_GELU v (1 + tanh(sqrt(2 / pi)
 *            (v + 0.044715 v^3))) / 2; RC_ACT_SILU v / (1 + exp(-v));
 *            RC_ACT_GATED_SILU silu(column j) * column n + j.
 *   y        `type` (RC_BF16, RC_F32) [pairs][ldy], ldy >= n, or null with
 *   y8       codes instead: pairs rows at least, n columns, group 1, as
 *            rc_fp8_quantize gives them for the f32 values.
 * Places outside offsets are left as they were.  experts 1 .. RC_EXPERTS_MAX,
 * pairs 0 .. RC_EXPERTS_MAX_PAIRS,
 * (pairs / 128 + experts) * (n / 32 + 1) < 2^31 - 152.
 * The work is shared out on the host for even shares of the pairs; uneven ones
 * cost time, not results.  Activations are good to 2^-15 of themselves, however
 * small they are against the sum (below 2^-126 of it: 0).  Results are
 * bit-identical from call to call.  One expert without source is a plain
 * quantised layer with its activation: offsets {0, rows}.
 * Device checks: offsets that descend or leave 0 .. pairs (the expert is left
 * out) and a source outside x (taken as row 0) are reported.
 * Errors: RC_ERR_INVALID_ARG, RC_ERR_SHAPE. */
#define RC_ACT_NONE 0
#define RC_ACT_GELU 1
#define RC_ACT_SILU 2
#define RC_ACT_GATED_SILU 3
rc_status rc_experts_linear(rc_ctx* ctx, const rc_fp8* x, const rc_fp8* W, const float* b,
                            int experts, int n, const int32_t* offsets, const int32_t* source,
                            int pairs, int act, void* y, int ldy, int type, const rc_fp8* y8,
                            rc_stream stream);

/* Waits for `stream`, then reports (and clears) the context's device error
 * word: RC_ERR_DEVICE_ASSERT if a kernel met a bad index or count,
 * RC_ERR_TIMEOUT if a bounded wait gave up, RC_ERR_CUDA on a CUDA error. */
rc_status rc_sync(rc_ctx* ctx, rc_stream stream);

/* Timing probe.  rc_probe_enable(ctx, which, capacity) makes the context
 * record a pair of CUDA events on the launching stream around each of the
 * next `capacity` launches of kernel class `which` (RC_PROBE_GEMM: every
 * tensor-core GEMM of a block, five, or six when the cross-query projection
 * runs as its own GEMM; RC_PROBE_ATTENTION: the self- and the
 * cross-attention launch of a block;
 * RC_PROBE_LN: both LayerNorm-modulation launches of a block);
 * which = RC_PROBE_OFF disables it.  rc_probe_read waits for the recorded
 * events and returns the summed device time (ms) and the number of launches
 * recorded, then rearms the ring.  rc_probe_read_each does the same but
 * writes each launch's device time (ms, launch order) to the host array
 * ms_out[0 .. capacity) (caller-owned; launches beyond capacity are counted
 * in *launches but not written).  Errors: RC_ERR_INVALID_ARG, RC_ERR_CUDA. */
#define RC_PROBE_OFF 0
#define RC_PROBE_GEMM 1
#define RC_PROBE_ATTENTION 2
#define RC_PROBE_LN 3
rc_status rc_probe_enable(rc_ctx* ctx, int which, int capacity);
rc_status rc_probe_read(rc_ctx* ctx, double* total_ms, int* launches);
rc_status rc_probe_read_each(rc_ctx* ctx, float* ms_out, int capacity, int* launches);

/* Self-test of the device-side failure path (no counterpart in the paper):
 * every kernel of this library that waits on another agent (an mbarrier, a
 * flag) gives up after a bounded time, records RC_ERR_TIMEOUT in the
 * context's error word and returns, so the context stays usable.  This
 * entry point runs that bounded wait on its own: one thread polls a
 * context-owned device flag for at most timeout_us (1 .. 10^6)
 * microseconds; with set_flag = 0 nothing raises the flag, the wait gives
 * up and the next rc_sync returns RC_ERR_TIMEOUT; with set_flag = 1 the
 * flag is raised first and the wait ends at once.  Nothing faults or traps.
 * Errors: RC_ERR_INVALID_ARG. */
rc_status rc_selftest_wait(rc_ctx* ctx, int timeout_us, int set_flag, rc_stream stream);

/* Number of kernels this library has launched in the calling process. */
uint64_t rc_launch_count(void);

const char* rc_status_string(rc_status s);
const char* rc_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* REGIONCACHE_H */
