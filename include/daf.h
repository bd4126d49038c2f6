/*
 * daf.h - C ABI of the Decoupled Attention Fusion (DAF) per-layer prefill
 * attention library for AMD Instinct MI355X (gfx950).
 *
 * DAF (Sec. 2 of the paper) replaces full prefill attention over retrieved
 * documents whose KV caches were computed offline, one document at a time, by
 * three stages per layer:
 *   1. important-token self-attention: n = r*L_d selected rows, taken from
 *      every document, form one packed array whose queries see only keys of
 *      that array (Sec. 2 item 1; Complexity Analysis);
 *   2. question-document attention: the L_q question tokens, at the tail of the
 *      sequence, attend over all L_d + L_q keys, reading a hybrid KV cache in
 *      which the important tokens' rows already hold their recomputed K/V
 *      (Sec. 2 item 2);
 *   3. state fusion: the outputs of both stages are written into the layer's
 *      hidden states (Sec. 2 item 3).
 * The selection policy that picks the important tokens and the Q/K/V
 * projections stay with the caller: indices and projected Q/K/V are inputs.
 *
 * Conventions shared by every entry point
 * ---------------------------------------
 * Memory. Every tensor pointer is DEVICE memory owned by the caller; the
 *   library allocates and frees nothing. Scratch memory comes from the caller's
 *   `workspace`. Pointers must be 16-byte aligned.
 * Layouts. Tensors are token-major and contiguous: queries and outputs are
 *   [tokens][Hq][D], keys and values [tokens][Hkv][D], elements of `dtype`.
 *   One output row (Hq*D elements) is one row of the hidden-state buffer.
 *   LSE outputs are float32 [Hq][rows] (natural log of the softmax
 *   denominator, including the max), row = the output's token row.
 * Requests. A call serves a ragged batch of B >= 1 independent requests
 *   (daf_batch_t). Request b has L_d,b document tokens, L_q,b question tokens
 *   and n_b important tokens. Its rows are:
 *     important rows (q_imp, k_imp, v_imp, o_imp, idx): cu_imp[b] .. cu_imp[b+1]
 *     question rows  (q_q, k_q, v_q, o_q):              cu_q[b]   .. cu_q[b+1]
 *     token rows     (k_cache, v_cache, hidden):        tok_b .. tok_b + T_b,
 *       tok_b = cu_doc[b] + cu_q[b], T_b = L_d,b + L_q,b, documents first.
 * Indices. idx[cu_imp[b] + i] is the request-local original position of
 *   request b's i-th important token: 0 <= idx < L_d,b and strictly increasing
 *   within a request. This is NOT checked on the hot path (violations are
 *   undefined behaviour: duplicate rows make the scatters race);
 *   daf_check_indices() verifies it on the device.
 * Masks. Stage 1: important token i sees important token j iff j <= i (the
 *   condensed order is the original order, so this is causal by original
 *   position). Stage 2: question token j sees every document token and
 *   question tokens 0..j.
 * Numerics. bf16 or fp32 in; fp32 accumulation and softmax; outputs in the
 *   input dtype. bf16 attention rounds the softmax probabilities to bf16
 *   before the value product and normalises by the sum of those rounded
 *   probabilities, so each output row is a weighted mean of value rows with
 *   weights that sum to one; its LSE is the log of that same sum, within
 *   ln(1 + 2^-8) of the exact log-sum-exp (the bf16 rounding of a term that
 *   dominates its row). The unnormalised fp32 sums hold probabilities of at most
 *   2^32 per 16 keys (a row's running max is raised only past that), so value
 *   magnitudes times 2^32 per 16 keys must stay within fp32 (|V| below ~1e26
 *   for 32k keys); small values keep their precision down to bf16's smallest
 *   normal ones. Stage 2's key splits keep their normalised partial outputs
 *   in the input dtype (bf16: one more rounding of each split's weighted mean
 *   before the log-sum-exp merge) and their LSE in fp32.
 * Asynchrony. Work is enqueued on `stream` (NULL = the default stream) and the
 *   call returns without synchronising. Calls are re-entrant and thread-safe;
 *   the only state the library keeps is daf_layer_attn's second stream and its
 *   two events per device (created on first use, guarded by a mutex). Only calls
 *   whose two stages do not go in one launch use them: those with more than 32
 *   stage entries (one per request with important tokens, one per request with a
 *   question), and fp32 calls whose stage 1 has more than 448 pairs of a 128-row
 *   block and a query head. Calls that write the same buffers must be ordered by
 *   the caller.
 * Graph capture. The calls enqueue kernels and event record/wait operations
 *   only (no allocation, copy, memset or synchronisation), so a sequence of
 *   them can be captured into a HIP graph and replayed. Where daf_layer_attn or
 *   daf_decoder_layer uses the second stream (see Asynchrony), it joins the
 *   capture through its fork event and rejoins the caller's stream before the
 *   call returns. Make the first such call on a device outside any capture (it
 *   creates the stream and events), and make no other such call on that device
 *   from another stream or thread while its capture is open: the shared second
 *   stream stays part of the capture until it ends.
 * Errors. Every host-visible precondition is checked before anything is
 *   enqueued; on failure the call returns a non-zero daf_status_t, enqueues
 *   nothing, and daf_last_error() describes the problem (thread-local). A
 *   failed kernel launch returns DAF_ERR_HIP. No C++ exception crosses the ABI.
 */
#ifndef DAF_H_
#define DAF_H_

#include <stddef.h>
#include <stdint.h>

#include <hip/hip_runtime_api.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  DAF_OK = 0,
  DAF_ERR_INVALID_ARG = 1, /* null pointer, bad size, inconsistent offsets */
  DAF_ERR_ALIGNMENT = 2,   /* pointer or row size not a multiple of 16 bytes */
  DAF_ERR_UNSUPPORTED = 3, /* head_dim / dtype the kernels do not cover */
  DAF_ERR_WORKSPACE = 4,   /* workspace missing or smaller than required */
  DAF_ERR_HIP = 5          /* a HIP runtime call or kernel launch failed */
} daf_status_t;

typedef enum { DAF_BF16 = 0, DAF_F32 = 1 } daf_dtype_t;

/* Attention shape. Query head h reads key/value head h / (Hq / Hkv). */
typedef struct {
  int32_t n_q_heads;   /* Hq >= 1 */
  int32_t n_kv_heads;  /* Hkv >= 1, divides Hq */
  int32_t head_dim;    /* D: 64 or 128 */
  int32_t dtype;       /* daf_dtype_t of every tensor */
  float softmax_scale; /* > 0, or 0 for 1/sqrt(D) */
} daf_attn_cfg_t;

/* Ragged batch. All three arrays are HOST memory, [batch + 1] prefix sums
 * starting at 0: cu_doc of L_d,b, cu_q of L_q,b, cu_imp of n_b (n_b <= L_d,b).
 * The library reads them during the call only. */
typedef struct {
  int32_t batch;
  const int32_t *cu_doc;
  const int32_t *cu_q;
  const int32_t *cu_imp;
} daf_batch_t;

/* daf_gather_important `src_layout` values. */
enum {
  DAF_SRC_TOKENS = 0, /* src has T_b rows per request starting at tok_b */
  DAF_SRC_DOCS = 1    /* src has L_d,b rows per request starting at cu_doc[b] */
};

/* daf_fuse `flags` bits. */
enum {
  DAF_FUSE_KV = 1,    /* hybrid KV cache + question KV append */
  DAF_FUSE_HIDDEN = 2 /* stage outputs into the hidden states */
};

/* Gather the important rows into one contiguous array per batch (the row
 * collection step of stage 1, Sec. 2 item 1).
 *   dst[cu_imp[b] + i] = src[base_b + idx[cu_imp[b] + i]]   (row_bytes each)
 * with base_b = tok_b for DAF_SRC_TOKENS or cu_doc[b] for DAF_SRC_DOCS. Rows
 * are copied bit for bit; row_bytes must be a positive multiple of 16. Used
 * for the hidden rows that feed the caller's QKV projection and for K/V rows
 * of a full-length cache. */
daf_status_t daf_gather_important(const daf_batch_t *batch, int32_t src_layout,
                                  const void *src, int64_t row_bytes,
                                  const int32_t *idx, void *dst,
                                  hipStream_t stream);

/* Important-token selection, the step before the path (Sec. 2 item 1: tokens
 * are chosen by the deviation of their recomputed KV from the offline cache,
 * aggregated over several early layers, typically the 2nd to the 4th).
 *   k_fresh[l], k_cached[l], l < n_layers (1..8): a HOST array of DEVICE
 *   pointers per argument; each tensor is [sum L_d][Hkv][D] of `dtype`,
 *   request b's document rows from cu_doc[b] (documents only), 16-byte aligned.
 *   scores (DEVICE float32 [sum L_d], output): per document token, the mean
 *   over the layers of the L2 norm of k_fresh - k_cached over its Hkv*D values
 *   (the paper names the signal but not the norm or the aggregation).
 *   idx (DEVICE int32 [sum n], output): for request b, the n_b = cu_imp[b+1] -
 *   cu_imp[b] tokens with the highest scores (equal scores: lower index
 *   first), request-local, strictly increasing - the idx the other entry
 *   points take.
 * Hkv * D * element size must not exceed 4096 bytes (DAF_ERR_UNSUPPORTED). */
daf_status_t daf_select_important(const daf_attn_cfg_t *cfg,
                                  const daf_batch_t *batch, int32_t n_layers,
                                  const void *const *k_fresh,
                                  const void *const *k_cached, float *scores,
                                  int32_t *idx, hipStream_t stream);

/* Stage 1, important-token self-attention (Sec. 2 item 1; Complexity
 * Analysis: important tokens attend only to each other, O(r^2 L_d^2)).
 *   q_imp [sum n][Hq][D], k_imp / v_imp [sum n][Hkv][D] -> o_imp [sum n][Hq][D]
 *   lse_imp: nullable float32 [Hq][sum n].
 * Within request b, row i attends rows 0..i of the same request (causal in the
 * condensed order, which is the original order). */
daf_status_t daf_imp_self_attn(const daf_attn_cfg_t *cfg,
                               const daf_batch_t *batch, const void *q_imp,
                               const void *k_imp, const void *v_imp,
                               void *o_imp, float *lse_imp, hipStream_t stream);

/* Attention of queries at given positions of a key sequence, for the
 * comparison the Complexity Analysis draws: schemes that recompute selected
 * tokens and the question over the full context (the CacheBlend pattern:
 * important and question tokens over all L_d + L_q keys, O(r L_d^2 + L_d L_q))
 * and full recomputation (every token over its prefix), against which DAF's
 * O(r^2 L_d^2 + L_q (L_d + L_q)) is measured; the Hardware Compatibility
 * paragraph notes that such unified recomputation needs non-standard masks.
 *   q [n_rows][Hq][D], k / v [n_keys][Hkv][D] -> o [n_rows][Hq][D];
 *   lse: nullable float32 [Hq][n_rows].
 * Row i sees keys 0 .. q_pos[i]; q_pos (DEVICE int32 [n_rows]) must be
 * strictly increasing with values in [0, n_keys) - not checked, violations are
 * undefined behaviour. q_pos = NULL means bottom-right causal: row i sees keys
 * 0 .. i + n_keys - n_rows (requires n_rows <= n_keys); with n_rows = n_keys
 * that is full causal self-attention. One sequence per call; no workspace. */
daf_status_t daf_position_attn(const daf_attn_cfg_t *cfg, int32_t n_rows,
                               int32_t n_keys, const void *q,
                               const int32_t *q_pos, const void *k,
                               const void *v, void *o, float *lse,
                               hipStream_t stream);

/* Bytes of workspace daf_qdoc_attn needs for this shape (0 on bad input). */
size_t daf_qdoc_workspace_size(const daf_attn_cfg_t *cfg,
                               const daf_batch_t *batch);

/* Stage 2, question-document attention (Sec. 2 item 2: an L_q x (L_d + L_q)
 * attention over the hybrid KV cache; Complexity Analysis: O(L_q (L_d+L_q))).
 *   q_q [sum L_q][Hq][D]; k_cache / v_cache hold T_b token rows per request
 *   (the hybrid cache: daf_fuse(DAF_FUSE_KV) first) -> o_q [sum L_q][Hq][D];
 *   lse_q: nullable float32 [Hq][sum L_q].
 * Question row j of request b attends cache rows 0 .. L_d,b + j. The keys are
 * split across workgroups; partial results (each split's normalised output in
 * the input dtype and its fp32 LSE) live in `workspace` (at least
 * daf_qdoc_workspace_size bytes, 16-byte aligned, contents undefined after
 * the call) and are merged by log-sum-exp. */
daf_status_t daf_qdoc_attn(const daf_attn_cfg_t *cfg, const daf_batch_t *batch,
                           const void *q_q, const void *k_cache,
                           const void *v_cache, void *o_q, float *lse_q,
                           void *workspace, size_t ws_bytes,
                           hipStream_t stream);

/* State fusion and hybrid-cache construction, as in-place row scatters (Sec. 2
 * item 2: the important tokens' K/V are updated in the document cache before
 * question-document attention; Sec. 2 item 3: stage outputs are fused into the
 * hidden states).
 * DAF_FUSE_KV (needs k_imp, v_imp, k_q, v_q, k_cache, v_cache):
 *   k_cache[tok_b + idx[.]] = k_imp[.],   k_cache[tok_b + L_d,b + j] = k_q[.]
 *   (same for v) - the hybrid cache, with the question's K/V after the docs.
 * DAF_FUSE_HIDDEN (needs o_imp, o_q, hidden [sum T][Hq*D]):
 *   hidden[tok_b + idx[.]] = o_imp[.],    hidden[tok_b + L_d,b + j] = o_q[.]
 * Rows are copied bit for bit; every other row is left untouched. Pointers not
 * needed by the selected flags may be NULL. */
daf_status_t daf_fuse(const daf_attn_cfg_t *cfg, const daf_batch_t *batch,
                      uint32_t flags, const int32_t *idx, const void *k_imp,
                      const void *v_imp, const void *k_q, const void *v_q,
                      void *k_cache, void *v_cache, const void *o_imp,
                      const void *o_q, void *hidden, hipStream_t stream);

/* Bytes of workspace daf_layer_attn needs (0 on bad input). */
size_t daf_layer_workspace_size(const daf_attn_cfg_t *cfg,
                                const daf_batch_t *batch);

/* One DAF attention layer (Sec. 2 items 1-3), in the order the paper fixes:
 * hybrid KV write-back (DAF_FUSE_KV) first, then stage 2 (with its split
 * merge); stage 1 needs none of these and runs beside them: in the same launch
 * as stage 2, or for large batches (see Asynchrony) on a stream the library owns
 * (one per device, default priority), forked from `stream` and joined back into
 * it with events. All of the call's work is ordered on `stream` for the caller.
 * Arguments as in the stage calls. o_imp and o_q receive the stage outputs; the same rows are written into `hidden` exactly
 * as DAF_FUSE_HIDDEN would (the state fusion happens in the stage epilogues,
 * without a separate pass). */
daf_status_t daf_layer_attn(const daf_attn_cfg_t *cfg, const daf_batch_t *batch,
                            const int32_t *idx, const void *q_imp,
                            const void *k_imp, const void *v_imp,
                            const void *q_q, const void *k_q, const void *v_q,
                            void *k_cache, void *v_cache, void *o_imp,
                            float *lse_imp, void *o_q, float *lse_q,
                            void *hidden, void *workspace, size_t ws_bytes,
                            hipStream_t stream);

/* For callers that cannot allocate (code under HIP graph capture, serving
 * loops or harnesses that forbid hipMalloc): daf_layer_attn with the stage-2
 * workspace taken from a static device array of the library instead of a
 * caller buffer, all work on `stream` (no second stream). Arguments and
 * results as in daf_layer_attn. The array holds daf_layer_noalloc_max_bytes()
 * bytes (48 MiB) on every device the library runs on, kept until the process
 * ends; a batch whose workspace (daf_layer_workspace_size) exceeds it returns
 * DAF_ERR_WORKSPACE and enqueues nothing. The call allocates nothing: no
 * hipMalloc, hipFree, stream or event creation. Every call on one device
 * shares that device's array, so calls that can overlap on one device (other
 * streams, other threads) race; order them on one stream. No result depends on
 * what an earlier call left in the array. */
size_t daf_layer_noalloc_max_bytes(void);
daf_status_t daf_layer_attn_noalloc(const daf_attn_cfg_t *cfg, const daf_batch_t *batch,
                                    const int32_t *idx, const void *q_imp,
                                    const void *k_imp, const void *v_imp,
                                    const void *q_q, const void *k_q, const void *v_q,
                                    void *k_cache, void *v_cache, void *o_imp,
                                    float *lse_imp, void *o_q, float *lse_q,
                                    void *hidden, hipStream_t stream);

/* Debug check of the index precondition: writes to *d_bad_count (device
 * int32) the number of entries of idx that are out of [0, L_d,b) or not
 * greater than their predecessor in the same request. */
daf_status_t daf_check_indices(const daf_batch_t *batch, const int32_t *idx,
                               int32_t *d_bad_count, hipStream_t stream);

/* Static name of a status code. */
const char *daf_status_string(daf_status_t status);

/* Dense projection of the decoder layer around the attention: the QKV
 * computation phase of Sec. 2 item 2 (run on the important and question rows
 * only) and the projections that the fused compact state feeds (Sec. 2 item
 * 3): C = A W^T (+ bias) (+ residual), bf16 in and out.
 *   A [M][K] and W [N][K] row-major (W in the usual [out][in] layout);
 *   bias [N] or NULL; residual [M][N] or NULL, and may be C itself (an
 *   in-place residual add); C [M][N].
 * fp32 accumulation; bias and residual are added in fp32 before the single
 * rounding to bf16. N must be a positive multiple of 128 and K of 64
 * (DAF_ERR_UNSUPPORTED otherwise); every pointer 16-byte aligned. M = 0 is a
 * no-op. */
daf_status_t daf_linear(int64_t M, int32_t N, int32_t K, const void *A,
                        const void *W, const void *bias, const void *residual,
                        void *C, hipStream_t stream);

/* The MLP's gate and up projections with the gate applied in the epilogue:
 * C[m][j] = SiLU((A Wg^T)[m][j]) * (A Wu^T)[m][j], SiLU(g) = g / (1 + exp(-g)),
 * where Wgu [2I][K] holds the gate rows then the up rows (bf16, fp32
 * accumulation, one rounding). A [M][K], C [M][I]. I a positive multiple of
 * 64 and K of 64 (DAF_ERR_UNSUPPORTED otherwise); pointers 16-byte aligned. */
daf_status_t daf_linear_swiglu(int64_t M, int32_t I, int32_t K, const void *A,
                               const void *Wgu, void *C, hipStream_t stream);

/* RMS normalisation before the projections: y = x / sqrt(mean(x^2) + eps) * w
 * per row (x, y [rows][width], w [width], bf16; fp32 arithmetic). width must
 * be a positive multiple of 8; y may be x. */
daf_status_t daf_rmsnorm(int64_t rows, int32_t width, const void *x,
                         const void *w, float eps, void *y, hipStream_t stream);

/* Rotary position embedding, in place, of n_heads heads of head_dim features
 * at the start of each of `rows` rows (row pitch row_stride elements, bf16):
 * features (i, i + head_dim/2) of a head rotate by pos[row] *
 * theta^(-2i/head_dim) (the angle in fp64). This is how the recomputed q and
 * k of the important and question rows take their original positions
 * (Sec. 2 item 1 keeps the original order). head_dim even, pos int32 [rows]. */
daf_status_t daf_rope(int64_t rows, int32_t n_heads, int32_t head_dim,
                      int64_t row_stride, void *x, const int32_t *pos,
                      float theta, hipStream_t stream);

/* MLP gate: out[r][j] = SiLU(gu[r][j]) * gu[r][width + j], SiLU(g) =
 * g / (1 + exp(-g)); gu [rows][2 width] (gate then up), out [rows][width],
 * bf16. width a positive multiple of 8. */
daf_status_t daf_silu_mul(int64_t rows, int32_t width, const void *gu,
                          void *out, hipStream_t stream);

/* Weights of one decoder layer (bf16, projections [out][in]): the reading
 * taken for the model the paper evaluates on (Qwen2.5-7B, Sec. 3) is the
 * pre-norm decoder layer
 *   h = RMSNorm(x) w_in; q,k,v = h W^T + b; RoPE(q, k); o = attention
 *   x += o wo^T; h = RMSNorm(x) w_post; x += (SiLU(h wg^T) * (h wu^T)) wd^T */
typedef struct {
  const void *w_in;            /* [hidden] */
  const void *wq, *bq;         /* [Hq*D][hidden], [Hq*D] */
  const void *wk, *bk;         /* [Hkv*D][hidden], [Hkv*D] */
  const void *wv, *bv;         /* [Hkv*D][hidden], [Hkv*D] */
  const void *wo;              /* [hidden][Hq*D] */
  const void *w_post;          /* [hidden] */
  const void *wgu;             /* [2*inter][hidden]: the gate rows, then the up rows */
  const void *wd;              /* [hidden][inter] */
  int32_t hidden, inter;       /* multiples of 128 */
  float eps, rope_theta;
} daf_layer_weights_t;

enum { DAF_LAYER_DAF = 0, DAF_LAYER_FULL = 1 };

/* Workspace daf_decoder_layer needs (0 on bad input). */
size_t daf_decoder_layer_workspace_size(const daf_attn_cfg_t *cfg,
                                        const daf_layer_weights_t *w,
                                        const daf_batch_t *batch,
                                        int32_t mode);

/* One decoder layer of prefill, in place on the residual stream x (bf16
 * [rows][hidden]) at positions pos (int32 [rows]).
 * DAF_LAYER_DAF (Sec. 2 items 1-3): only the important and question rows are
 *   recomputed. rows = sum n + sum L_q, ordered as the stage calls take them:
 *   every request's important rows (in idx order), then every request's
 *   question rows. Their q/k/v come from the projections; the important and
 *   question K/V are written into k_cache / v_cache (the hybrid cache, as
 *   DAF_FUSE_KV) and the DAF attention runs as in daf_layer_attn; the other
 *   document rows are not touched. The updated x is the compact state the
 *   next layer takes (Sec. 2 item 3).
 * DAF_LAYER_FULL (the full-recomputation baseline of Sec. 3): every token is
 *   recomputed; rows = sum T_b, each request's documents then its question,
 *   causal attention over the request's own rows; idx, k_cache and v_cache
 *   are not used (may be NULL).
 * workspace: at least daf_decoder_layer_workspace_size bytes, 256-byte
 * aligned, contents undefined after the call. Errors as for the other calls;
 * nothing is enqueued when a check fails. */
daf_status_t daf_decoder_layer(const daf_attn_cfg_t *cfg,
                               const daf_layer_weights_t *w,
                               const daf_batch_t *batch, int32_t mode,
                               const int32_t *idx, const int32_t *pos, void *x,
                               void *k_cache, void *v_cache, void *workspace,
                               size_t ws_bytes, hipStream_t stream);

/* ---- Paged 8-bit K/V cache -------------------------------------------------
 *
 * The offline document K/V that DAF reuses (Sec. 1), held in 8 bits and in pages
 * that sequences share: a document set is stored once, each request forks it,
 * gets its own copy of the pages it writes its recomputed rows into (the hybrid
 * cache, Sec. 2 item 2), answers its question over it and decodes from it.
 *
 * A page holds DAF_PAGE_TOKENS tokens of every layer and K/V head: token t of a
 * sequence lies in slot t % 64 of the page table[seq][t / 64]. Per layer, page and
 * head it has e4m3 codes (OCP: 3 mantissa bits, largest 448, no infinities) and one
 * scale each for K and V, 0 or a power of two >= 2^-100; a value is code * scale.
 * V is stored transposed, so that a product over tokens reads tokens in order.
 *
 * The arrays are DEVICE memory, owned by the caller and 16-byte aligned. A new
 * cache has refs and len all 0; nothing else needs a value. What the calls below
 * read on the device is not checked by the host: table entries outside
 * [0, n_pages) count as pages that are not there (no keys, nothing read or
 * written), sequences outside [0, n_seqs) as empty ones, and len is read as at
 * most max_seq_pages * 64. No such value makes a call read or write out of
 * bounds. Calls that change a cache are ordered by the caller with the calls
 * that use it (one stream, or events). */
enum { DAF_PAGE_TOKENS = 64 };

typedef struct {
  int32_t n_layers, n_pages;     /* >= 1 */
  int32_t n_kv_heads, head_dim;  /* Hkv >= 1; D: 64 or 128 */
  int32_t n_seqs, max_seq_pages; /* rows and row length of table; max_seq_pages < 2^25 */
  void *k;        /* e4m3 [n_layers][n_pages][Hkv][64][D] */
  void *v;        /* e4m3 [n_layers][n_pages][Hkv][D][64] */
  float *k_scale; /* [n_layers][n_pages][Hkv] */
  float *v_scale; /* [n_layers][n_pages][Hkv] */
  int32_t *table; /* [n_seqs][max_seq_pages]: page ids */
  int32_t *len;   /* [n_seqs]: tokens held */
  int32_t *refs;  /* [n_pages]: table entries that name the page; 0 = free */
} daf_cache_t;

/* Rows of a ragged batch of requests on a cache. cu is HOST memory, the [n + 1]
 * prefix sums (from 0) of the rows per request, read during the call only. seq
 * (DEVICE int32 [n]) is each request's sequence; NULL: request b is sequence b.
 * pos (DEVICE int32 [cu[n]]) is each row's position in its sequence, strictly
 * increasing within a request; NULL: a request's rows are the last ones of its
 * sequence (row j of m at position len - m + j). */
typedef struct {
  int32_t n;
  const int32_t *cu;
  const int32_t *seq;
  const int32_t *pos;
} daf_cache_rows_t;

/* Write the rows' K/V (k, v [cu[n]][Hkv][D] of cfg's dtype) into one layer of
 * the cache: pos = NULL appends (daf_pages_extend has taken the pages and raised
 * len already), pos = the important tokens' positions makes the hybrid cache
 * (Sec. 2 item 2; daf_pages_unshare first where pages are shared).
 *   A page and head's scale becomes the larger of its present one, if a token of
 * the page stays (one below len, or with pos = NULL below the new rows, that the
 * call does not write), and the smallest power of two >= 2^-100 under which the
 * largest new magnitude is at most 448 (none for all zeros). Codes are rounded to
 * nearest even; the codes that stay are rounded again where the scale grows (a
 * loss only where they fall below the smallest normal code). Where no token of
 * the page stays, its other slots become 0. Infinities count as the largest
 * finite value of the dtype, NaN stays NaN and does not count for the scale.
 *   Rows whose position is not in [0, len) are left out. The result is undefined
 * (but in bounds) if positions do not increase, if two requests of the call name
 * the same page, or where a page is shared: its other owners see the rows too. */
daf_status_t daf_cache_write(const daf_attn_cfg_t *cfg, const daf_cache_t *cache,
                             int32_t layer, const daf_cache_rows_t *rows,
                             const void *k, const void *v, hipStream_t stream);

/* The rows' K/V of one layer as values (k, v [cu[n]][Hkv][D] of cfg's dtype, both
 * of which hold them exactly), e.g. the k_cached of daf_select_important. k or v
 * may be NULL (not wanted). Rows whose position is not in [0, len), or whose page
 * is not there, become 0. */
daf_status_t daf_cache_read(const daf_attn_cfg_t *cfg, const daf_cache_t *cache,
                            int32_t layer, const daf_cache_rows_t *rows, void *k,
                            void *v, hipStream_t stream);

/* Bytes of workspace daf_cache_attn needs (0 on bad input or none needed), at most
 * 544 MB. */
size_t daf_cache_attn_workspace_size(const daf_attn_cfg_t *cfg,
                                     const daf_cache_t *cache,
                                     const daf_cache_rows_t *rows, int32_t max_len);

/* Attention of the rows over one layer of the cache: question rows (stage 2,
 * Sec. 2 item 2, on the hybrid cache), rows at given positions, or the single row
 * per sequence of a decode step.
 *   q [cu[n]][Hq][D] -> o [cu[n]][Hq][D]; lse: nullable float32 [Hq][cu[n]].
 * A row sees the keys 0 .. its position of its sequence, as far as len goes (pos =
 * NULL: causal, aligned to the end; pos need not increase here). A row that sees
 * no key gets o = 0 and lse = -infinity. Keys that no row of the call sees may
 * hold anything, NaN included; all others must be finite. A score of NaN or infinity,
 * as q may give, makes the row's o and lse of that head NaN; one of -infinity counts as
 * a key that is not seen.
 *   max_len: a HOST bound on the sequences' len (at most max_seq_pages * 64) that
 * the launch is planned for; len is read on the device, at most max_len counts.
 *   Softmax and sums in fp32; the codes, and q in bf16, enter the products exactly.
 * bf16: a probability enters the value product with an error of at most 2^-11 of itself,
 * or 2^-35 of its row's largest one; fp32: q and the probabilities enter as three bf16
 * terms each (24 bits). |V| must stay below 2^100.
 *   workspace: at least daf_cache_attn_workspace_size bytes, 16-byte aligned,
 * contents undefined after the call; calls that may run at the same time, captured
 * ones included, need one each. */
daf_status_t daf_cache_attn(const daf_attn_cfg_t *cfg, const daf_cache_t *cache,
                            int32_t layer, const daf_cache_rows_t *rows,
                            int32_t max_len, const void *q, void *o, float *lse,
                            void *workspace, size_t ws_bytes, hipStream_t stream);

/* Page calls. They work on all layers, take sequence and page lists in DEVICE
 * memory and never wait for the device. Those that take pages take the free ones
 * (refs 0) of the lowest ids, in the order of the requests and of their pages, and
 * do all or nothing: *status (DEVICE int32) becomes 0, or the number of pages that
 * were lacking, or -1 if an argument is invalid (a sequence out of range or named
 * twice, a length out of range, positions that do not increase), and unless it is 0
 * nothing else changes.
 *
 * Workspace of any of them (fork, unshare, compact); 0 on bad input. 16-byte
 * aligned, contents undefined after the call; calls on different caches that may run
 * at the same time need one each. */
size_t daf_pages_workspace_size(const daf_cache_t *cache);

/* Lengthen n (<= 4096) distinct sequences by n_new[i] >= 0 tokens: pages as needed,
 * len raised. The scales of the pages taken become 0 in every layer, so that nothing of
 * what lay there counts in a later write; a token's K/V are undefined until it is
 * written. seq NULL: sequences 0 .. n-1; n_new NULL: one token each. */
daf_status_t daf_pages_extend(const daf_cache_t *cache, int32_t n,
                              const int32_t *seq, const int32_t *n_new,
                              int32_t *status, hipStream_t stream);

/* Make the empty (len 0) sequence dst[i] a copy of src[i], i < n (<= 4096): full
 * pages are shared (refs + 1), a last page that is not full is copied into a page
 * of its own (one that is not there stays so). dst are distinct and none of them is a src; a src may be named
 * several times. */
daf_status_t daf_pages_fork(const daf_cache_t *cache, int32_t n,
                            const int32_t *src, const int32_t *dst,
                            int32_t *status, void *workspace, size_t ws_bytes,
                            hipStream_t stream);

/* Give the sequences of `rows` (n <= 256, distinct) copies of their own of the
 * pages that hold a row's position and whose refs is above 1 before the call. */
daf_status_t daf_pages_unshare(const daf_cache_t *cache,
                               const daf_cache_rows_t *rows, int32_t *status,
                               void *workspace, size_t ws_bytes, hipStream_t stream);

/* Empty n (<= 2^23) sequences: refs - 1 for their pages (free at 0), their table entries
 * become -1, len 0. A sequence named twice or out of range is no error. seq NULL:
 * sequences 0 .. n-1. */
daf_status_t daf_pages_free(const daf_cache_t *cache, int32_t n,
                            const int32_t *seq, hipStream_t stream);

/* Copy the contents of page src[i] to page dst[i], i < n, in every layer; refs and
 * tables stay as they are. No page may be a dst twice, or both a src and a dst
 * (undefined contents); pairs with an id outside [0, n_pages) are left out. */
daf_status_t daf_pages_copy(const daf_cache_t *cache, int32_t n, const int32_t *src,
                            const int32_t *dst, hipStream_t stream);

/* Move the *n_live (DEVICE int32, output) pages in use to the ids 0 .. *n_live - 1:
 * the i-th used page at or past n_live, in order of ids, goes to the i-th free one
 * below; refs and the tables (entries below len) follow. */
daf_status_t daf_pages_compact(const daf_cache_t *cache, int32_t *n_live,
                               void *workspace, size_t ws_bytes, hipStream_t stream);

/* Detail of the last failure on the calling thread ("" if none). */
const char *daf_last_error(void);

/* Library version, major * 10000 + minor * 100 + patch. */
int32_t daf_version(void);

#ifdef __cplusplus
}
#endif

#endif /* DAF_H_ */
