/*
 * hswa.h -- C ABI of the hybrid sliding-window / full attention library for NVIDIA B200 (sm_100a).
 *
 * The library implements the attention hot path of a layer stack that interleaves Sliding Window Attention
 * layers (window W, 128 in the paper) with Full Attention layers (paper Sec. 2.1), over the dual-pool KV
 * cache of paper Sec. 3.1.1: Full layers keep the whole sequence in pages reached through a per-request
 * block table (equal prefixes may share physical pages, Sec. 3.1.3); SWA layers keep strictly O(W) KV per
 * request in a ring of R pages reached through a ring table and a ring head.
 *
 * Conventions
 *   - "device" pointers are CUDA device addresses on the current device; "host" pointers are ordinary
 *     host memory.  Every array is caller-owned; the library never frees or keeps caller memory.
 *   - Every call that takes `stream` (a cudaStream_t passed as void*) is asynchronous on that stream and
 *     returns after the launches are queued.  No call synchronises except hswa_get_async_error,
 *     hswa_create and hswa_destroy.
 *   - The library allocates exactly one 16-byte device error word per handle (hswa_create) and nothing
 *     else; scratch memory is a caller-provided workspace (hswa_workspace_bytes).
 *   - Host-detectable misuse returns a status at once and launches nothing.  Device-detectable misuse
 *     (hswa_validate_batch; bounded waits inside kernels) is recorded in the error word, the offending
 *     access is skipped, and the kernel returns normally: nothing traps, asserts or spins without bound.
 *   - Within a step the library may overlap consecutive fused decode calls issued through one handle on one
 *     stream (programmatic dependent launch): a later kernel reads the batch arrays and its layer's pool while
 *     the earlier one drains, and waits before touching q, k_new, v_new or its outputs.  This relies on the
 *     contract below that the batch arrays are constant during a step and that only this library, through this
 *     handle, writes the pools; any other call on the handle (append, prefill, advance, error read) ends the
 *     overlap, and two consecutive calls on the same pool never overlap.  A caller that writes a pool itself
 *     between two decode calls of a step, or shares pools between handles, switches the overlap off with
 *     hswa_set_overlap(h, 0).
 *   - No global mutable state except the static scratch of hswa_decode_attn_static_ws; a handle may be used
 *     from one thread at a time.
 *
 * Symbols (bf16 everywhere KV or Q are stored):
 *   Hq, Hkv query / KV heads, G = Hq / Hkv (query head h uses KV head h / G), D head_dim, P page_size,
 *   W window, R ring_pages, C = R * P ring slots, B batch, ctx[r] tokens cached before the step,
 *   n[r] new tokens of request r in the step, T = sum n[r], p = ctx[r] + i the absolute position of the
 *   i-th new token.
 *
 * Pool layout (one pool per layer): bf16 [num_pages][2][Hkv][P][D], index 1 being 0 = K, 1 = V, so a
 * (page, K|V, head) slab is P * D contiguous elements.  The pool base must be 256-byte aligned (TMA
 * descriptors are built over it); q, k_new, v_new and out must be 16-byte aligned.
 *
 * Position -> storage (Sec. 3.1.1, "Full index authoritative, Full -> SWA mapping"):
 *   Full layer: page = block_table[r][p / P], slot = p % P.
 *   SWA  layer: s = (ring_head[r] + (p - ctx[r])) mod C (mathematical mod),
 *               page = ring_table[r][s / P], slot = s % P.
 * Attention (plain softmax attention over the logical sequence; the cache is only storage):
 *   keys j in [lo, p], lo = 0 on a Full layer and max(0, p - W + 1) on an SWA layer (W keys including the
 *   query's own position); out = softmax(sm_scale * q K^T) V with fp32 accumulation, lse = natural-log
 *   log-sum-exp of the scaled scores.
 *   Slots that hold no key of [lo, p] (page tails behind the cached context, ring slots older than the window or
 *   never written, pages no request refers to) may contain anything, bit patterns of NaN and infinity included:
 *   no decode or prefill call lets them change a result (Sec. 3.1.3: attention must not read invalid or
 *   overwritten slots).
 *
 * Supported shapes: D in {64, 128}; P in {16, 32, 64}; 1 <= G <= 8; W >= 1; R * P >= W + 1.
 */
#ifndef HSWA_H_
#define HSWA_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct hswa_handle hswa_handle; /* opaque */

typedef enum {
  HSWA_OK = 0,
  HSWA_ERR_INVALID_ARG = 1, /* null pointer, negative size, inconsistent fields */
  HSWA_ERR_UNSUPPORTED = 2, /* shape outside the supported set */
  HSWA_ERR_WORKSPACE = 3,   /* workspace missing, misaligned or too small */
  HSWA_ERR_CUDA = 4,        /* a CUDA runtime / driver call failed, or no sm_100 device */
  HSWA_ERR_BOUNDS = 5,      /* device-side validation found an out-of-range id or length */
  HSWA_ERR_TIMEOUT = 6      /* a bounded wait inside a kernel ran out */
} hswa_status;

/* Immutable per model. */
typedef struct {
  int32_t num_q_heads;  /* Hq */
  int32_t num_kv_heads; /* Hkv, divides Hq */
  int32_t head_dim;     /* D */
  int32_t page_size;    /* P */
  int32_t window;       /* W (paper: 128) */
  int32_t ring_pages;   /* R; 0 selects ceil(W / P) + 1 */
  float sm_scale;       /* 0 selects 1 / sqrt(D) */
  int32_t out_dtype;    /* 0 = bf16 output, 1 = fp32 output */
} hswa_config;

/* One layer's cache.  `pool` is a device pointer, caller-owned, layout above. */
typedef struct {
  void* pool;
  int64_t num_pages;
  int32_t is_swa; /* per-layer flag: 1 = SWA layer (ring storage, window mask), 0 = Full layer */
} hswa_layer;

/* One step's batch.  All arrays are DEVICE pointers, caller-owned, constant during the step (every layer
 * of the step reuses them); only hswa_step_advance changes ctx_len / ring_head. */
typedef struct {
  int32_t batch;              /* B >= 0 */
  const int32_t* ctx_len;     /* [B] tokens cached before this step */
  const int32_t* q_indptr;    /* [B+1] prefix sums of n[r]; NULL means n[r] = 1 for all r (decode) */
  const int32_t* block_table; /* [B][max_blocks] page ids valid in every Full layer's pool */
  int32_t max_blocks;
  const int32_t* ring_table; /* [B][R] page ids valid in every SWA layer's pool */
  const int32_t* ring_head;  /* [B] ring slot in [0, C) of position ctx_len[r] (the next write) */
  int32_t max_q_len;         /* host-known upper bound of n[r]   (launch geometry only) */
  int32_t total_q;           /* T, host-known                      */
  int32_t max_ctx_len;       /* host-known upper bound of ctx_len[r] (launch geometry only) */
} hswa_batch;

/* Create / destroy a handle on the current CUDA device.  hswa_create validates the config (status
 * UNSUPPORTED / INVALID_ARG), checks the device is compute capability 10.x and allocates the error word.
 * Both calls synchronise the device.  `cfg` is a host pointer and is copied. */
hswa_status hswa_create(const hswa_config* cfg, hswa_handle** out);
void hswa_destroy(hswa_handle* h);

/* Switches the overlap of consecutive fused decode calls (see Conventions) on (default) or off for this handle.
 * Off, every kernel waits for all earlier work on the stream before it reads anything.  (No paper counterpart:
 * a scheduling knob of this library.) */
hswa_status hswa_set_overlap(hswa_handle* h, int32_t enabled);

/* Bytes of workspace (device memory, 256-byte aligned, caller-owned) that is enough for every decode call
 * (hswa_decode_attn, _shared_prefix, _mtp with max_total_q = max_batch * q_len) on batches bounded by the three
 * arguments; hswa_prefill_attn needs none.  An upper bound over all smaller batches and contexts.  Pure host
 * arithmetic. */
size_t hswa_workspace_bytes(const hswa_handle* h, int32_t max_batch, int32_t max_total_q, int32_t max_ctx_len);

/* Exact bytes of workspace ONE decode call needs (split-K partials of paper Sec. 2.2's memory-bound decode: the
 * key range of a Full layer is cut into splits whose (m, l, o) partials live in the workspace): the call on a
 * layer of the given kind with batch->batch = batch, batch->max_ctx_len = max_ctx_len, the given
 * shared_prefix_len (0 for hswa_decode_attn) and q_len (1, or 2-4 for hswa_decode_attn_mtp).  A call is accepted
 * iff its workspace_bytes is at least this.  0 for SWA layers, for calls that need no split, and for arguments
 * out of range.  Pure host arithmetic. */
size_t hswa_decode_workspace_need(const hswa_handle* h, int32_t is_swa, int32_t batch, int32_t max_ctx_len,
                                  int32_t shared_prefix_len, int32_t q_len);

/* Debug aid (paper Sec. 3.1.3: attention must never read invalid or overwritten slots): checks on the device,
 * for the given layer kind, that every id and length the step would use is in range (0 <= ctx <= max_ctx_len,
 * 0 <= n <= max_q_len, block-table coverage of ctx + n, page ids < num_pages, ring_head in [0, C)).  The first
 * violation is recorded in the error word as {HSWA_ERR_BOUNDS, request, index, value}; index -1 / -2 / -3 / -4
 * name ctx, n, block-table coverage and ring head. */
hswa_status hswa_validate_batch(hswa_handle* h, const hswa_layer* layer, const hswa_batch* batch, void* stream);

/* KV append (Sec. 3.1.1 pools; Sec. 3.1.3: an SWA pool stays at window magnitude).
 * k_new, v_new: device, bf16 [T][Hkv][D].  Token i of request r is written at the storage location of
 * position ctx[r] + i.  On an SWA layer later tokens overwrite earlier ones, so only the last min(n, C)
 * tokens of a request are written.  Nothing else in the pool changes.
 * Caller guarantees that pages receiving an append are not shared with another request.
 * A position the block table does not cover, or a page id outside the pool, is recorded in the error word
 * (HSWA_ERR_BOUNDS) and that row is not written. */
hswa_status hswa_kv_append(hswa_handle* h, const hswa_layer* layer, const hswa_batch* batch, const void* k_new,
                           const void* v_new, void* stream);

/* Batched GQA decode attention, one new token per request (batch->q_indptr must be NULL).  Paper Sec. 2.2:
 * decode is memory-bound and its cost is the KV bytes read -- every cached token on a Full layer, the last W
 * on an SWA layer (Sec. 2.1), found through the block table / ring of Sec. 3.1.1.
 * q: device bf16 [B][Hq][D].  out: device [B][Hq][D] in cfg.out_dtype.  lse: device fp32 [B][Hq] or NULL.
 * k_new, v_new: device bf16 [B][Hkv][D], or both NULL.
 *   non-NULL: the new token's K/V are appended (fused into the attention kernel) and attended to.
 *   NULL:     the caller already ran hswa_kv_append with the same un-advanced batch; position ctx[r] is
 *             read from the cache.
 * Full layers split the key range over thread blocks (split-K) and merge the partial results; partials
 * live in `workspace` (hswa_decode_workspace_need bytes; too few: HSWA_ERR_WORKSPACE, nothing launched).
 * On a Full layer the block table must cover position max_ctx_len (max_blocks * P > max_ctx_len), else
 * HSWA_ERR_INVALID_ARG; a request whose ctx_len exceeds max_ctx_len is recorded as HSWA_ERR_BOUNDS. */
hswa_status hswa_decode_attn(hswa_handle* h, const hswa_layer* layer, const hswa_batch* batch, const void* q,
                             const void* k_new, const void* v_new, void* out, float* lse, void* workspace,
                             size_t workspace_bytes, void* stream);

/* Cascade decode for batches whose requests all share a cached prefix (paper Sec. 3.1.3: equal token prefixes
 * share KV pages; Sec. 3.1.4: multi-user shared system prompts).  Same arguments and results as
 * hswa_decode_attn plus shared_prefix_len: the caller (its prefix tree) guarantees that the first
 * shared_prefix_len tokens of EVERY request in the batch map to the same physical pages, i.e. the leading
 * shared_prefix_len / P block-table entries are identical across requests, that shared_prefix_len is a multiple
 * of P and that shared_prefix_len <= ctx_len[r] for all r.  On Full layers the shared keys are then attended
 * once per group of requests as a dense tensor-core problem (rows = requests x heads) instead of being streamed
 * once per request, and merged with the per-request suffixes in the split combine.  SWA layers, shapes the
 * tensor-core stage does not cover (it needs D = 128, P = 64, G = 8) and prefixes shorter than 128 tokens take
 * the hswa_decode_attn path; results are the same up to fp32 rounding order.  shared_prefix_len = 0 is
 * hswa_decode_attn.  Not a multiple of P, negative or above max_ctx_len: HSWA_ERR_INVALID_ARG. */
hswa_status hswa_decode_attn_shared_prefix(hswa_handle* h, const hswa_layer* layer, const hswa_batch* batch,
                                           int32_t shared_prefix_len, const void* q, const void* k_new,
                                           const void* v_new, void* out, float* lse, void* workspace,
                                           size_t workspace_bytes, void* stream);

/* Multi-token decode (paper Sec. 6.2: the models draft with 3 MTP layers, so a decode step verifies the last
 * accepted token plus up to 3 drafts).  Every request has exactly q_len new tokens, 1 <= q_len <= 4;
 * batch->q_indptr must be NULL, batch->total_q = B and batch->max_q_len = 1 as for hswa_decode_attn.
 * q: device bf16 [B][q_len][Hq][D]; k_new, v_new: device bf16 [B][q_len][Hkv][D] (required); out: device
 * [B][q_len][Hq][D]; lse: device fp32 [B][q_len][Hq] or NULL.  Token i of request r has position ctx[r] + i
 * and attends causally (to the cache and to new tokens 0..i; on SWA layers inside its own window).  The q_len
 * tokens end up appended (on a ring that requires q_len <= C - W + 1, checked: HSWA_ERR_INVALID_ARG): on Full
 * layers by an append launch ahead of one kernel that streams the KV once for all q_len tokens, on SWA layers
 * inside the attention kernel, which stages the ring (or, for rings of more than 192 slots, just the window) once
 * for all tokens; a window of more than about 500 tokens on such a ring does not fit one block's shared memory:
 * HSWA_ERR_UNSUPPORTED.  Workspace: as
 * hswa_decode_attn with max_total_q = max_batch * q_len.
 * After the step call hswa_step_advance with a q_indptr describing the ACCEPTED tokens per request. */
hswa_status hswa_decode_attn_mtp(hswa_handle* h, const hswa_layer* layer, const hswa_batch* batch, int32_t q_len,
                                 const void* q, const void* k_new, const void* v_new, void* out, float* lse,
                                 void* workspace, size_t workspace_bytes, void* stream);

/* Decode attention for callers that cannot allocate device memory.  (The paper has no counterpart of this
 * call; it exists for deployment reasons only.)
 * Same arguments, results and errors as hswa_decode_attn, minus the workspace: the split-K partials go to a
 * fixed array of HSWA_STATIC_WS_BYTES bytes that is part of the library's device image, so this call performs
 * no cudaMalloc / cudaFree and calls no allocating routine.  It serves code that runs under a fixed memory
 * budget, or inside a section where an allocation (and the device-wide synchronisation it implies) is not
 * allowed, and that therefore has no workspace to offer.
 *   - Limit: a batch whose partials need more than HSWA_STATIC_WS_BYTES (roughly B * Hq * ceil((max_ctx_len
 *     + 1) / 4096) * (4 * D + 8) bytes on a Full layer, more for small batches, which get shorter splits;
 *     SWA layers need none) is rejected with
 *     HSWA_ERR_WORKSPACE and nothing is launched.
 *   - Every GPU that loads the library holds the array until the process exits.
 *   - The first call on a device looks up the array's device address (with that device current, which must be
 *     the handle's device); make that first call before any stream capture begins.
 *   - All calls on a device share the one array and it keeps whatever the last call left there.  No part of
 *     it has to start at zero: each call writes every partial it later reads.  Two calls that overlap on the
 *     GPU (different streams, or different handles) race on it; issue them on one stream. */
#define HSWA_STATIC_WS_BYTES (64u << 20)
hswa_status hswa_decode_attn_static_ws(hswa_handle* h, const hswa_layer* layer, const hswa_batch* batch,
                                       const void* q, const void* k_new, const void* v_new, void* out, float* lse,
                                       void* stream);

/* Chunked prefill attention: request r extends its cached context by n[r] new tokens.  Paper Sec. 2.1:
 * prefill is compute-bound; a Full layer attends the whole prefix plus the chunk causally, an SWA layer only
 * inside its window of W keys, which is where the roughly 1/7 cost of the hybrid stack comes from; Sec. 5.2:
 * fixed-size chunks against a growing cached prefix.
 * q: device bf16 [T][Hq][D]; k_new, v_new: device bf16 [T][Hkv][D] (required); out: device [T][Hq][D];
 * lse: device fp32 [T][Hq] or NULL.
 * Keys j < ctx[r] are read from the cache AS IT IS BEFORE THIS CHUNK'S APPEND (pages on a Full layer; the
 * ring on an SWA layer), keys j >= ctx[r] from k_new / v_new.  Causal mask on Full layers, causal + window
 * mask on SWA layers; key tiles wholly outside the mask are skipped.
 * fuse_append != 0: the chunk's K/V are also appended to the cache by a second launch (the append kernel of
 * hswa_kv_append) queued on `stream` right behind the attention kernels, i.e. ordered after every read of the
 * old ring contents (an SWA chunk longer than C - W + 1 tokens overwrites ring slots its own first queries
 * need, so "append, then attend" is not available on SWA layers).  The append is fused into the call, not into
 * the attention kernel. */
hswa_status hswa_prefill_attn(hswa_handle* h, const hswa_layer* layer, const hswa_batch* batch, const void* q,
                              const void* k_new, const void* v_new, int32_t fuse_append, void* out, float* lse,
                              void* workspace, size_t workspace_bytes, void* stream);

/* Cross attention to an encoder's states of another length (paper Sec. 3.1.1: one logical view over paged storage; the
 * states are the cached context of a Full layer, written with hswa_kv_append).  Request r attends with its n[r] decoder
 * tokens to ALL of its ctx_len[r] cached positions: no causal mask, nothing is appended.  ctx_len[r] = 0 gives zeros
 * and an lse of minus infinity; n[r] = 0 leaves nothing to do for the request.
 * q: device bf16 [T][Hq][D]; out: device [T][Hq][D] in cfg.out_dtype; lse: device fp32 [T][Hq] or NULL.
 * batch->q_indptr may be NULL (one token per request, the serving step); with it, rows of q behind the last request's
 * do not matter and those of out and lse are left as they were (max_q_len = 0: all of them).  Probabilities enter the
 * PV product as bf16; row sums and lse are taken over the fp32 values.  Workspace: hswa_cross_workspace_need bytes (0:
 * none needed), else HSWA_ERR_WORKSPACE.  The block table must cover max_ctx_len and the layer must not be an SWA layer
 * (HSWA_ERR_INVALID_ARG); max_ctx_len is at most 2^30, for single tokens 65535 * 4096 (HSWA_ERR_UNSUPPORTED, the need
 * is then 0).  A request longer than max_ctx_len or max_q_len, or with row offsets outside [0, total_q], is recorded as
 * HSWA_ERR_BOUNDS (index -1 / -2 / -2); what the bounds cover is computed, other rows of out and lse stay as they were.
 *
 * This call and the eviction calls below refuse a current device other than the handle's (HSWA_ERR_INVALID_ARG).
 *
 * hswa_cross_workspace_need: exact bytes for a call with these host-known fields; pure host arithmetic. */
size_t hswa_cross_workspace_need(const hswa_handle* h, int32_t batch, int32_t total_q, int32_t max_q_len, int32_t max_ctx_len);
hswa_status hswa_cross_attn(hswa_handle* h, const hswa_layer* layer, const hswa_batch* batch, const void* q, void* out,
                            float* lse, void* workspace, size_t workspace_bytes, void* stream);

/* Eviction from a Full layer's cache by accumulated attention weight (no paper counterpart: Sec. 3.1.3 evicts whole
 * segments and out-of-window SWA KV; this shrinks a request's Full KV to the positions that attention uses).  Every
 * (request, KV head) keeps its own positions: the cache stores rotated keys and a Full layer attends to all of them, so
 * their order and their original positions do not matter to the attention calls.
 *
 * hswa_attn_weights, after an attention call on the layer, with the q and lse of that call and the batch as it was (not
 * advanced), its new tokens appended already (fused or by hswa_kv_append):
 *   weights[r][kh][j] = decay * weights[r][kh][j] + sum over tokens i < n[r] and the G query heads h of KV head kh of
 *                       exp(sm_scale * q[r,i,h] . k[j] - lse[r,i,h])   over the rows that see position j.
 *   causal != 0 (self attention): token i sees j <= ctx[r] + i, and positions ctx[r] .. ctx[r] + n[r] - 1 are new: what
 *     their weights held before counts as 0.   causal == 0 (hswa_cross_attn): token i sees every j < ctx[r].
 *   decay = 0 reads none of the old weights.  A row whose lse is minus infinity saw nothing and adds nothing, whatever
 *   its q holds.  To judge a prompt by its last n tokens only, pass those tokens' q and lse with ctx_len reduced by n.
 *   The weights inherit the lse's error: the decode calls' row sums take probabilities rounded to bf16, up to 2^-8 off
 *   on rows of few keys.
 *   After hswa_decode_attn_mtp the batch needs row offsets, q_indptr[r] = r * q_len with max_q_len = q_len and total_q =
 *   B * q_len: the batch of that call (q_indptr = NULL) would mean one row per request.  Rejected drafts have no vote
 *   when their lse is set to minus infinity before the call; their positions lie behind the advanced ctx_len.
 *   q: device bf16 [T][Hq][D]; lse: device fp32 [T][Hq]; weights: device fp32 [B][Hkv][weights_stride], columns at or
 *   past the request's last position are not touched.  weights_stride and the block table must cover max_ctx_len, decay
 *   must be finite and >= 0: HSWA_ERR_INVALID_ARG; max_ctx_len + max_q_len is at most 2^30: HSWA_ERR_UNSUPPORTED.  A
 *   request longer than max_ctx_len or max_q_len, with row offsets outside [0, total_q], or whose ctx + n passes
 *   weights_stride or the block table, is recorded as HSWA_ERR_BOUNDS (index -1 / -2 / -2 / -3) and left out.  Sums are
 *   in fp32 in a fixed order: repeated calls on equal inputs agree bit for bit.
 *
 * hswa_evict_select: keep_idx[r][kh][0 .. kept) = the kept = min(keep_len[r], ctx_len[r]) positions of largest
 *   weight, in ascending order; entries from kept to max_keep are set to -1, kept_len[r] = kept.  The first
 *   protect_first and the last protect_last positions rank above all others; equal weights are taken from the lowest
 *   position on; NaN ranks lowest.  ctx_len, keep_len, kept_len: device int32 [B]; weights as above; keep_idx: device
 *   int32 [B][Hkv][max_keep].  ctx_len is the length AFTER the step (call it behind hswa_step_advance); kept_len must be
 *   another array (HSWA_ERR_INVALID_ARG), and max_ctx_len at most 2^30 (HSWA_ERR_UNSUPPORTED).  A ctx_len outside
 *   [0, max_ctx_len] or a keep_len outside [0, max_keep] is recorded as HSWA_ERR_BOUNDS (index -1 / -2) and clamped.
 *
 * hswa_evict_compact: copies K and V of position keep_idx[r][kh][i], i < kept_len[r], to position i behind
 *   dst_block_table (device int32 [B][dst_max_blocks], another array, pages of the same pool), and its weight (weights
 *   and weights_out both given or both NULL; different arrays) to weights_out[r][kh][i].  Nothing else is written.  The
 *   caller guarantees that the destination pages are pages of no block table in use, this batch's included: source
 *   pages, which other requests may share, are only read.  Afterwards dst_block_table and kept_len take the place of
 *   block_table and ctx_len for this layer; run it for every Full layer of the step with equal kept_len, so that one
 *   ctx_len serves all.  On the SWA layers of a hybrid stack, a ctx_len cut below W - 1 hides the window's older keys:
 *   keep at least min(ctx_len, W - 1).  Rings and ring_head stay as they are; swa_valid_from holds positions and moves
 *   with ctx_len, to max(0, swa_valid_from - (ctx_len - kept_len)), by the caller.  Entry i of a compacted table is no
 *   longer token i, nor the same token for every head: such a request is no donor of a prefix, with its Full KV nor its
 *   masks.  Ids and positions out of range are recorded as HSWA_ERR_BOUNDS and the row is not copied. */
hswa_status hswa_attn_weights(hswa_handle* h, const hswa_layer* layer, const hswa_batch* batch, int32_t causal, const void* q,
                              const float* lse, float decay, float* weights, int64_t weights_stride, void* stream);
hswa_status hswa_evict_select(hswa_handle* h, int32_t batch, const int32_t* ctx_len, int32_t max_ctx_len, const float* weights,
                              int64_t weights_stride, const int32_t* keep_len, int32_t max_keep, int32_t protect_first,
                              int32_t protect_last, int32_t* keep_idx, int32_t* kept_len, void* stream);
hswa_status hswa_evict_compact(hswa_handle* h, const hswa_layer* layer, const hswa_batch* batch, const int32_t* keep_idx,
                               const int32_t* kept_len, int32_t max_keep, const int32_t* dst_block_table, int32_t dst_max_blocks,
                               const float* weights, int64_t weights_stride, float* weights_out, int64_t weights_out_stride,
                               void* stream);

/* A Full layer's cache in 4 bits (no paper counterpart: Sec. 2.2's decode is bound by the bytes of the cache, which this
 * makes 3.6 times fewer).  Values are e2m1 (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives), 16 neighbouring elements of a row
 * share an e4m3 scale, and a layer has one fp32 scale for K and one for V: an element stands for e2m1 * e4m3 * scale.
 *
 * Pool: uint8 [num_pages][2][Hkv][P * (D / 2 + D / 16)], 256-byte aligned.  A slab holds the P rows' values, D / 2 bytes each
 * (element 2i in the low half of byte i), and behind them the P rows' scales, D / 16 bytes each.  Block tables, lengths and
 * batches are those of the bf16 layers; SWA layers have no 4-bit form.  A layer of another head count, head dim or page size
 * than the handle's cannot be told from the pointer: it is the caller's to match.
 *
 * hswa_packed_append: rounds the step's rows into the cache, row i of request r at position ctx_len[r] + i.  A block of largest
 *   magnitude a gets the scale f = e4m3((a / s) / 6), at most 448, and its elements x the values e2m1(x / (f s)), at most 6 in
 *   magnitude; all roundings go to the nearest, ties to the even code.  Quotients are taken in fp32: with a scale s of at most 14
 *   significant bits the codes are those of exact arithmetic; with a longer one, where an exact quotient lies within 2^-22 (relative) of the
 *   middle between two codes, either may be held.  A block whose f rounds to 0 is held as zeros; infinities
 *   and NaN are held as finite values.  k_new, v_new: device bf16 [T][Hkv][D].
 * hswa_packed_read: the same rows back, k_out, v_out: device bf16 [T][Hkv][D], each element the value it stands for, rounded to fp32
 *   and then to bf16 (exact where the layer's scale is a power of two).  With ctx_len = 0 and n[r] a request's length it reads the whole cache;
 *   after an append it gives the chunk as later steps will see it.
 *   Both: a request's rows past max_q_len, its rows outside the block table or behind a page id out of range, and a ctx_len outside
 *   [0, max_ctx_len] are recorded as HSWA_ERR_BOUNDS and left out.  Pages that several requests share are the caller's to keep
 *   from being written by more than one.
 * hswa_packed_attn: softmax(sm_scale q K^T) V over the cache, any number of tokens per request.  causal != 0: token i sees
 *   j <= ctx_len[r] + i, so the step's rows have been appended before (the cache holds ctx_len[r] + n[r] positions, and a token
 *   sees its own row as the cache holds it).  causal == 0: every token sees all j < ctx_len[r] (an encoder's states).  A token
 *   that sees nothing gives zeros and an lse of minus infinity.  q: device bf16 [T][Hq][D]; out: device [T][Hq][D] in
 *   cfg.out_dtype; lse: device fp32 [T][Hq] or NULL.  Held values enter the products exactly; q enters them in fp16 after a
 *   power of two (exact but for elements below 2^-28 of the largest finite one of a KV head's rows in the step); probabilities enter the PV product as
 *   fp16 (each off by 2^-11 of itself or, below 2^-21 of the row's largest so far, by 2^-32 of that, at most), row sums and lse are taken over the
 *   fp32 values.  batch->q_indptr may be NULL (one token per request).  Slots behind a
 *   request's last row may hold anything.  Workspace: hswa_packed_workspace_need bytes, else HSWA_ERR_WORKSPACE; 256-byte
 *   aligned.  A request longer than max_ctx_len or max_q_len, with row offsets outside [0, total_q], or whose keys
 *   pass the block table, is recorded as HSWA_ERR_BOUNDS (index -1 / -2 / -2 / -3); what the bounds cover is computed, other rows
 *   of out and lse stay as they were.
 * All refuse a current device other than the handle's, scales that are not within [2^-64, 2^64], a block table that does not cover
 * max_ctx_len (HSWA_ERR_INVALID_ARG), and max_ctx_len + max_q_len above 2^30 (HSWA_ERR_UNSUPPORTED); hswa_packed_attn an sm_scale whose
 * product with k_scale is past fp32 (HSWA_ERR_INVALID_ARG); append and read 2^30 blocks of 16 or more at once and more than
 * 65535 KV heads (HSWA_ERR_UNSUPPORTED).
 *
 * hswa_packed_workspace_need: exact bytes for a call with these host-known fields; pure host arithmetic. */
typedef struct {
  void* pool;
  int64_t num_pages;
  float k_scale; /* fp32 scale of the layer's K */
  float v_scale; /* fp32 scale of the layer's V */
} hswa_packed_layer;

hswa_status hswa_packed_append(hswa_handle* h, const hswa_packed_layer* layer, const hswa_batch* batch, const void* k_new,
                               const void* v_new, void* stream);
hswa_status hswa_packed_read(hswa_handle* h, const hswa_packed_layer* layer, const hswa_batch* batch, void* k_out, void* v_out,
                             void* stream);
size_t hswa_packed_workspace_need(const hswa_handle* h, int32_t batch, int32_t total_q, int32_t max_q_len, int32_t max_ctx_len,
                                  int32_t causal);
hswa_status hswa_packed_attn(hswa_handle* h, const hswa_packed_layer* layer, const hswa_batch* batch, int32_t causal, const void* q,
                             void* out, float* lse, void* workspace, size_t workspace_bytes, void* stream);

/* Bookkeeping of pages on the device (paper Sec. 3.1.3: equal prefixes share physical pages).  ref[p] (device int32 [num_pages])
 * is the number of holders of page p: rows of block tables, and whatever the caller counts besides (a prefix cache).  A page
 * of count 0 is free; the lowest-numbered free pages are taken first, so results depend on the arguments alone.  Page ids are those
 * of block tables and hold for every layer's pool; P is the handle's page size.  held[r] is the number of pages of row r, the
 * first held[r] places of its table row.  Nothing is synchronised: counts and tables stay on the device.
 *
 * hswa_pages_fork: the tables of a step's rows from those of the step before, for beams, parallel samples, finished and new
 *   requests at once.  New row r continues old row parent[r] (in [0, rows_in), or -1: a new request) at len[r] tokens (0 for a new
 *   request, else at most held[parent] * P; fewer than the parent had takes tokens back), with room for need[r] tokens
 *   (held_out = ceil(max(len, need) / P)).  The len / P full pages are shared with the parent.  Of the places behind them, those
 *   whose page the parent alone holds (ref 1) and none of its children shares go on to its first child, the lowest r; every other
 *   place gets a fresh page.  Where that replaces a partly filled page, (copy_src[r], copy_dst[r]) is the pair to be copied in
 *   every layer's pool before the step writes (hswa_pages_copy), else -1, -1.  Old rows without a child give up their pages.
 *   Written: ref_out (device int32 [num_pages]), table_out (device int32 [rows_out][out_max_blocks], the
 *   first held_out[r] places of each row), held_out, copy_src, copy_dst (device int32 [rows_out]).  Pages given up by a call are
 *   free from the next call on, since its copies still read them.  If the free pages do not suffice, or a row's arguments are out
 *   of range, nothing is done: ref_out becomes a copy of ref, the other arrays stay as they were, and HSWA_ERR_BOUNDS is recorded
 *   (request -1, index = pages wanted, value = pages free; or request = row, index -1 for held, -2 for parent, len, need).  Page
 *   ids out of range are recorded and neither counted nor copied.  Workspace: hswa_pages_workspace_need bytes.
 *   On a hybrid stack these are the Full layers' pages.  A row's ring on the SWA layers is its own: one child takes over its parent's ring
 *   pages, every other child needs R of its own, filled by hswa_pages_copy on each SWA layer's pool (the pairs of the parent's and the
 *   child's ring_table entries, place by place) before the step writes.  ring_head goes with them, moved back (mod C) by as many slots
 *   as the child takes tokens back.  Copies of a ring that has been L tokens long, taken back or not, hold the keys from position L - C
 *   on, and a child at len tokens needs those from len - W + 1 on: from a row as long as it has been, C - W + 1 tokens at most.
 *
 * hswa_pages_compact: moves live pages into the lowest free ones, up to max_moves of them: while it lies below, the i-th lowest
 *   free page takes the i-th highest live one.  move_src[i], move_dst[i] (device int32 [max_moves]) are the pairs to be copied in
 *   every layer's pool, -1 behind the last; page_map (device int32 [num_pages]) gives every page's new number, for holders outside
 *   the tables; ref_out the counts under the new numbers; table_out (device int32 [rows][max_blocks], may be table)
 *   the first held[r] places of each row under them.  After all moves the live pages are 0 .. live - 1.
 *
 * hswa_pages_copy: page dst[i] of every pool becomes a copy of page src[i], i < pairs (device int32 arrays; -1, -1: no pair), in
 *   n_pools pools (host array of device pointers, 16-byte aligned) of num_pages pages of page_bytes bytes (a multiple of 16): bf16
 *   pools 4 * Hkv * P * D bytes, 4-bit pools 2 * Hkv * P * (D / 2 + D / 16).  No page may be the destination of two pairs, or of one
 *   and the source of another (the lists of the two calls above keep to that).  Ids out of range are recorded and not copied.
 *
 * All refuse a current device other than the handle's (HSWA_ERR_INVALID_ARG).  Fork and compact refuse more than 4096 rows, 2^23 pages
 * or 2^30 entries of a table (HSWA_ERR_UNSUPPORTED), and an output that is an input or another output, table_out of hswa_pages_compact
 * and its table apart (HSWA_ERR_INVALID_ARG); copy 2^31 pages or more, pages of more than 2^30 bytes, and as many pairs as make 2^31 pieces
 * of 4 KB of one pool (HSWA_ERR_UNSUPPORTED). */
size_t hswa_pages_workspace_need(const hswa_handle* h, int64_t num_pages);
hswa_status hswa_pages_fork(hswa_handle* h, int64_t num_pages, const int32_t* ref, int32_t* ref_out, int32_t rows_in,
                            const int32_t* held, const int32_t* table, int32_t max_blocks, int32_t rows_out, const int32_t* parent,
                            const int32_t* len, const int32_t* need, int32_t* table_out, int32_t out_max_blocks, int32_t* held_out,
                            int32_t* copy_src, int32_t* copy_dst, void* workspace, size_t workspace_bytes, void* stream);
hswa_status hswa_pages_compact(hswa_handle* h, int64_t num_pages, const int32_t* ref, int32_t* ref_out, int32_t rows,
                               const int32_t* held, const int32_t* table, int32_t max_blocks, int32_t* table_out, int32_t* page_map,
                               int32_t max_moves, int32_t* move_src, int32_t* move_dst, void* stream);
hswa_status hswa_pages_copy(hswa_handle* h, int32_t n_pools, void* const* pools, int64_t num_pages, int64_t page_bytes, int32_t pairs,
                            const int32_t* src, const int32_t* dst, void* stream);

/* SWA-aware prefix reuse helpers (paper Sec. 3.1.3 "SWA-Aware Prefix Cache Tree", Sec. 3.1.1 "Data movement",
 * Sec. 3.1.2 layerwise prefetch).
 *
 * hswa_window_safe_len: pure host arithmetic.  A donor matches a new request on its first match_len tokens; its
 * SWA KV survives only where swa_valid[i] != 0 (host array of at least match_len bytes).  Returns the largest hit
 * length L <= match_len such that every position in [max(0, L - (W - 1)), L) is valid, i.e. the cached keys the
 * next token's window needs are all there (0 is always safe; a NULL mask means nothing is valid).
 *
 * hswa_swa_window_gather / _scatter: move ONLY the W - 1 cached positions the next token's window needs between
 * the rings of an SWA layer and a compact buffer bf16 [B][W-1][2 (K,V)][Hkv][D]; entry j of request r is position
 * ctx_len[r] - (W - 1) + j.  Gather reads the rings (positions below 0 become zeros); scatter writes the ring
 * slots those positions map to under batch->ring_head / ring_table (positions below 0 are skipped) and touches
 * nothing else.  `buf` is device memory or pinned host memory (16-byte aligned): gather + scatter with a host
 * buffer is the offload / loadback of a request's SWA state, scatter into a fresh ring seeds it after a prefix
 * hit.  (W - 1) * 4 * Hkv * D bytes per request and layer move instead of the whole context.  Layer must be an
 * SWA layer (HSWA_ERR_INVALID_ARG otherwise); asynchronous on `stream`, so a copy stream can load layer l + 1
 * while layer l computes. */
int64_t hswa_window_safe_len(int64_t match_len, int32_t window, const uint8_t* swa_valid);
hswa_status hswa_swa_window_gather(hswa_handle* h, const hswa_layer* layer, const hswa_batch* batch, void* buf,
                                   void* stream);
hswa_status hswa_swa_window_scatter(hswa_handle* h, const hswa_layer* layer, const hswa_batch* batch, const void* buf,
                                    void* stream);

/* Out-of-window SWA release bookkeeping and dual-index matching (paper Sec. 3.1.3 items 2 and 3).
 *
 * State: swa_valid_from[r] (device int32 [B], caller-owned, starts at 0 for a fresh request, or at
 * max(0, ctx - (W - 1)) for a ring seeded with hswa_swa_window_scatter) is the first cached position of request
 * r whose SWA KV is still valid; the valid SWA positions of a live request are the suffix [swa_valid_from, ctx).
 *
 * hswa_swa_release, once per step AFTER hswa_step_advance: moves the boundary forward to ctx - C (the ring has
 * overwritten everything older) and, for requests with release[r] != 0 (device uint8 [B]; NULL: all), to
 * ctx - (W - 1): the paper's release events -- a prefill chunk completed, the request terminated, every N tokens
 * generated in decode -- drop everything the next token's window cannot reach, which keeps SWA use at window
 * magnitude.  Which event fired is the scheduler's knowledge, hence the flags.  The boundary never moves back.
 *
 * hswa_swa_valid_mask: the per-position SWA status a prefix-tree node records: mask[r][p] = 1 iff
 * swa_valid_from[r] <= p < ctx_len[r], for p < mask_stride (0 beyond ctx); mask is uint8 [B][mask_stride] in
 * device memory or pinned host memory.
 *
 * hswa_prefix_hit_len: pure host arithmetic.  A cached prefix matches a new request on its first match_len tokens;
 * its nodes carry per-token Full status (full_valid, host uint8, NULL: nothing valid) and SWA status (swa_valid, as
 * for hswa_window_safe_len).  Returns the largest L <= match_len such that every position in [0, L) has Full KV
 * (Full layers read all of them) and every position in [max(0, L - (W - 1)), L) has SWA KV.  Evicting the SWA part
 * of old segments on its own therefore keeps the prefix reusable; evicting a whole segment ends it there. */
hswa_status hswa_swa_release(hswa_handle* h, int32_t batch, const int32_t* ctx_len, const uint8_t* release,
                             int32_t* swa_valid_from, void* stream);
hswa_status hswa_swa_valid_mask(hswa_handle* h, int32_t batch, const int32_t* ctx_len, const int32_t* swa_valid_from,
                                int64_t mask_stride, uint8_t* mask, void* stream);
int64_t hswa_prefix_hit_len(int64_t match_len, int32_t window, const uint8_t* full_valid, const uint8_t* swa_valid);

/* Step advance, once per step after all layers (paper Sec. 3.1.1: one logical view over both pools -- every
 * layer of a step maps positions with the same lengths and ring heads, so they move once, after the last
 * layer): ctx_len[r] += n[r], ring_head[r] = (ring_head[r] + n[r]) mod C.  ctx_len, ring_head: device int32 [B], updated in place.  q_indptr: device or NULL (n = 1). */
hswa_status hswa_step_advance(hswa_handle* h, int32_t batch, int32_t* ctx_len, int32_t* ring_head,
                              const int32_t* q_indptr, void* stream);

/* Synchronises `stream`, copies the error word to info[4] = {status, request, index, value} (host), clears
 * it, and returns info[0] as a status (HSWA_OK when nothing was recorded). */
hswa_status hswa_get_async_error(hswa_handle* h, void* stream, int32_t info[4]);

const char* hswa_status_string(hswa_status s);

/* Work balance of mixed-length prefill batches (paper Sec. 5.3: requests whose cached prefixes differ a lot make
 * the ranks / blocks that got the long ones finish last; the paper buckets by length, inside one launch the
 * equivalent is the order in which blocks are handed out).
 *
 * hswa_set_prefill_order: order in which the Full-layer tile kernel of hswa_prefill_attn takes the (request,
 * 128-token tile) pairs of a batch.  Tile b of request r walks ceil(ctx[r] / 128) + b + 1 key tiles.
 *   0: request by request in batch order, tiles ascending;
 *   1: every request's last tile first, requests interleaved;
 *   2 (default): longest request first -- requests in descending order of their longest tile's work, the tiles of a
 *      request together (their blocks share K/V pages in L2) and longest first, so that the launch ends on the
 *      shortest tiles of the shortest request;
 *   3: globally longest tile first, whatever its request.
 * Orders 2 and 3 are computed on the device from ctx_len and q_indptr.  Results do not depend on the order.
 *
 * hswa_set_block_trace: debug aid.  With a device buffer int64 [capacity_blocks][4] set (NULL, 0 switches it off),
 * every non-empty block of that kernel writes {start, end (nanoseconds of the GPU's global timer), SM id,
 * request << 32 | tile} at its linear block index (x + gridDim.x * (y + gridDim.y * z)); blocks beyond the capacity write nothing.  The caller
 * zeroes the buffer first and reads it after synchronising: the idle tail of every SM follows from it. */
hswa_status hswa_set_prefill_order(hswa_handle* h, int32_t mode);
hswa_status hswa_set_block_trace(hswa_handle* h, int64_t* buf, int64_t capacity_blocks);

/* Read-bandwidth probe (no paper counterpart; a measuring aid).  Streams `bytes` of device memory at `buf`
 * (128-byte aligned, a multiple of 32 KB) through shared memory with the same kind of bulk copies the decode
 * kernels use and does nothing with them; timed by the caller with events, bytes / time is the practical ceiling
 * for a read-only HBM stream on this GPU, which the roofline of paper Sec. 2.2's memory-bound decode is judged
 * against next to the copy-based peak.  Asynchronous on `stream`. */
hswa_status hswa_probe_read_stream(hswa_handle* h, const void* buf, size_t bytes, void* stream);

/* Self-test of the bounded waits (no paper counterpart; failure detection of the library itself).  Every wait
 * on a pipeline barrier inside the kernels gives up after a fixed number of SM clocks, records
 * HSWA_ERR_TIMEOUT in the error word and lets the block finish.  This call launches a one-block kernel whose
 * consumer warp waits, with a limit of limit_clocks (1 .. 2e9), on a barrier that its producer never arms: the
 * wait runs out, the kernel returns normally, and hswa_get_async_error then reports {HSWA_ERR_TIMEOUT, -1, 0, 7}.
 * Nothing traps, nothing is left in flight, and the context stays usable. */
hswa_status hswa_selftest_wait_timeout(hswa_handle* h, int64_t limit_clocks, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* HSWA_H_ */
