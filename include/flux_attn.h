/*
 * flux_attn.h -- C ABI of libflux_attn.so: routed hybrid attention for one B200.
 *
 * The library runs the per-layer hot path of Flux Attention: a cached hard
 * routing bit per (request, layer) sends the layer to causal Full Attention
 * (Eq. 1) or to Sparse Attention over a condensed KV subset (Eq. 2; here the
 * streaming subset: an attention sink of `sink` leading positions plus a local
 * window of the `window` latest positions, query included), in prefill and in
 * autoregressive decode.
 *
 * General rules
 *  - Every entry point returns FLUX_OK (0) or a negative FLUX_E_* code; none
 *    throws, exits or prints.  flux_last_error() gives a message for the last
 *    failure on the calling thread.
 *  - The library allocates no device memory.  The caller owns every device
 *    buffer, including the workspace whose size flux_workspace_size() reports;
 *    a plan owns host memory only.
 *  - "device" pointers are CUDA global-memory addresses valid on the current
 *    device; "host" pointers are ordinary CPU addresses.  Each argument says
 *    which it is.  Device buffers must be 16-byte aligned.
 *  - Calls are asynchronous on `stream` (a cudaStream_t passed as void*, NULL
 *    for the default stream) unless stated otherwise.  Conditions that only the
 *    device can see (a mask byte outside {0,1}, a NaN logit, a context length
 *    outside [1, max_context], a wait that ran out) set bits in a device status
 *    word; flux_plan_status() synchronises the stream and returns them.
 *  - All tensors are bfloat16 unless stated otherwise; accumulation is fp32.
 *  - Layouts: Q and O rows are [n_q_heads][head_dim]; a KV cache of one
 *    (layer, request) is [rows][n_kv_heads][head_dim], token-major, so one
 *    token's keys of all heads are one contiguous 2*n_kv_heads*head_dim-byte row.
 *    Query head h reads KV head h / (n_q_heads / n_kv_heads).
 *  - Mask encoding (Sec. 3.1, "Deterministic Inference via Hard Routing"):
 *    1 = FA, 0 = SA.
 */
#ifndef FLUX_ATTN_H
#define FLUX_ATTN_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define FLUX_OK                   0
#define FLUX_E_INVALID_ARG       -1  /* null / misaligned pointer, bad index, bad size          */
#define FLUX_E_UNSUPPORTED_SHAPE -2  /* head_dim != 128, n_q_heads % n_kv_heads != 0, G > 16    */
#define FLUX_E_CAPACITY          -3  /* batch or length beyond what the plan was created for    */
#define FLUX_E_WORKSPACE         -4  /* workspace missing or too small                          */
#define FLUX_E_DEVICE_TIMEOUT    -5  /* a bounded device-side wait gave up                      */
#define FLUX_E_CUDA              -6  /* a CUDA runtime / driver call failed                     */
#define FLUX_E_DEVICE_FLAG       -7  /* device-side input check failed (see status bits)        */

/* bits of the device status word returned by flux_plan_status() */
#define FLUX_STATUS_BAD_MASK      1u   /* mask byte not 0/1                                     */
#define FLUX_STATUS_NAN_LOGIT     2u   /* routing logit is NaN                                  */
#define FLUX_STATUS_BAD_LENGTH    4u   /* ctx_len / pos outside [1, max_context]                */
#define FLUX_STATUS_WAIT_EXPIRED  8u   /* an mbarrier wait hit its iteration limit              */
#define FLUX_STATUS_NONFINITE     16u  /* a K or V entry to be stored in 8 bits is NaN or infinite */
#define FLUX_STATUS_BAD_POINTER   32u  /* an 8-bit cache's address is NULL or not 16-byte aligned */
#define FLUX_STATUS_BAD_PAGE      64u  /* a page table row or entry that cannot be: outside its range, listed twice, missing where it is needed, not counted */
#define FLUX_STATUS_NO_PAGES      128u /* a pool has run out of free pages                      */

#define FLUX_KV_FULL        0  /* every layer's cache holds every position: row = position          */
#define FLUX_KV_COMPACT_SA  1  /* an SA layer's cache holds sink + window rows only (Sec. 3.3)      */

typedef struct {
    int32_t n_layers;
    int32_t n_q_heads;
    int32_t n_kv_heads;
    int32_t head_dim;       /* must be 128                                                      */
    int32_t sink;           /* S >= 0: leading positions every SA query keeps                   */
    int32_t window;         /* W >= 1: latest positions an SA query keeps, itself included      */
    float   softmax_scale;  /* 0 selects 1/sqrt(head_dim); Eq. 1 leaves the scale out           */
    int32_t max_batch;      /* largest B any call will pass                                     */
    int32_t max_context;    /* largest context length; every full cache has >= this many rows   */
    int32_t kv_layout;      /* FLUX_KV_FULL or FLUX_KV_COMPACT_SA                               */
} flux_config;

typedef struct flux_plan flux_plan; /* opaque host object */

/* Plan life cycle.  Creating a plan validates the configuration and queries the
 * current device (SM count, shared memory); it launches nothing.  Host memory
 * only; flux_plan_destroy frees it.  *plan is set to NULL on failure. */
int flux_plan_create(const flux_config *cfg, flux_plan **plan);
int flux_plan_destroy(flux_plan *plan);

/* Device workspace (split-K partials, status word, debug records, staging for
 * the *_host calls, 21 MB of accumulators for flux_attn_prefill_packed).  bytes_out (host) receives the size for this configuration.
 * The caller allocates it (256-byte aligned), zero-fills it once, and hands it
 * over; it must stay valid and untouched by others while the plan is in use. */
int flux_workspace_size(const flux_config *cfg, size_t *bytes_out);
int flux_plan_set_workspace(flux_plan *plan, void *workspace /*device*/, size_t bytes);

/* Layer Router front end (Sec. 3.1, "Architecture and Feature Extraction"; Appendix D.1): from
 * the layer's query tensor x_Q to the routing logits of one (request, layer).
 *   f  = concat(mean over tokens of q_first, mean over tokens of q_last)      [2*n_q_heads*head_dim]
 *        (Prefill-Suffix Pooling; index = segment*Hq*D + head*D + channel)
 *   h1 = silu(w_enc1 f + b_enc1);  u = w_enc2 h1 + b_enc2                      Context Encoder
 *   h2 = silu(w_head1 u + b_head1); (pi_FA, pi_SA) = w_head2 h2 + b_head2      Router Head
 * The paper names these stages but not the pooling operator, the widths or the activation; the
 * token mean and silu(x) = x / (1 + exp(-x)) are this library's choice.
 *   q_first, q_last  bf16 [n_first][n_q_heads][head_dim] and [n_last][..][..], device: the first
 *                    and the last prompt tokens of x_Q (the paper pools 100 + 100; shorter
 *                    prompts pass min(100, n) tokens each, the two may overlap).  n_* >= 1.
 *   w                host struct of device pointers: weights bf16 row-major [out][in], biases
 *                    fp32; widths enc_dim (E) and head_hidden (R) multiples of 8, <= 4096;
 *                    w_enc1 [E][2*Hq*D], w_enc2 [E][E], w_head1 [R][E], w_head2 [2][R] (row 0 = FA).
 *   logits_out       fp32 [2] on the device, 8-byte aligned, e.g. the (request, layer) slot of the
 *                    [B][n_layers][2] array later given to flux_router_apply.
 * One launch on `stream` (pooling + four matrix-vector products, fp32 accumulation, a fixed
 * summation order); scratch is in the workspace, so calls for different layers must be
 * stream-ordered.  Cost does not depend on the prompt length.  The launch may begin while the
 * kernel before it in the stream is still draining, and reads the WEIGHTS AND BIASES (nothing
 * else) before that kernel has finished: the work enqueued immediately before this call must not
 * be what writes them.  The kernel's CTAs (one per SM) wait for one another between stages; the
 * waits are bounded (about a second, then FLUX_STATUS_WAIT_EXPIRED in the status word and
 * unspecified logits), which only a kernel of another stream that holds SMs for that long can
 * cause.  Errors: NULL / misaligned pointers, n_* < 1 -> FLUX_E_INVALID_ARG; widths
 * not multiples of 8 -> FLUX_E_UNSUPPORTED_SHAPE; widths > 4096 -> FLUX_E_CAPACITY. */
typedef struct {
    int32_t enc_dim;       /* E */
    int32_t head_hidden;   /* R */
    const void *w_enc1;  const float *b_enc1;
    const void *w_enc2;  const float *b_enc2;
    const void *w_head1; const float *b_head1;
    const void *w_head2; const float *b_head2;
} flux_router_weights;
int flux_router_forward(flux_plan *plan, const flux_router_weights *w, const void *q_first, int32_t n_first,
                        const void *q_last, int32_t n_last, float *logits_out /*device*/, void *stream);

/* Hard routing, once per request batch at prefill; the result is cached for all
 * decode steps (Sec. 3.1 "Deterministic Inference via Hard Routing", Sec. 3.3).
 *   logits       fp32 [B][n_layers][2], FA logit first; device or host memory;
 *                ignored when mask_or_null is given.
 *   mask_or_null uint8 [B][n_layers] ready-made decisions (device or host), or NULL.
 *   mask_out     uint8 [B][n_layers], device; receives 1 where pi_FA >= pi_SA (a tie
 *                keeps FA), else 0.  The plan remembers this pointer: later calls
 *                read the routing decision from it, so it must stay alive.
 * Host inputs are validated on the host (NaN logit or mask byte outside {0,1}
 * -> FLUX_E_INVALID_ARG, nothing launched) and staged through the workspace;
 * device inputs are checked by the kernel (status bits).  B <= max_batch. */
int flux_router_apply(flux_plan *plan, const float *logits, const uint8_t *mask_or_null,
                      int32_t B, uint8_t *mask_out, void *stream);

/* Prefill of one layer for one request (Eq. 1 or Eq. 2 by mask[req][layer]),
 * causal.  Query rows sit at absolute positions q_start .. q_start+Nq-1 (chunked
 * prefill, Appendix D.3 "chunk size"); k, v hold positions 0 .. q_start+Nq-1 as
 * [rows][n_kv_heads][head_dim] with row = position (a FULL-layout cache or the
 * projection output itself).
 *   q, out   [Nq][n_q_heads][head_dim], device.    k, v  device, read only.
 * Nq == 0 is a successful no-op.  q_start + Nq <= max_context. */
int flux_attn_prefill(flux_plan *plan, int32_t layer, int32_t req, const void *q,
                      const void *k, const void *v, int32_t q_start, int32_t Nq,
                      void *out, void *stream);

/* Prefill of one request under a block mask: Sparse Attention (Eq. 2) whose condensed key subset
 * is given in blocks of 64 positions, the unit in which the sparse kernels the paper runs select
 * keys (Appendix D.3, "block size"; Sec. 4.1 names the block patterns).  Query position i attends
 * to { j <= i : block_mask[i / 64][j / 64] != 0 }: causality still holds inside a kept block.
 *   block_mask  uint8 [n_q_blocks][n_kv_blocks], device, row-major; rows are ABSOLUTE query blocks
 *               (row (q_start + r) / 64 serves chunk row r), so one matrix serves every chunk;
 *               entries beyond the diagonal are ignored.  n_kv_blocks <= 4096 (else FLUX_E_CAPACITY).
 *   q, out      [Nq][n_q_heads][head_dim], device; k, v as in flux_attn_prefill.
 *   q_start     multiple of 64.
 * Independent of the routing decision (no layer / request arguments).  A query whose mask row
 * keeps no block up to its own gets a zero output row and raises FLUX_STATUS_BAD_MASK. */
int flux_attn_prefill_blocks(flux_plan *plan, const void *q, const void *k, const void *v,
                             int32_t q_start, int32_t Nq, const uint8_t *block_mask,
                             int32_t n_kv_blocks, void *out, void *stream);

/* Prefill of one layer for several requests in one launch (Eq. 1 or Eq. 2 by mask[b][layer], causal): the prompts, or
 * prompt chunks, of requests 0 .. B-1 packed row after row.  The paper runs batch 1 (Appendix C.3); this
 * is flux_attn_prefill for the admission batches a server has.
 *   q, out   [q_rows[B]][n_q_heads][head_dim]; request b's new tokens are rows q_rows[b] .. q_rows[b+1]-1.
 *   k, v     [k_rows[B]][n_kv_heads][head_dim]; request b's keys, position 0 first, are rows k_rows[b] .. k_rows[b+1]-1.
 *            Its new tokens are the last of these positions (equal counts: a whole prompt; more keys than new tokens: a
 *            chunk whose earlier positions are already there).
 *   q_rows, k_rows  HOST int32 [B + 1], non-decreasing, first entry >= 0; read during the call.  k_rows may equal q_rows.
 *            A request without new tokens is skipped (its keys are not looked at).
 *   q_stride, k_stride, v_stride  elements from one row of q / k / v to the next (multiples of 8, at least heads *
 *            head_dim): slices of one fused projection output need no copy.  out rows are contiguous.
 * Items that few rows leave long are cut along the keys and added up in the workspace, and work is drawn from a counter there: calls
 * of one plan (and graphs captured from it) must not overlap.  B <= the routed batch; keys per request <= max_context.  Rows outside the requests' ranges are neither read into any
 * result nor written.  What stands in another request's rows, NaN and infinities included, does not reach a request's
 * output.  Inside one request a non-finite V entry reaches, in its channel and the query heads of its KV head, also rows that mask it (0 x inf): all rows of
 * every query tile that walks the 128-position key tile it stands in.  Query tiles are 128 rows counted from the request's first new row (in
 * the last head of an odd group two of them go together); one walks the key tiles up to its last row's position, in a
 * sparse request those of the sink and those from its first row's window on.  The calls for single requests do the same.
 * Dispatch records: one per request (of a skipped request: mode -1).  Errors: a request with more new tokens than keys,
 * decreasing row bounds, misaligned pointers (out: 32 bytes) or strides -> FLUX_E_INVALID_ARG; too long -> FLUX_E_CAPACITY. */
int flux_attn_prefill_packed(flux_plan *plan, int32_t layer, int32_t B, const void *q, const void *k, const void *v,
                             int64_t q_stride, int64_t k_stride, int64_t v_stride, const int32_t *q_rows /*host*/,
                             const int32_t *k_rows /*host*/, void *out, void *stream);

/* KV cache in 8 bits: half the bytes of every decode step, twice the context in the same memory.  (The paper keeps bf16
 * caches; Sec. 3.3's retention rule is unchanged.)  Each cache -- K and V of one (layer, request) -- is one opaque device
 * buffer of flux_kvq_cache_size() bytes, 16-byte aligned (128 is better); it need not be cleared.  Positions are held in blocks of 16 with
 * one fp32 scale per block and head:
 *   FLUX_KVQ_E4M3  scale = the smallest power of two with max |x| <= 448 scale, code = x / scale rounded to e4m3 (to nearest,
 *                  ties to even): relative error of an entry up to 2^-4, whatever the other channels' size (beyond 448 * 2^119 entries
 *                  saturate)
 *   FLUX_KVQ_INT8  scale = max |x| / 127 rounded to fp32, code = x / scale rounded to an integer (ties to even): absolute error
 *                  up to max |x| / 254; about a third of e4m3's error on rows without outlying channels
 * (scales are at least 2^-100: of such a block entries up to 2^-110, in int8 2^-101, become 0).  The newest block stays in bf16 until it is complete, so what a
 * cache holds depends on the positions' values alone, not on how they arrived (each position still has to be stored once, in order).  A NaN or infinite entry is stored as 0 and
 * raises FLUX_STATUS_NONFINITE.  In the FLUX_KV_COMPACT_SA layout a sparse layer's cache holds sink + window (rounded up to
 * 64-position tiles).
 *
 * flux_kvq_cache_size: bytes of one cache.  compact: 1 for a sparse layer's cache under FLUX_KV_COMPACT_SA, else 0;
 * max_len: the longest length the cache will hold. */
#define FLUX_KVQ_E4M3 0
#define FLUX_KVQ_INT8 1
int flux_kvq_cache_size(const flux_config *cfg, int32_t compact, int32_t max_len, size_t *bytes_out);

/* Store rows of B requests into their caches: whole prompts, chunks, or single tokens of a decode step.
 *   k, v        [total_rows][n_kv_heads][head_dim], device, row strides in elements (multiples of 8).
 *   row_start   int32 [B + 1], device: request b's rows are row_start[b] .. row_start[b+1]-1 (none: skipped).
 *   pos         int32 [B], device: position of request b's first row = tokens the cache holds already.  The cache must have
 *               been filled up to there by this call (the begun block's rows are read back from it); storing the
 *               tokens of its newest block (complete or not) again, from any place in that block on, is allowed.  Requests have caches of their own
 *               (reading shared ones is fine); a cache is read with the fmt it was filled with.
 * Rows outside [0, total_rows) or positions from max_context on raise FLUX_STATUS_BAD_LENGTH and nothing of that request is
 * stored; a cache address that is NULL or misaligned raises FLUX_STATUS_BAD_POINTER likewise (here and in the calls below). */
int flux_kvq_store(flux_plan *plan, int32_t layer, int32_t B, int32_t fmt, const void *k, const void *v, int64_t k_stride,
                   int64_t v_stride, int32_t total_rows, const int32_t *row_start, const int32_t *pos, void *const *k_caches,
                   void *const *v_caches, void *stream);

/* The values a cache stands for, as bf16 rows (code x scale in fp32, rounded once): e.g. the earlier positions for a chunked
 * prefill.  Arguments as in flux_kvq_store; ctx_len int32 [B], device: tokens each cache holds; positions pos[b] .. must lie
 * below it (else FLUX_STATUS_BAD_LENGTH, nothing written for that request).  Positions a compact cache has dropped give zeros. */
int flux_kvq_load(flux_plan *plan, int32_t layer, int32_t B, int32_t fmt, const void *const *k_caches, const void *const *v_caches,
                  const int32_t *ctx_len, int32_t total_rows, const int32_t *row_start, const int32_t *pos, void *k_out, void *v_out,
                  void *stream);

/* flux_attn_decode over 8-bit caches: same arguments, modes, dispatch records and treatment of inactive requests; any batch up to
 * the routed one, one launch whose CTAs never wait for each other.  ctx_len[b] must be the number of tokens stored in request b's
 * caches; above max_context it raises FLUX_STATUS_BAD_LENGTH and gives a zero row.  (B * n_kv_heads * max_context / 32 has to stay
 * below 2^30, else FLUX_E_CAPACITY.)  V may have any magnitude: blocks of one request may differ by all the range of their scales, and outputs keep
 * their precision down to about 2^-97.  The split-K partials and arrival counters are in
 * the workspace: calls of one plan (and graphs captured from it) must not overlap.  Records and flux_debug_touched bits are positions.
 *
 * flux_attn_decode_step_kvq: flux_kvq_store of one token per request at position ctx_len - 1 and flux_attn_decode_kvq in one launch
 * (the caches hold the same; the outputs can differ in rounding); requests with ctx_len <= 0 are skipped.  k_new, v_new [B][n_kv_heads][head_dim]. */
int flux_attn_decode_kvq(flux_plan *plan, int32_t layer, int32_t B, int32_t fmt, const void *q, const void *const *k_caches,
                         const void *const *v_caches, const int32_t *ctx_len, void *out, void *stream);
int flux_attn_decode_step_kvq(flux_plan *plan, int32_t layer, int32_t B, int32_t fmt, const void *q, const void *k_new,
                              const void *v_new, void *const *k_caches, void *const *v_caches, const int32_t *ctx_len, void *out,
                              void *stream);

/* Norm of every query and key head and rotation by its position, in one pass (the paper's backbones do both between the
 * projections and attention; the calls above take Q and K after them).  For each head of head_dim channels
 *   y = x (w + weight_offset) / sqrt(mean(x^2) + eps)           left out for q, k whose weight is NULL
 *   (y_a, y_b) -> scale (y_a cos t - y_b sin t, y_b cos t + y_a sin t),   t = position * inv_freq[i]
 * over the pairs i = 0 .. rotary_dim / 2 - 1, channels (i, i + rotary_dim / 2), or (2 i, 2 i + 1) when interleaved; channels from
 * rotary_dim on are normed only.  fp32, rounded once.  (The mean of squares is formed in fp32: entries beyond 2^60 overflow it, and what is
 * smaller than 2^-60 is lost to it, which matters only to rows of nothing else with an eps below 2^-100.)
 *   q_weight, k_weight  bf16 [head_dim], device, 16-byte aligned, or NULL.
 *   freqs               uint64 [rotary_dim / 2], device: inv_freq / 2 pi as a fraction of a turn in units of 2^-64 (flux_rope_freqs),
 *                       so that angles are exact at any position.  May be NULL when rotary_dim is 0.
 *   rotary_dim          multiple of 16, 0 .. head_dim.     scale  factor of sine and cosine (1 for the plain rotation).
 * flux_rope_freqs: host function, inv_freq (radians per position, whatever scaling went into them) to freqs, n <= head_dim / 2 each. */
typedef struct {
    const void *q_weight, *k_weight;
    const uint64_t *freqs;
    float eps, weight_offset, scale;
    int32_t rotary_dim, interleaved;
} flux_rope;
int flux_rope_freqs(const double *inv_freq /*host*/, int32_t n, uint64_t *freqs_out /*host*/);

/* Rows to rows: q [n_rows][n_q_heads][head_dim], k [n_rows][n_kv_heads][head_dim], row strides in elements (multiples of 8); pos
 * int32 [n_rows], device, any value.  q or k may be NULL (left out); an output may be its input (same address and stride),
 * but not overlap it otherwise. */
int flux_qk_norm_rope(flux_plan *plan, const flux_rope *rope, const void *q, const void *k, int64_t q_stride, int64_t k_stride,
                      int32_t n_rows, const int32_t *pos, void *q_out, void *k_out, int64_t q_out_stride, int64_t k_out_stride,
                      void *stream);

/* Paged KV cache: the K and V rows of a layer in pages of page_size positions that requests hold through a table, so that no request
 * needs room for its longest length, requests share the pages of a common prefix, and a sparse request keeps only the pages of its
 * sink and window.  (The paper keeps one contiguous cache per request.)  Position p of request b is row p mod page_size of page
 * table[b * max_pages + p / page_size]; FLUX_PAGE_NONE marks positions that are not held.  A contiguous FULL cache is a pool whose table
 * counts upwards.  kv_layout plays no part here.
 *   k, v   bf16 [n_pages][page_size][n_kv_heads][head_dim], device, 16-byte aligned.
 *   table  int32 [B][max_pages], device.  page_size: 16, 32, 64, 128 or 256; n_pages <= 2^24; max_pages * page_size <= 2^30.
 * Tables may be one per layer (sparse layers then release what they do not need) or shared by several layers.
 *
 * flux_paged_store: rows into their pages, with norm and rotation by the row's own position on the way when rope is given.
 *   k, v        [total_rows][n_kv_heads][head_dim], row strides in elements (multiples of 8); q likewise or NULL.
 *   row_start   int32 [B + 1], device: request b's rows are row_start[b] .. row_start[b+1]-1, in order of the requests.
 *   pos         int32 [B], device: position of request b's first row.
 *   q_out, k_out  [total_rows][heads][head_dim], contiguous: normed and rotated query rows (with q, which needs a rope), and the key
 *               rows as they are stored (or NULL), e.g. for flux_attn_prefill_packed.  Only rows of requests are written.
 * Rows at FLUX_PAGE_NONE are not stored (a sparse request drops them); an entry outside the pool raises FLUX_STATUS_BAD_PAGE.  Row bounds
 * outside [0, total_rows] or positions from min(max_context, max_pages * page_size) on raise FLUX_STATUS_BAD_LENGTH, and nothing of that
 * request is stored.  A page that several rows of the table hold is overwritten for all of them: see flux_pages_reserve.
 *
 * flux_paged_load: positions pos[b] .. of requests of ctx_len[b] tokens as rows (e.g. the earlier positions for a prompt
 * chunk); positions must lie below ctx_len (else FLUX_STATUS_BAD_LENGTH, nothing written for that request), positions not held give zeros. */
#define FLUX_PAGE_NONE (-1)
typedef struct {
    void *k, *v;
    const int32_t *table;
    int32_t n_pages, page_size, max_pages;
} flux_pages;
int flux_paged_store(flux_plan *plan, int32_t B, const flux_rope *rope, const void *q, const void *k, const void *v, int64_t q_stride,
                     int64_t k_stride, int64_t v_stride, int32_t total_rows, const int32_t *row_start, const int32_t *pos,
                     const flux_pages *pages, void *q_out, void *k_out, void *stream);
int flux_paged_load(flux_plan *plan, int32_t B, const flux_pages *pages, const int32_t *ctx_len, int32_t total_rows,
                    const int32_t *row_start, const int32_t *pos, void *k_out, void *v_out, void *stream);

/* flux_attn_decode over paged caches: same modes, dispatch records and treatment of inactive requests; any batch up to the
 * routed one, one launch whose CTAs never wait for each other.  q rows may be strided (elements, a multiple of 8); out is contiguous.
 * Positions a request does not keep are not read, so whatever stands in them, or behind the last position of a page, does no harm.  A
 * non-finite entry of V at a kept position makes its channel of the head's rows non-finite (an infinity may become NaN, as weights are two
 * numbers of either sign).  A NaN in K makes the head's rows non-finite; an infinity does so in rows whose query entry has its sign, and
 * in rows of the other sign the score is -inf, so the position has weight 0 (a row of nothing but such scores is a zero row).  In the step
 * with a rope query rows are two numbers, possibly of different sign, so there an infinity in K can make rows of either sign non-finite.
 * A non-finite entry of a query row concerns that row alone: it is non-finite, or zero where all its scores are -inf.
 * A kept position whose page is FLUX_PAGE_NONE or outside the pool counts as masked and raises FLUX_STATUS_BAD_PAGE (a request without
 * any position left: a zero row).  ctx_len above max_context or max_pages * page_size raises FLUX_STATUS_BAD_LENGTH and gives a zero row.
 * (B * n_kv_heads * max_context / 16 has to stay below 2^30, else FLUX_E_CAPACITY.)  Split-K partials and arrival counters are in the
 * workspace, shared with the 8-bit decode: calls of one plan (and graphs captured from it) must not overlap.  Records and
 * flux_debug_touched bits are positions.
 *
 * flux_attn_decode_step_paged: flux_paged_store of one token per request at position ctx_len - 1 (rope may be NULL) and
 * flux_attn_decode_paged in one launch, from the projections to the output: q, k_new, v_new are rows of request b at b * stride, as they
 * come out of the projection when rope is given.  The pages hold the same as after the two calls; outputs can differ in rounding.
 * The page of position ctx_len - 1 must be there and be the request's own (flux_pages_reserve); if it is not there, the token is
 * lost and FLUX_STATUS_BAD_PAGE raised.  Both calls take launch overlap (flux_plan_set_launch_overlap): of the pages the kernel before may
 * only write positions ctx_len - 1 and ctx_len - 2 (a store or a step of one of the newest two tokens qualifies), and tables count as
 * pointer tables.  The page calls below write both; the first paged decode behind page calls of the same plan in a stream therefore
 * waits for them like without overlap.  Behind those of another plan, or those that a replayed graph ends with, it does not (a plan notes
 * its page calls when they are enqueued or captured): put the setting off, or a kernel between them. */
int flux_attn_decode_paged(flux_plan *plan, int32_t layer, int32_t B, const void *q, int64_t q_stride, const flux_pages *pages,
                           const int32_t *ctx_len, void *out, void *stream);
int flux_attn_decode_step_paged(flux_plan *plan, int32_t layer, int32_t B, const flux_rope *rope, const void *q, const void *k_new,
                                const void *v_new, int64_t q_stride, int64_t k_stride, int64_t v_stride, const flux_pages *pages,
                                const int32_t *ctx_len, void *out, void *stream);

/* Bookkeeping of a pool, on the device: nothing is read back, so a decode step with forked requests is one captured graph.
 *   table    int32 [n_rows][max_pages]: one row per request, or per (layer, request).
 *   refs     int32 [n_pages], 16-byte aligned: table entries that hold a page; 0: the page is free.  All entries FLUX_PAGE_NONE and
 *            all refs 0 is an empty pool.
 *   slabs    device array of n_slabs device addresses (16-byte aligned): every buffer in which page p is bytes [p * page_bytes,
 *            (p + 1) * page_bytes), page_bytes = page_size * n_kv_heads * 256 -- K and V pools of each layer the table serves.
 *   scratch  flux_pages_scratch_size() bytes, 16-byte aligned, no contents kept between calls.
 * A call lists up to 4096 rows (rows: int32 [n], device; NULL: rows 0 .. n - 1 where that is allowed).  Calls on one pool must not
 * overlap.  What a call does depends on its arguments alone, not on how the GPU schedules it: free pages are given out lowest first, in
 * the order of the list.  A listed row outside the table raises FLUX_STATUS_BAD_PAGE, and so does a row listed twice to be reserved or as
 * dst of a fork; a length that cannot be raises FLUX_STATUS_BAD_LENGTH.  Such entries of the list are left out (of a row listed twice, the
 * later ones).  flux_pages_release takes a row as often as it is listed, each time with that range.
 *
 * flux_pages_reserve  makes the pages of positions len[i] .. new_len[i] - 1 row rows[i]'s own, so that they can be written: missing ones are
 *   taken from the free pages; one that other rows hold too is replaced by a free page, into which the positions below len[i] that it
 *   holds are copied in all slabs.  If everyone who holds a page is listed and begins to write inside it, the last of them keeps it.
 *   Rows are served in order until the pages run out: that row and those behind it stay as they were and raise
 *   FLUX_STATUS_NO_PAGES.  granted (int32 [n], device, or NULL): 1 where the row was served.  Entries outside the pool or without a
 *   count raise FLUX_STATUS_BAD_PAGE, and the row is left out.
 * flux_pages_fork     row dst[i] lets go of its pages and takes the pages of row src[i] that hold positions below len[i]; all i at once
 *   (every source is read before any row is written), so beams may be permuted.  What a source has released the new row lacks too: a
 *   sparse request is forked at its own length, or where the pages of the window before len[i] are still held.  Entries outside the
 *   pool or without a count raise FLUX_STATUS_BAD_PAGE: the new row lacks those of its source, and letting go of them counts nothing.
 * flux_pages_release  gives up the pages of row rows[i] whose positions all lie in [begin[i], end[i]): everything (0, INT32_MAX), what a
 *   sparse request at length ctx_len does not need (sink, ctx_len - window), what was written beyond a length (length, INT32_MAX).
 * flux_pages_compact  moves the pages in use, in all slabs, to page numbers 0 .. used - 1 and corrects the table: those that lie beyond, in
 *   order, go to the free pages below, in order.  map_out (int32 [n_pages], device, or NULL): where a page is now, FLUX_PAGE_NONE for a
 *   free one; used_out (int32, device, or NULL).  Entries that hold a free page or none of the pool are taken out and raise
 *   FLUX_STATUS_BAD_PAGE. */
typedef struct {
    int32_t *table, *refs;
    void *const *slabs;
    void *scratch;
    int32_t n_rows, max_pages, n_pages, page_size, n_slabs;
} flux_page_pool;
int flux_pages_scratch_size(const flux_page_pool *pool, size_t *bytes_out);
int flux_pages_reserve(flux_plan *plan, const flux_page_pool *pool, int32_t n, const int32_t *rows, const int32_t *len,
                       const int32_t *new_len, int32_t *granted, void *stream);
int flux_pages_fork(flux_plan *plan, const flux_page_pool *pool, int32_t n, const int32_t *src, const int32_t *dst, const int32_t *len,
                    void *stream);
int flux_pages_release(flux_plan *plan, const flux_page_pool *pool, int32_t n, const int32_t *rows, const int32_t *begin,
                       const int32_t *end, void *stream);
int flux_pages_compact(flux_plan *plan, const flux_page_pool *pool, int32_t *map_out, int32_t *used_out, void *stream);

/* Sparse-decode KV retention after prefill (Sec. 3.3: a sparse layer keeps only
 * the rows its kernel needs).  Copies, for one (layer, request), the rows of
 * k_src/v_src ([n][n_kv_heads][head_dim], row = position) that decode will need
 * into the layer's cache: all n rows for an FA layer or the FULL layout; for an
 * SA layer in the COMPACT_SA layout rows [0,S) to slots [0,S) and rows
 * [max(S,n-W), n) to slot S + ((position - S) mod W).  All pointers device. */
int flux_kv_retain(flux_plan *plan, int32_t layer, int32_t req, const void *k_src,
                   const void *v_src, int32_t n, void *k_cache, void *v_cache, void *stream);

/* Append one new token per request to the caches of one layer (Sec. 3.3).
 *   k_new, v_new       [B][n_kv_heads][head_dim], device.
 *   k_caches, v_caches device arrays of B device pointers (this layer's cache of
 *                      each request).
 *   pos                int32 [B], device: position being written (= context length
 *                      before the append).  pos < 0 skips the request.
 * FA layers and the FULL layout write row pos; SA layers in COMPACT_SA write
 * slot pos (pos < S) or S + ((pos - S) mod W). */
int flux_kv_append(flux_plan *plan, int32_t layer, int32_t B, const void *k_new,
                   const void *v_new, void *const *k_caches, void *const *v_caches,
                   const int32_t *pos, void *stream);

/* One decode step of one layer for the whole batch: one query row per request at
 * position ctx_len-1 (its K, V already appended).  FA requests stream the whole
 * cache, SA requests only their sink + window rows (Appendix C.3); one launch serves
 * mixed modes, split over all SMs in equal-byte spans, followed by a combine pass (small
 * batches: one launch does both, see flux_debug_decode_kernel).
 *   q, out    [B][n_q_heads][head_dim], device.
 *   k_caches, v_caches  device arrays of B device pointers.
 *   ctx_len   int32 [B], device: context length including the new token;
 *             <= 0 marks an inactive request (its output row is zero-filled). */
int flux_attn_decode(flux_plan *plan, int32_t layer, int32_t B, const void *q,
                     const void *const *k_caches, const void *const *v_caches,
                     const int32_t *ctx_len, void *out, void *stream);

/* flux_kv_append and flux_attn_decode of one layer in one launch (Sec. 3.3: the new token's K, V
 * join the cache, then the token attends): the kernel stores k_new / v_new at position
 * ctx_len - 1 of each request's cache (ring slot for a compact sparse cache) and reads that one
 * row from k_new / v_new instead of the cache, so no second kernel and no ordering between the
 * two is needed.  Same results as the two calls with pos = ctx_len - 1.  At small batches the
 * saved launch is a visible part of a decode step.
 *   k_new, v_new  [B][n_kv_heads][head_dim], device.   Everything else as in flux_attn_decode;
 *   requests with ctx_len <= 0 are skipped (nothing stored, zero output row). */
int flux_attn_decode_step(flux_plan *plan, int32_t layer, int32_t B, const void *q,
                          const void *k_new, const void *v_new, void *const *k_caches,
                          void *const *v_caches, const int32_t *ctx_len, void *out, void *stream);

/* Head-level sparsity, the alternative the paper argues against (Sec. 2.3 "Motivational
 * Observations", Fig. 1(b); Appendix C.3 "Implementation of Sparsity Baselines"): inside ONE layer
 * some KV heads (with their query-head groups) attend densely and the others keep only sink +
 * window.  Same arithmetic as flux_attn_decode, but the mode comes per (request, KV head) from
 * head_mask instead of the cached layer mask, so the routed stack and a head-level stack of the
 * same KV byte budget can be timed on the same kernel.  The request is walked over its whole
 * length if any of its heads is dense; warps that own a sparse head read only its sink + window
 * rows and idle for the rest of the walk, and the dense heads' rows are 256-byte pieces of the
 * token-major cache rows -- the fragmented access and the intra-layer imbalance the paper describes.
 *   head_mask  uint8 [B][n_kv_heads] on the device: 1 = dense (Eq. 1), 0 = sink + window (Eq. 2);
 *              other values set FLUX_STATUS_BAD_MASK and count as dense.
 *   other arguments as flux_attn_decode; caches must be in the FLUX_KV_FULL layout
 *   (else FLUX_E_UNSUPPORTED_SHAPE).  No routing call is needed beforehand. */
int flux_attn_decode_heads(flux_plan *plan, int32_t B, const void *q, const void *const *k_caches,
                           const void *const *v_caches, const int32_t *ctx_len,
                           const uint8_t *head_mask /*device*/, void *out, void *stream);

/* Decode step for callers that cannot allocate device memory at all.  (The paper
 * has no counterpart: this is a packaging variant of flux_attn_decode, not part of
 * the method.)  Who needs it: code that runs inside a host program which owns all
 * device memory and passes in only the operator's own tensors, and loops that may
 * not risk the device-wide synchronisation an allocation can cause.  The split-K
 * scratch that flux_attn_decode keeps in the caller's workspace sits here in a
 * fixed array of about 9.6 MB inside the library image, held on every GPU the
 * process uses until it exits.  No plan and no workspace are needed; the call
 * makes no cudaMalloc / cudaFree and uses no allocating library routine.
 *   cfg        shapes as for flux_plan_create (max_batch is ignored).
 *   mask       uint8 [B][n_layers], device: the routing decision (1 FA, 0 SA).
 *   q, out, k_caches, v_caches, ctx_len: as in flux_attn_decode, all device.
 *   status_out optional device uint32: receives the FLUX_STATUS_* bits of this call.
 * Limits (beyond them the call returns FLUX_E_CAPACITY and launches nothing):
 * B <= 64, n_q_heads / n_kv_heads <= 8, n_kv_heads <= 16.
 * The first call on each device resolves the array's device address and sets a
 * kernel attribute; make that first call before any stream capture begins.
 * All calls on a device share the one array, which keeps the previous call's
 * contents (the status word is cleared at the start of each call): calls whose
 * kernels may overlap on the GPU -- different streams, or several host threads --
 * race on it and must be serialised by the caller. */
int flux_attn_decode_noalloc(const flux_config *cfg, int32_t layer, int32_t B,
                             const uint8_t *mask, const void *q,
                             const void *const *k_caches, const void *const *v_caches,
                             const int32_t *ctx_len, void *out, uint32_t *status_out,
                             void *stream);

/* The same decode step for callers whose activations live in host memory: brings
 * q, k_new, v_new (host) to the device, appends, attends, and delivers the result
 * to out (host).  With pinned (page-locked) buffers the kernels read the inputs from
 * host memory and write the result there directly, each byte crossing the bus once
 * and no copy operation in the stream (three launches); with pageable buffers the
 * call stages them through the workspace with four asynchronous copies.
 * Asynchronous on `stream` like the rest; the host buffers must stay untouched
 * until the stream is synchronised.  The caches, pointer tables, pos and ctx_len
 * stay on the device. */
int flux_attn_decode_host(flux_plan *plan, int32_t layer, int32_t B, const void *q_host,
                          const void *k_new_host, const void *v_new_host,
                          void *const *k_caches, void *const *v_caches, const int32_t *pos,
                          const int32_t *ctx_len, void *out_host, void *stream);

/* Prefill for host-resident activations: q (host) is copied to the device buffer
 * q_dev, the layer runs as flux_attn_prefill, and out_dev is copied to out_host. */
int flux_attn_prefill_host(flux_plan *plan, int32_t layer, int32_t req, const void *q_host,
                           void *q_dev, const void *k, const void *v, int32_t q_start,
                           int32_t Nq, void *out_dev, void *out_host, void *stream);

/* Synchronises `stream`, reads the device status word and clears it.  Returns
 * FLUX_OK with *status_bits == 0, FLUX_E_DEVICE_TIMEOUT if a wait expired, or
 * FLUX_E_DEVICE_FLAG for the input-check bits.  status_bits (host) may be NULL.
 * A kernel that gave up on a wait leaves its hand-over state in the workspace wherever it
 * stood; when the word reports a timeout this call also puts that state (the arrival counters
 * of the single-launch decode, the router front end's counters, launch number and tagged
 * activations) back to zero on `stream`, so the calls that follow start clean. */
int flux_plan_status(flux_plan *plan, uint32_t *status_bits, void *stream);

/* Dispatch record of the latest flux_attn_decode / flux_attn_prefill on this
 * plan, for verification: synchronises `stream` and copies n_records records of
 * 8 int32 each to records_out (host):
 *   { mode (1 FA, 0 SA), layer, request, n, a_begin, a_end, b_begin, b_end }
 * where [a_begin,a_end) and [b_begin,b_end) are the cache rows the kernel reads
 * for the newest query row (b is empty for FA).  Decode writes one record per
 * request, prefill one record.  n_records_out (host) receives the count. */
int flux_debug_dispatch(flux_plan *plan, int32_t *records_out, int32_t max_records,
                        int32_t *n_records_out, void *stream);

/* Which KV rows the kernels actually read, for verification.  While a bitmap is set, the decode
 * kernel sets bit r of request b's words for every cache row r (slot, in a compact sparse cache)
 * whose K and V it loads, and the tcgen05 prefill kernel sets the bits of every position of every
 * KV tile it loads (request words 0; tiles are 128 positions, clipped to the rows present).
 *   bitmap  uint32 [max_batch][words_per_request], device, zeroed by the caller; NULL turns the
 *           recording off (the default).  words_per_request * 32 >= max_context.
 * The bits accumulate over launches until the caller clears the buffer. */
int flux_debug_touched(flux_plan *plan, uint32_t *bitmap, int32_t words_per_request);

/* Per-kernel device timing for roofline reports.  flux_profile_enable creates
 * max_records pairs of CUDA events (host objects; max_records == 0 turns
 * profiling off and destroys them); while enabled, every launch of a dominant
 * kernel (FLUX_KERNEL_DECODE: the split-K decode kernel, FLUX_KERNEL_PREFILL: the
 * prefill attention kernel) is bracketed by two event records on its stream until
 * the pairs run out.  flux_profile_read synchronises `stream`, sums the elapsed
 * time of the recorded launches of `kind` into *total_ms, stores their count in
 * *launches (both host), and resets the recorder. */
#define FLUX_KERNEL_DECODE  0
#define FLUX_KERNEL_PREFILL 1
int flux_profile_enable(flux_plan *plan, int32_t max_records);
int flux_profile_read(flux_plan *plan, int32_t kind, double *total_ms, int64_t *launches,
                      void *stream);

/* A decode step evaluated in pieces over disjoint key ranges, and the merge of the pieces: the building blocks for
 * spreading one long context over several GPUs (each holds a range of the cache rows, evaluates its piece, the
 * pieces are exchanged -- B * n_q_heads * 130 floats per piece -- and merged).  Eq. 1 / Eq. 2 are sums over keys,
 * so pieces over disjoint key sets merge exactly, by rescaling with the difference of their maxima.
 *
 * flux_attn_decode_partial: as flux_attn_decode, restricted per request to the key positions
 * [key_begin[b], key_end[b]) (device int32 arrays; clamped to [0, ctx_len[b]]).  A request that reads its rows
 * densely (FA, or SA while sink + window still cover the context) reads exactly those rows; a sparse request is
 * evaluated whole by the call whose range holds its newest position ctx_len[b] - 1 and yields an empty piece in
 * every other call.  Instead of an output row the call writes, for every (request, query head), the piece
 *   part_o  fp32 [B][n_q_heads][head_dim]  sum over the range's kept keys of 2^(s_j - m) V_j   (not normalised)
 *   part_ml fp32 [B][n_q_heads][2]         m = the maximum scaled score in log2 units (s_j = scale * log2(e) * q.k_j;
 *                                          -1e30 for an empty piece), l = sum of 2^(s_j - m)
 * both device memory.  Always runs the two-launch kernels.
 *
 * flux_attn_combine: merges n_sets pieces laid out [n_sets][B][n_q_heads][...] (what an all-gather of the ranks'
 * pieces produces) into out bf16 [B][n_q_heads][head_dim]: m = max m_s, O = sum_s O_s 2^(m_s - m), l likewise,
 * out = O / l (a row whose pieces are all empty is zero).
 *
 * The exchange without a library call (the paper has no counterpart: it runs on one GPU).  Every rank owns a gather
 * buffer gather_o fp32 [world][B][n_q_heads][head_dim], gather_ml fp32 [world][B][n_q_heads][2] and a flag array
 * uint32 [world], zero-filled once, and knows the addresses of all ranks' three arrays as they are mapped on ITS
 * GPU (its own plainly, the peers' through peer access / IPC or symmetric memory; on one NVSwitch domain: up to 8).
 * flux_attn_decode_partial_push evaluates this rank's piece like flux_attn_decode_partial and its merge kernel
 * stores every row straight into slot `rank` of every rank's gather buffer (plain stores to peer memory), then --
 * after a system-scope fence by every CTA and a ticket among them -- sets entry `rank` of every rank's flag array to
 * `seq` (release, system scope).  flux_attn_combine_wait is flux_attn_combine over this rank's own gather buffer,
 * each CTA first waiting (acquire, system scope) until all `world` flags equal `seq`.  The wait is bounded:
 * wait_cycles SM clock cycles (0 = about a second), then FLUX_STATUS_WAIT_EXPIRED and `out` is left unwritten.
 * `seq` is any non-zero value that differs from the one used for the previous exchange through the same buffers
 * (a step counter).  A rank may push exchange k + 1 into a buffer only when every rank has finished merging exchange
 * k out of it: use one buffer set per layer (a rank cannot finish layer l + 1 of a step before every rank has
 * merged layer l of it), or two sets alternately.  Both kernels of the pushing call and the waiting merge never wait
 * for a kernel of the same GPU: the writers of the flags are kernels on other GPUs.  Errors: as the calls above;
 * world outside [1, 8], rank outside [0, world), seq == 0 -> FLUX_E_INVALID_ARG. */
typedef struct {
    int32_t world, rank;
    float *gather_o[8];      /* rank p's gather_o as addressable from this GPU */
    float *gather_ml[8];
    uint32_t *flags[8];
} flux_peer_set;
int flux_attn_decode_partial_push(flux_plan *plan, int32_t layer, int32_t B, const void *q, const void *const *k_caches,
                                  const void *const *v_caches, const int32_t *ctx_len, const int32_t *key_begin /*device*/,
                                  const int32_t *key_end /*device*/, const flux_peer_set *peers /*host*/, uint32_t seq,
                                  void *stream);
int flux_attn_combine_wait(flux_plan *plan, int32_t B, int32_t world, const float *gather_o, const float *gather_ml,
                           const uint32_t *flags /*device, this rank's own*/, uint32_t seq, int64_t wait_cycles,
                           void *out /*device bf16 [B][n_q_heads][head_dim]*/, void *stream);
int flux_attn_decode_partial(flux_plan *plan, int32_t layer, int32_t B, const void *q, const void *const *k_caches,
                             const void *const *v_caches, const int32_t *ctx_len, const int32_t *key_begin,
                             const int32_t *key_end, float *part_o, float *part_ml, void *stream);
int flux_attn_combine(flux_plan *plan, int32_t B, int32_t n_sets, const float *part_o, const float *part_ml, void *out,
                      void *stream);

/* Launch overlap for the single-launch decode kernel, the 8-bit and the paged decode (off by default).  With it on, a decode launch
 * builds its schedule and requests its first K / V tiles while the previous kernel in the stream is
 * still draining, and waits for that kernel only before it reads the query rows, the newest K / V row
 * (position ctx_len - 1, from the cache or from k_new / v_new) and before it writes anything.  The
 * caller promises in return that the kernel enqueued immediately before each decode call on the same
 * stream does not write: ctx_len, the routing mask, the pointer tables, or cache rows of the layer
 * being read at positions below ctx_len - 1.  (A decode call of the previous layer, flux_kv_append and
 * flux_attn_decode_step of any layer, and kernels that only produce q / k_new / v_new all qualify.)
 * Launches further back are done by then: every kernel here lets the next one start early only behind its own dependency wait,
 * and a kernel of the caller's in the same stream that does so at all (programmatic launches) has to keep to that too.
 * Results are the same either way; the two-launch kernels ignore the setting.  flux_attn_decode_kvq and
 * flux_attn_decode_step_kvq take it likewise; of an 8-bit cache the kernel before may only write the blocks of 16 positions
 * that hold ctx_len - 1 and ctx_len - 2 (a store or a step of one of the newest two tokens qualifies).  flux_attn_decode_paged and
 * flux_attn_decode_step_paged take it too: the kernel before may write positions ctx_len - 1 and ctx_len - 2 of the pages, and must not
 * write the page table, but the page calls of the same plan (flux_pages_reserve and so on) may come right before. */
int flux_plan_set_launch_overlap(flux_plan *plan, int32_t on);

/* Which kernels flux_attn_decode / flux_attn_decode_step launch.  FLUX_DECODE_AUTO (the default)
 * runs the single-launch kernel for batches of at most 32 requests and at most 64 KV heads (one launch
 * does the split-K attention and the merge: the first CTAs of a (request, KV head) merge one query head
 * each once all its CTAs have announced their partials; it covers the batch-1 latency setting of Appendix C.3 and the batched workloads alike) and
 * the two-launch pair (split-K kernel + combine pass) beyond that; the other two values force one of
 * them where the shape allows.  Both compute Eq. 1 / Eq. 2 over the same rows.  The single-launch
 * kernel is issued with programmatic stream serialisation: it starts with a grid-dependency wait (see
 * flux_plan_set_launch_overlap), so results never depend on it, and it lets the next such launch in
 * the stream be set up while it drains.  Its CTAs (one per SM) wait for one another when they merge
 * (bounded: about a second), so it expects to get the GPU's SMs while it runs; if other work -- another
 * stream's long kernel, a second launch of this kernel running at the same time -- keeps some of its
 * CTAs from starting for that long, the wait expires, FLUX_STATUS_WAIT_EXPIRED is raised and the
 * outputs of that launch are not valid.  Callers that run several decode streams on one GPU at once
 * select FLUX_DECODE_TWO_LAUNCH, whose kernels never wait for each other. */
#define FLUX_DECODE_AUTO          0
#define FLUX_DECODE_TWO_LAUNCH    1
#define FLUX_DECODE_SINGLE_LAUNCH 2
int flux_debug_decode_kernel(flux_plan *plan, int32_t which);

/* Exercises the give-up path of the kernels' bounded waits without any fault: launches one warp
 * that waits, with the same bounded wait the prefill kernel uses, on a barrier nothing arrives
 * at.  After limit_cycles SM clock cycles (1 .. 2e9) the wait runs out, the kernel sets
 * FLUX_STATUS_WAIT_EXPIRED and returns; flux_plan_status() then reports FLUX_E_DEVICE_TIMEOUT
 * and clears the word.  While the bit is set, prefill CTAs return at once without computing. */
int flux_debug_wait_probe(flux_plan *plan, int64_t limit_cycles, void *stream);

/* Number of kernels this plan has launched so far (host counter). */
int64_t flux_launch_count(const flux_plan *plan);

/* Message for the most recent failure on the calling thread ("" if none). */
const char *flux_last_error(void);

/* Library version, "major.minor". */
const char *flux_version(void);

#ifdef __cplusplus
}
#endif
#endif /* FLUX_ATTN_H */
