/*
 * flux.h - C ABI of the Flux Attention inference hot path for AMD MI355X (gfx950).
 *
 * The path: a per-layer Layer Router turns the prompt's boundary tokens into a hard
 * Full-Attention / Sparse-Attention decision (paper Sec. 3.1), the decision is cached
 * (Sec. 3.3), and each layer then runs causal grouped-query Full Attention (Eq. 1) or
 * Sparse Attention (Eq. 2; the streaming variant of Sec. 4.1 / App. C.3: sink tokens plus a
 * causal local window) over ONE contiguous bf16 KV cache, in prefill and in decode, or over
 * pages of 8-bit codes that all sequences take from one pool.
 *
 * General rules
 *  - Every pointer is a raw address.  "dev" = device memory of the context's GPU, "host" =
 *    ordinary host memory.  The caller owns every tensor and the stream; the library owns only
 *    the workspace inside flux_ctx and never allocates in the hot calls.
 *  - All calls are asynchronous on `stream` (a hipStream_t passed as void*; NULL = the default
 *    stream) and never synchronise, except flux_create, flux_destroy, flux_last_device_status.
 *  - Return value: 0 = FLUX_OK, negative = error.  Everything that can be checked from host
 *    arguments is checked before any launch.  What only the device can see (a cache that would
 *    overflow) is clamped so that no access leaves the buffers, and recorded in a sticky status
 *    word readable with flux_last_device_status.
 *  - mode bytes: 1 = FA, 0 = SA (the paper's r_hard; "r_hard = 0 executes SA", Sec. 3.1).
 *  - bf16 tensors are 16-bit brain floats; their base addresses and all strides must be
 *    multiples of 8 elements (16 bytes).  head_dim must be 64 or 128.
 *  - Results are deterministic: the same call (inputs, host bounds, workspace size) gives bit-identical outputs.  In
 *    decode, and in prefill where keys are shared out over workgroups (see there), the order of a sequence's sums also
 *    depends on the other sequences of the call.
 *  - Calls that share one flux_ctx must be ordered on one stream: they share its workspace and the arrival counters in
 *    it.  Calls that overlap on one context all the same can spoil each other's results and leave a counter non-zero,
 *    which spoils later calls too: such a context is to be destroyed.
 */
#ifndef FLUX_H_
#define FLUX_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

enum {
  FLUX_OK = 0,
  FLUX_EINVAL = -1,      /* null pointer, bad head ratio, unsupported head_dim, negative size,
                            misaligned pointer or stride */
  FLUX_ECAPACITY = -2,   /* growth known on the host exceeds the cache capacity */
  FLUX_EWORKSPACE = -3,  /* the context's workspace is too small for this call */
  FLUX_EHIP = -4,        /* a HIP runtime call failed; text via flux_strerror */
  FLUX_ENOMEM = -5       /* allocation failed in flux_create */
};

/* Bits of the sticky device status word. */
enum {
  FLUX_DEV_KV_OVERFLOW = 1,   /* flux_kv_append dropped rows that did not fit `capacity` */
  FLUX_DEV_BAD_LENGTH = 2,    /* a kv_len / cu_seqlens value was inconsistent and was clamped */
  FLUX_DEV_BAD_PAGE = 4       /* a page or slot number of a paged cache lies outside its pool and was left out */
};

typedef struct flux_ctx flux_ctx;   /* opaque; owns ONLY its device workspace */

/* Attention shape and the SA pattern of one call.
 * SA visibility (Eq. 2 with the streaming subset): key j is seen by query position i iff
 * j <= i and (j < n_sink or i - j < window); the query's own position counts inside the window.
 * FA (Eq. 1): every j <= i.  Query head h reads KV head h / (n_q_heads / n_kv_heads). */
typedef struct {
  int32_t n_q_heads, n_kv_heads, head_dim;
  int32_t n_sink, window;
  float softmax_scale;      /* 0 => 1/sqrt(head_dim) (the scale Eq. 1 leaves out "for clarity") */
  int32_t out_dtype;        /* 0 = bf16, 1 = fp32 */
  int32_t sa_block;         /* 0 or 1: the token-exact SA rule above.  A power of two b > 1: the
                               block-granular rule of App. C.3 (a block of b positions is the minimum
                               unit of sparsity; the paper uses 64): with B(x) = x / b, key j is seen
                               by query i iff j <= i and (B(j) < ceil(n_sink / b) or
                               B(i) - B(j) < ceil(window / b)). */
} flux_attn_cfg;

/* One LAYER's KV cache, caller-owned: element (b, h, t, d) of K is
 * k[b*stride_b + h*stride_h + t*stride_t + d], d contiguous, same strides for V.
 * head_dim <= stride_t <= 2^22 elements. */
typedef struct {
  void* k;                  /* dev bf16 */
  void* v;                  /* dev bf16 */
  int64_t stride_b, stride_h, stride_t;   /* in elements */
  int32_t* kv_len;          /* dev int32[batch]: valid positions per sequence */
  int32_t batch, capacity;  /* capacity = positions per sequence the buffers can hold */
} flux_kv_cache;

/* Create a context on `device` with a workspace of `workspace_bytes` (0 = a default that covers
 * batch*heads up to 256 and contexts up to 1M positions).  Synchronous.  The context may only
 * be used with that device current. */
int flux_create(flux_ctx** out, int device, size_t workspace_bytes);
int flux_destroy(flux_ctx* ctx);

/* Static text for an error code; for FLUX_EHIP the text of the last HIP error seen. */
const char* flux_strerror(int code);

/* Bytes of workspace flux_attn_decode needs for this shape (pure host arithmetic;
 * router and append need less than 64 KiB; prefill and flux_xa_select use what there is).  0 on invalid arguments. */
size_t flux_workspace_needed(const flux_attn_cfg* cfg, int batch, int max_kv_len);

/* Returns the sticky device status bits (>= 0) and clears them.  Synchronous: copies the word back and
 * waits for `stream`; when a bit was set it then writes the cleared word and waits for `stream` again. */
int flux_last_device_status(flux_ctx* ctx, void* stream);

/* Layer Router, hard-routing inference form (Sec. 3.1 "Architecture and Feature Extraction"
 * and "Deterministic Inference via Hard Routing"; pooling of the first and last 100 tokens,
 * App. C.1).  For each of the `batch` sequences packed in x (rows cu_seqlens[b] ..
 * cu_seqlens[b+1]-1, each `hidden` wide):
 *   p      = mean of the first `pool` and last `pool` rows (every row once if the sequence has
 *            at most 2*pool rows, or if pool == 0)                         fp32
 *   h      = SiLU(w1 p + b1)                                               fp32
 *   logits = w2 h + b2 = (pi_FA, pi_SA)                                    fp32
 *   mode   = 1 (FA) if pi_FA >= pi_SA else 0 (SA)       (argmax; a tie goes to index 0 = FA)
 * x dev bf16 [T, hidden]; cu_seqlens dev int32 [batch+1]; w1 dev bf16 [inner, hidden];
 * b1 dev bf16 [inner] or NULL; w2 dev bf16 [2, inner]; b2 dev bf16 [2] or NULL;
 * mode_out dev uint8 [batch]; logits_out dev fp32 [batch, 2] or NULL.
 * hidden must be a multiple of 8 and at most 16384, inner a multiple of 8 and at most 4096.
 * Cost does not depend on the sequence length when pool > 0. */
int flux_router(flux_ctx* ctx, const void* x, const int32_t* cu_seqlens, int batch, int hidden,
                int pool, const void* w1, const void* b1, const void* w2, const void* b2, int inner,
                uint8_t* mode_out, float* logits_out, void* stream);

/* Append new K/V rows to the tail of each sequence's cache (the cache every later step of
 * Sec. 3.3 reads).  k_new, v_new: dev bf16 [total_new, n_kv_heads, head_dim], rows of sequence b
 * are cu_new[b] .. cu_new[b+1]-1 (dev int32 [batch+1]).  Row r of sequence b goes to position
 * kv_len[b] + r; afterwards kv_len[b] += rows of b.  `total_new` and `max_new` (the largest
 * per-sequence row count) are host values; max_new > capacity gives FLUX_ECAPACITY.  Rows that
 * would pass `capacity` on the device are dropped and FLUX_DEV_KV_OVERFLOW is raised. */
int flux_kv_append(flux_ctx* ctx, const flux_kv_cache* cache, int n_kv_heads, int head_dim,
                   const void* k_new, const void* v_new, const int32_t* cu_new, int total_new,
                   int max_new, void* stream);

/* Prefill attention of one layer (Eq. 1 / Eq. 2, routed per sequence by `mode`, Sec. 3.3).
 * q dev bf16 [T, n_q_heads, head_dim], rows of sequence b are cu_q[b] .. cu_q[b+1]-1 (dev int32
 * [batch+1]).  The n_q(b) queries of sequence b are the LAST n_q(b) positions of its cache:
 * query row r sits at position kv_len[b] - n_q(b) + r (append first, then attend; a chunk of a
 * longer prompt and a whole prompt are the same call).  mode dev uint8 [batch].
 * out dev [T, n_q_heads, head_dim] in cfg->out_dtype.  max_q_len, max_kv_len: host upper bounds
 * on n_q(b) and kv_len[b] (they size the launch; larger than needed is valid, smaller truncates
 * nothing: of rows beyond max_q_len only such are computed as share a tile of 64 or 128 with rows within it; a bound far above the
 * real lengths costs empty workgroups, and max_q_len from 32768 on (or from 16384 on with max_kv_len from 32768 on) selects
 * the launch shape tuned for long prompts).  All launch shapes give the same results bit for bit, with one exception:
 * where max_kv_len > max_q_len (queries behind a cached context), the batch has at most 64 sequences, the launch is not of
 * the long shape, and the queries alone would not fill the chip, the keys of a tile of query rows may be shared out over
 * several workgroups.  Whether and how depends on both bounds, on the lengths and modes of the whole batch and on the room
 * for partial results in the workspace (lists of up to 1024 keys never are); the sums are then taken in another order
 * than in one walk.  SA tiles that the mask hides are skipped,
 * not masked: their K/V rows are never read.  A 64-key tile that is partly visible is read whole
 * (up to kv_len[b]), so the cached rows below kv_len[b] must hold finite values; those of V up to 2^64 in magnitude (rows are summed
 * with weights of up to 2^32 before they are divided by the weights' sum).  If the device finds n_q(b) > kv_len[b]
 * (the caller did not append first), only the first
 * kv_len[b] query rows of that sequence are computed and FLUX_DEV_BAD_LENGTH is raised. */
int flux_attn_prefill(flux_ctx* ctx, const flux_attn_cfg* cfg, const void* q, const int32_t* cu_q,
                      int max_q_len, int max_kv_len, const flux_kv_cache* cache,
                      const uint8_t* mode, void* out, void* stream);

/* Prefill attention of one layer with a BLOCK-SPARSE visible set for the sequences whose mode byte is 0 (Eq. 2
 * over an arbitrary set of key blocks: the substrate of the sparse modes of Sec. 4.1 that choose blocks by content;
 * a block of 64 positions is the minimum unit of sparsity, App. C.3).  Same arguments and conventions as
 * flux_attn_prefill; cfg->n_sink, window and sa_block are not used.  A sequence with mode byte 1 runs FA.
 *   block_mask: dev uint8 [batch, mask_heads, n_qblocks, n_kblocks], mask_heads = 1 (all heads share one matrix)
 *               or n_q_heads.  Positions are grouped in blocks of 64.  For sequence b, row rq of its matrix belongs
 *               to the query block  (kv_len[b] - n_q(b)) / 64 + rq  (row 0 is the block that holds its first query
 *               of this call), column kb to key block kb.  Query position i sees key j iff j <= i and
 *               (flag[block of i, block of j] != 0 or block of i == block of j): the causal order holds inside
 *               blocks, and a query's own block is always kept.  Key blocks that no query block of a 128-row tile
 *               keeps are not loaded.
 *   n_kblocks * 64 >= max_kv_len and n_qblocks * 64 >= max_q_len, else FLUX_EINVAL.  A run of queries that starts
 *   inside a block spans one block more than its length suggests: on the device, a pair that lies outside the
 *   matrix counts as not kept and raises FLUX_DEV_BAD_LENGTH. */
int flux_attn_prefill_blocksparse(flux_ctx* ctx, const flux_attn_cfg* cfg, const void* q, const int32_t* cu_q,
                                  int max_q_len, int max_kv_len, const flux_kv_cache* cache, const uint8_t* mode,
                                  const uint8_t* block_mask, int mask_heads, int n_qblocks, int n_kblocks, void* out,
                                  void* stream);

/* Block selection of the XA sparse mode (Sec. 4.1; Table 3: stride 16, threshold 0.9, selection mode "Inverse",
 * block 64) for whole prompts: writes, for every sequence and query head, the keep matrix that
 * flux_attn_prefill_blocksparse consumes (mask_heads = n_q_heads).  The paper gives the method's name ("Block
 * Sparse Attention with Antidiagonal Scoring") and these parameters, nothing more; what is computed is this reading:
 *   - the scaled scores of a head are cut into squares of stride x stride positions; of a square only the
 *     antidiagonal is sampled (query offset r against key offset stride-1-r: the "Inverse" order), and only the
 *     causal samples inside the prompt; e[a][b] = the mean of the samples of square (a, b);
 *   - softmax over every row a of e (its squares b <= a);
 *   - mass of a block pair = the sum of those probabilities inside it / the rows of e the query block has;
 *   - query block I keeps every key block whose mass is at least the mass of the block at which the masses, taken
 *     in descending order, first reach `threshold` (equal masses are kept together), and always its own block.
 * q, cu_q, cache as in flux_attn_prefill, with n_q(b) == kv_len[b] for every sequence (a whole prompt, appended
 * first; anything else raises FLUX_DEV_BAD_LENGTH and scores the first min(n_q, kv_len) positions).  stride must be
 * 16; 0 < threshold <= 1; cfg->softmax_scale as in Eq. 1; cfg->n_sink, window, sa_block, out_dtype are not used.
 * block_mask: dev uint8 [batch, n_q_heads, n_qblocks, n_kblocks], every byte written (0 or 1);
 * n_kblocks * 64 >= max_kv_len, n_qblocks * 64 >= max_q_len, n_kblocks <= 4096 (262144 positions), else FLUX_EINVAL.
 * max_q_len bounds the prompt lengths (host); a prompt found longer on the device is scored up to the bound, rounded
 * up to whole blocks, and FLUX_DEV_BAD_LENGTH is raised.  The scores of as many heads at a time as fit go through the
 * workspace (with r = ceil(max_q_len / 2048), one head takes 32 KB * r * (r + 1), and 64 KB * r are used at least; a smaller
 * workspace is valid and slower; so is a bound far above the lengths, which counts here as if the prompts were as long).
 * The masses are computed in fp32 from exact bf16 products: near a tie between the threshold and a partial sum
 * of masses the selection can differ from one made in higher precision. */
int flux_xa_select(flux_ctx* ctx, const flux_attn_cfg* cfg, const void* q, const int32_t* cu_q, int max_q_len,
                   int max_kv_len, const flux_kv_cache* cache, int stride, float threshold, uint8_t* block_mask,
                   int n_qblocks, int n_kblocks, void* stream);

/* Decode attention of one layer: one query per sequence at position kv_len[b]-1 (append first).
 * q dev bf16 [batch, n_q_heads, head_dim]; out dev [batch, n_q_heads, head_dim].
 * FA streams all kv_len[b] cached rows; SA reads only rows [0, n_sink) and
 * [kv_len[b]-window, kv_len[b]) and never touches the rest (App. B.3).
 * max_kv_len: host upper bound on the number of keys any sequence of this call ATTENDS TO; the
 * largest kv_len[b] (or the capacity) is always valid.  The split of the work over the chip is taken
 * on the device from the lengths and mode bytes found there, so a loose bound costs idle
 * workgroups and a ragged batch is spread as evenly as a uniform one; the bound limits the launch
 * and the workspace.  One launch.  A caller that knows every sequence of this layer is SA may pass
 * min(max kv_len, n_sink + window) (both rounded up to multiples of sa_block when that is set).
 * A sequence that attends to more keys than the bound is cut at the bound (its oldest visible
 * keys are kept) and FLUX_DEV_BAD_LENGTH is raised. */
int flux_attn_decode(flux_ctx* ctx, const flux_attn_cfg* cfg, const void* q, int max_kv_len,
                     const flux_kv_cache* cache, const uint8_t* mode, void* out, void* stream);

/* One whole decode step of a layer (Sec. 3.3, the decode path; App. B.3): the same result and the same cache
 * contents as flux_kv_append of one row per sequence followed by flux_attn_decode, bit for bit, in one launch instead of two
 * (for a sparse layer, whose kernels run for some tens of microseconds, the append launch is a tenth of the step).
 *   k_new, v_new: dev bf16 [batch, n_kv_heads, head_dim], 16-byte aligned: the row sequence b appends at position
 *                 kv_len[b] (before the call).  A sequence whose cache is full drops its row, raises
 *                 FLUX_DEV_KV_OVERFLOW and attends to what is cached, as the pair of calls would.
 *   max_kv_len:   >= 1; bound on the keys any sequence attends to AFTER the append (see flux_attn_decode).
 *   cache:        a full cache (not a ring); kv_len[b] is read by every workgroup and moved on at the end of the
 *                 call (kv_len[b] += 1, cut at the capacity).
 * Other arguments as flux_attn_decode.  The workgroup with the beginning of a sequence's key list stores the new row;
 * workgroups that attend to it read it from k_new / v_new; the last workgroup to have read the lengths moves them on. */
int flux_attn_decode_append(flux_ctx* ctx, const flux_attn_cfg* cfg, const void* q, const void* k_new, const void* v_new,
                            int max_kv_len, const flux_kv_cache* cache, const uint8_t* mode, void* out, void* stream);

/* flux_attn_decode for callers that cannot allocate device memory at all (code under HIP graph capture, tight
 * serving loops, harnesses that forbid hipMalloc): no context, and no hipMalloc / hipFree / allocating library
 * call inside.  The split-K partial results go to a static device array of FLUX_STATIC_SCRATCH_BYTES that
 * every GPU the library runs on holds until the process ends; the call works on the CURRENT device, whose
 * copy of the array is looked up once (at flux_create on that device, else at the first call).
 * Same arguments and results (bit for bit) as flux_attn_decode (which merges in the launch that streams the keys, on arrival
 * counters of its context; here that takes a second launch: the array holds no state between calls), plus
 *   status: dev uint32 (4-byte aligned), caller-owned, or NULL.  The FLUX_DEV_* bits of this call are OR-ed
 *           into it (sticky; the caller reads and clears it); with NULL they go to a word nobody reads.
 * A shape whose partials exceed the array gives FLUX_EWORKSPACE: the partials take
 * min(1024 + pairs, pairs * ceil(max_kv_len / 256)) * min(group, 16) * (head_dim + 2) * 4 bytes with
 * pairs = batch * n_kv_heads * ceil(group / 16), group = n_q_heads / n_kv_heads (2.3 MB for batch 8, 32/8
 * heads of 128 at any length).  All calls on one GPU share that GPU's array: calls that overlap on one GPU
 * (two streams, two threads) race and must be ordered by the caller (they spoil each other's results, not those of later
 * calls).  Nothing needs clearing between calls. */
#define FLUX_STATIC_SCRATCH_BYTES ((size_t)16 * 1024 * 1024 + 256)
int flux_attn_decode_static(const flux_attn_cfg* cfg, const void* q, int max_kv_len, const flux_kv_cache* cache,
                            const uint8_t* mode, void* out, uint32_t* status, void* stream);

/* ---- Sparse-decode residency (Sec. 3.3 "Efficient Deployment": a sparse layer keeps only the minimal
 * KV cache its kernel needs and never stores the rest of the history; retrieval layers keep everything).
 *
 * A RING cache is a flux_kv_cache read with these rules: capacity >= n_sink + window rows per
 * (sequence, head); row p < n_sink holds position p; position p >= n_sink lives in row
 * n_sink + (p - n_sink) % window, overwriting the position that has just left the window; kv_len[b] is the
 * LOGICAL length (positions appended so far) and is not bounded by capacity.  The rows stored for a
 * sequence are then exactly the keys Eq. 2 lets its newest position see.  n_sink and window must be the
 * same in every call on one ring cache.  A ring cache serves decode only: the prompt is prefilled on a
 * full cache (the decision exists only after the router has seen the prompt), then compacted. */

/* flux_kv_append on a ring cache.  Same arguments as flux_kv_append plus the ring geometry.  Of the new
 * rows of a sequence only those that are still resident after the call are written (sinks, and the last
 * `window` positions), so any number of rows may be appended at once.  kv_len[b] += rows of b. */
int flux_kv_append_ring(flux_ctx* ctx, const flux_kv_cache* ring, int n_kv_heads, int head_dim, int n_sink,
                        int window, const void* k_new, const void* v_new, const int32_t* cu_new,
                        int total_new, int max_new, void* stream);

/* Copy what a sparse layer keeps from a full cache `src` (after prefill) into the ring cache `dst`:
 * positions [0, n_sink) and [max(len - window, n_sink), len) of every sequence, len = src kv_len[b]
 * (clamped to src capacity); sets dst kv_len[b] = len.  Same batch in both; src is not modified and may
 * be reused for the next layer's prompt. */
int flux_kv_compact_ring(flux_ctx* ctx, const flux_kv_cache* src, const flux_kv_cache* dst, int n_kv_heads,
                         int head_dim, int n_sink, int window, void* stream);

/* flux_attn_decode of a sparse layer on its ring cache: the query of sequence b sits at position
 * kv_len[b] - 1 (append first) and attends to every stored row (Eq. 2).  No mode argument: a ring cache
 * holds a sparse layer.  cfg->n_sink and cfg->window are the ring geometry; with cfg->sa_block = b > 1 the
 * ring must have been filled with n_sink and window rounded up to multiples of b. */
int flux_attn_decode_ring(flux_ctx* ctx, const flux_attn_cfg* cfg, const void* q, const flux_kv_cache* ring,
                          void* out, void* stream);

/* ---- Paged 8-bit KV caches: the same attention over a cache of half the bytes, whose sequences share one pool of pages.
 *
 * A PAGE holds FLUX_PAGE_TOKENS = 64 positions of a sequence (the block of App. C.3) for all KV heads of a layer, as e4m3 codes
 * (sign, 4 exponent bits, 3 fraction bits, bias 7, no infinity; the codes 0x7F and 0xFF are NaN) with one fp32 scale per page,
 * KV head and K or V: the value of a code is code * scale.  The block table says which pages a sequence has; it and the lengths
 * are the same for all layers, so a step plans its pages once (flux_page_plan) and then runs flux_kv_append_paged and
 * an attention call per layer, each on the layer's own pool. */
#define FLUX_PAGE_TOKENS 64
#define FLUX_MAX_PAGED_BATCH 4096   /* sequences of a flux_page_plan or flux_page_release call */

/* Which pages the sequences have, and which are free.  Page `table[b * table_pages + i]` holds positions 64 i .. 64 i + 63 of
 * sequence b; a sequence has ceil(kv_len[b] / 64) pages, and table entries behind them are not read.  A page may stand in the
 * tables of several sequences (a shared prefix) as long as nobody appends to it or releases it: flux_page_fork counts who has a
 * page, and keeps that so. */
typedef struct {
  int32_t* table;           /* dev int32 [batch, table_pages] */
  int32_t* kv_len;          /* dev int32 [batch]: valid positions per sequence */
  int32_t* free_pages;      /* dev int32 [n_pages]: the free pages are entries 0 .. n_free - 1 (not used by attention: may be NULL there) */
  int32_t* n_free;          /* dev int32 [1] (the same) */
  int32_t batch, table_pages;   /* table_pages <= 2^24 */
  int32_t n_pages;          /* pages of every layer's pool, at most 2^24: page numbers are 0 .. n_pages - 1 */
} flux_page_table;

/* One LAYER's pool, caller-owned: the code of (page p, KV head h, position t of the page, d) of K is byte
 * p*stride_p + h*stride_h + t*stride_t + d of k, same strides for V; strides are multiples of 16 bytes, head_dim <= stride_t <=
 * 2^20, and k and v are 16-byte aligned. */
typedef struct {
  void* k;                  /* dev e4m3 */
  void* v;                  /* dev e4m3 */
  float* k_scale;           /* dev fp32 [n_pages, n_kv_heads] */
  float* v_scale;           /* dev fp32 [n_pages, n_kv_heads] */
  int64_t stride_p, stride_h, stride_t;   /* in bytes */
  int32_t n_pages;
} flux_paged_kv;

/* Pages and slots for the new tokens of a step.  Sequence b gets the rows cu_new[b] .. cu_new[b+1]-1 (dev int32 [batch+1], cut
 * at total_new, the number of rows, host) at positions kv_len[b] .., and the ceil((kv_len[b] + rows) / 64) - ceil(kv_len[b] / 64)
 * pages it lacks for them: the i-th page needed, counted by sequence and then by position, is free_pages[n_free - 1 - i].
 * Writes those table entries, slots[t] = 64 * page + position % 64 for every row t (dev int32 [total_new]; -1: the row has no
 * place), then kv_len[b] += rows that have one and n_free -= pages taken.  Where the free pages do not suffice, or table_pages
 * does not, the last rows of the sequences that come too late get none and FLUX_DEV_KV_OVERFLOW is raised.  Numbers outside the
 * pool raise FLUX_DEV_BAD_PAGE: a sequence whose last, partly filled page has one gets no new rows; a free page that has one is
 * taken, but stands as -1 in the table and gives its rows no place (they count in kv_len[b]).
 * batch <= FLUX_MAX_PAGED_BATCH, batch * table_pages < 2^31. */
int flux_page_plan(flux_ctx* ctx, const flux_page_table* pt, const int32_t* cu_new, int total_new, int32_t* slots, void* stream);

/* Cut every sequence to its first keep_len[b] positions (dev int32 [batch]; 0: the request is done; kv_len[b] or more: nothing
 * changes; fewer: rejected tokens are taken back) and return the pages behind them, so that the next flux_page_plan takes the
 * page of the first sequence's first returned place first (a plan is taken back exactly).  Returned table entries become -1.
 * batch <= FLUX_MAX_PAGED_BATCH, batch * table_pages < 2^31.  Pages that stand in several tables must not be returned.  If the list
 * of free pages would grow past n_pages, or an entry lies outside the pool, FLUX_DEV_BAD_PAGE is raised and the page is not listed. */
int flux_page_release(flux_ctx* ctx, const flux_page_table* pt, const int32_t* keep_len, void* stream);

/* Quantise new K/V rows of one layer into their slots.  k_new, v_new: dev bf16 [total_new, n_kv_heads, head_dim]; slots: dev
 * int32 [total_new] as flux_page_plan writes them (rows of one page lie next to each other, in the order of their positions;
 * no two rows have the same slot); rows with a negative slot, which stand before or behind those of a page, are left out.  The
 * scale of a (page, head) is 2^e with the smallest e >= -100 for which no value of its block exceeds 448 * 2^e, the largest code; a page that holds rows already (slot % 64 of its
 * first new row is not 0) keeps its scale unless a new row needs a larger one: then the codes it holds are rounded to that.
 * Powers of two cost a code of 4 exponent bits nothing (values below 2^-14 of the block's largest one at most) and make that
 * second rounding exact but for such values.  Rounding is to nearest even.  Values that are not finite are
 * stored as NaN and do not count towards the scale; an attention result over such a row is NaN (prefill: also of earlier
 * queries that share a tile of 64 keys with it).  A slot outside the pool raises FLUX_DEV_BAD_PAGE and its row is left out.
 * total_new <= 2^30, (total_new / 64 + 1) * n_kv_heads <= 2^30. */
int flux_kv_append_paged(flux_ctx* ctx, const flux_paged_kv* kv, int n_kv_heads, int head_dim, const void* k_new, const void* v_new,
                         const int32_t* slots, int total_new, void* stream);

/* flux_attn_decode over a paged 8-bit cache: one query per sequence at position kv_len[b] - 1, mode bytes, SA rule, outputs and
 * determinism as there; keys and values are code * scale (any finite scale >= 0; one of V below 2^-126 counts as that; values of V up to
 * 2^64 in magnitude: rows are summed with weights of up to 2^32 before they are divided by the weights' sum, and a longer list of larger
 * values may pass the range of fp32).  Weights are held to 2^-16, for fp32 outputs to 2^-24.  max_kv_len: host upper bound on kv_len[b],
 * at most 64 * table_pages (which is always valid); pages of a longer list are left out, the oldest kept, and FLUX_DEV_BAD_LENGTH
 * is raised.  Where all sequences are SA, 64 * (ceil(n_sink / 64) + ceil(window / 64) + 1) is enough (n_sink and window rounded
 * up to multiples of sa_block).  The workspace that flux_workspace_needed names for these arguments is enough.
 * batch * n_kv_heads * ceil(group / 16) * (ceil(max_kv_len / 64) + 16) must be below 2^31 (FLUX_EINVAL).
 * A score scale * sk * (q . ck) is an fp32 number and may be of either sign, up to 2^24 in magnitude: beyond that fp32 does not tell
 * scores that are one apart from each other, and the row may be anything.
 * What lies behind kv_len[b] in a page is never used.  A table entry outside the pool counts as a page that is not there, and
 * raises FLUX_DEV_BAD_PAGE; rows without any key are zero. */
int flux_attn_decode_paged(flux_ctx* ctx, const flux_attn_cfg* cfg, const void* q, int max_kv_len, const flux_paged_kv* kv,
                           const flux_page_table* pt, const uint8_t* mode, void* out, void* stream);

/* flux_attn_prefill over a paged 8-bit cache: q, cu_q, max_q_len, max_kv_len, mode, out as there (the queries of sequence b are the
 * last n_q(b) positions of its pages: flux_page_plan and flux_kv_append_paged first); keys and values are code * scale (scales,
 * values and scores as in flux_attn_decode_paged).  Query rows beyond max_q_len are left as they were.
 * A tile of query rows holds all heads of a group, token by token, and walks only pages of which a row sees something.  Weights are
 * rounded to bf16 (by 2^-8 of one at most; the denominator sums the rounded ones), whatever out_dtype is, as in flux_attn_prefill.
 * Pages of a tile may be shared out over several workgroups where the batch has at most 64 sequences and max_kv_len is 961 (16
 * pages) or more, or 8129 (128 pages) or more where the tiles of max_q_len queries are many, as far as the workspace has room for their
 * results (any context will do), in a way that depends on the bounds, lengths and modes of the whole batch.
 * Where max_q_len * group <= 32, the batch has at most 64 sequences, max_kv_len is 449 (eight pages) or more and the workspace has
 * room (one of 18 MB always has), the rows of a sequence are worked on like a decode call's, and their weights are held as there.
 * kv_len[b] above max_kv_len raises FLUX_DEV_BAD_LENGTH (the oldest pages may be all that such a sequence is computed from).
 * max_q_len * group <= 2^30, and batch * (n_kv_heads * ceil(max_q_len * group / 64) + 8) <= 2^22 is always enough (FLUX_EINVAL).
 * What lies behind kv_len[b] in a page is never used; the codes of a page of which a row of a tile sees something must not be NaN
 * below that, or rows of the tile that do not see them may become NaN as well.  A table entry outside the pool counts as a page that is
 * not there, and raises FLUX_DEV_BAD_PAGE; rows without any key are zero. */
int flux_attn_prefill_paged(flux_ctx* ctx, const flux_attn_cfg* cfg, const void* q, const int32_t* cu_q, int max_q_len,
                            int max_kv_len, const flux_paged_kv* kv, const flux_page_table* pt, const uint8_t* mode,
                            void* out, void* stream);

/* ---- Heads on their way from the projection to the attention: norms and position rotation of queries and keys.
 *
 * For a head row x of head_dim values (D):
 *   y = x / sqrt(mean(x^2) + eps) * w     (w: q_norm or k_norm, one weight per dimension, the same for all heads; NULL: y = x)
 *   of the first rotary_dim dimensions (R) of y, pair i < R/2 with t = position * inv_freq[i] (radians, in real numbers):
 *     (a, b) -> (a cos t - b sin t, b cos t + a sin t),  a, b = dimensions i and i + R/2, or 2i and 2i + 1 where interleaved is 1.
 * Everything between is held in fp32 (angles in 64 bits until whole turns are taken off; keys that go into pages of 8-bit codes wholly in 64 bits), and rounded once, to
 * nearest even.  Positions are any int32 numbers. */
typedef struct {
  int32_t n_q_heads, n_kv_heads, head_dim;   /* head_dim 64 or 128 */
  int32_t rotary_dim;       /* a multiple of 16, at most head_dim; 0: no rotation */
  int32_t interleaved;      /* 0 or 1 */
  float eps;                /* 1e-30 or more where there is a norm */
  const void* q_norm;       /* dev bf16 [head_dim], 16-byte aligned, or NULL */
  const void* k_norm;       /* the same */
  const float* inv_freq;    /* dev fp32 [rotary_dim / 2], 16-byte aligned (rotary_dim 0: not used) */
} flux_head_cfg;

/* Rows of the projection: head h of token row t of q is q[t*stride_q + h*head_dim ..], the same for k and v (one buffer that holds
 * all three side by side is three pointers into it).  dev bf16, 16-byte aligned; strides in elements, multiples of 8, at
 * least a row of heads. */
typedef struct {
  const void* q;
  const void* k;
  const void* v;
  int64_t stride_q, stride_k, stride_v;
} flux_qkv_rows;

/* Queries and keys of `total` token rows: q_out dev bf16 [total, n_q_heads, head_dim], k_out dev bf16 [total, n_kv_heads, head_dim],
 * either NULL together with its input (v is not used).  positions: dev int32 [total] (rotary_dim 0: not used).  An output may be its
 * input where that has no gaps (stride = heads * head_dim); otherwise they must not overlap.  total <= 2^30. */
int flux_qk_norm_rope(flux_ctx* ctx, const flux_head_cfg* cfg, const flux_qkv_rows* in, const int32_t* positions, int total,
                      void* q_out, void* k_out, void* stream);

/* flux_qk_norm_rope and flux_kv_append in one pass: queries go to q_out (NULL together with in->q: keys and values alone), finished
 * keys and the values as they are to the tail of each sequence's cache; cu_new, total_new, max_new, lengths, FLUX_ECAPACITY and
 * FLUX_DEV_KV_OVERFLOW as in flux_kv_append.  positions: dev int32 [total_new], or NULL: row r of sequence b is at kv_len[b] + r, the
 * place that it goes to.  Rows of no sequence (before cu_new[0], from cu_new[batch] on) are left out, and q_out there is left as it was. */
int flux_qkv_append(flux_ctx* ctx, const flux_head_cfg* cfg, const flux_kv_cache* cache, const flux_qkv_rows* in,
                    const int32_t* cu_new, int total_new, int max_new, const int32_t* positions, void* q_out, void* stream);

/* flux_qk_norm_rope and flux_kv_append_paged in one pass: queries go to q_out (or both NULL), keys and values are quantised into their
 * slots; slots, scales and FLUX_DEV_BAD_PAGE as in flux_kv_append_paged, total_new <= 2^27.  A key's code is rounded once, from the value that the
 * formula names.  positions: dev int32 [total_new] (rotary_dim 0: not used).  Every row of q_out is written, whatever its slot is. */
int flux_qkv_append_paged(flux_ctx* ctx, const flux_head_cfg* cfg, const flux_paged_kv* kv, const flux_qkv_rows* in,
                          const int32_t* slots, const int32_t* positions, int total_new, void* q_out, void* stream);

/* ---- Pages that change hands.  `shares` (dev int32 [n_pages], the same for all layers) holds for every page how many rows of the table have it,
 * less one; 0 for a free page.  It begins as zeros; flux_page_plan and flux_page_release need not know it, as the pages that they give
 * and take have one holder.  A sequence that may hold shared pages gives them back through flux_page_fork. */

/* Sequence b goes on with the first n(b) = min(keep_len[b], kv_len[parent[b]]) positions of what sequence parent[b] holds now (dev int32 [batch]
 * each; parent NULL: b itself; parent[b] = -1: nothing, the request is done; keep_len NULL: all of them; below 0 counts as 0): beams that are
 * replaced, samples that begin as copies, prompts that requests share, finished requests and rejected tokens.  Row b of the table becomes the
 * first ceil(n(b) / 64) entries of row parent[b] as it was, places that it had behind them become -1, kv_len[b] = n(b), and shares is brought up to date.
 *   Pages that no row has any longer go back: they are listed behind the free pages, the one with the highest number first, so that the lowest is taken first.
 *   A last page that is partly filled (n(b) % 64 != 0) is appended to next, so nobody else may have it: of the sequences that have a page partly
 *   filled the first one keeps it if none has all of it filled; the others get a page each, in the order of the sequences, the j-th of them
 *   free_pages[n_free - 1 - j] (after those that went back were listed), and copies[j] = {page, its copy, n(b) % 64} (dev int32 [batch, 3]); *n_copies
 *   (dev int32) is their number, and entries behind them are left as they were.  flux_page_copy then copies them in each layer, before
 *   anything is appended.  Where the free pages do not suffice, such a sequence is cut to whole pages and FLUX_DEV_KV_OVERFLOW is raised.
 * Limits as in flux_page_release.  Of pools of more than 16384 pages the workspace holds 4 bytes per page beside what flux_create asks for at least (FLUX_EWORKSPACE; the default does).  Parents outside the batch count as -1 and lengths
 * outside the table are cut (FLUX_DEV_BAD_LENGTH); table entries outside the pool are not counted, are given on as -1 and raise FLUX_DEV_BAD_PAGE,
 * as does a page that more rows lost than had it by `shares` (it goes back all the same). */
int flux_page_fork(flux_ctx* ctx, const flux_page_table* pt, int32_t* shares, const int32_t* parent, const int32_t* keep_len,
                   int32_t* copies, int32_t* n_copies, void* stream);

/* Close the holes of the pool: as long as the lowest free page lies below the highest page in use (one that is not listed as free), the latter moves to
 * the former, at most max_moves times.  moves[j] = {from, to, 64} (dev int32 [max_moves, 3]), *n_moves (dev int32) their number, entries behind
 * them left as they were.  Tables and shares (NULL: nobody shares pages) follow; the free pages are listed again, the highest number first, so that
 * the lowest is taken first.  flux_page_copy then moves the codes in each layer (no page is both moved from and to), before the next attention or append call.  After a call with
 * enough moves the pages in use are 0 .. n_pages - n_free - 1.  n_pages <= 2^20, batch <= FLUX_MAX_PAGED_BATCH; the workspace holds 36 bytes per 256 pages
 * beside what flux_create asks for at least (FLUX_EWORKSPACE; the default does).  Numbers in the list outside the pool, or listed twice, are dropped from it and raise FLUX_DEV_BAD_PAGE, as do table entries outside the
 * pool (left as they were). */
int flux_page_compact(flux_ctx* ctx, const flux_page_table* pt, int32_t* shares, int32_t* moves, int max_moves, int32_t* n_moves,
                      void* stream);

/* Copy pages within one layer's pool: for each entry {from, to, rows} of `copies` (dev int32 [max_copies, 3]) before *n_copies (dev int32; NULL:
 * all of them) the codes of the first `rows` positions (0 .. 64, cut to that) and the scales of all heads.  Entries {-1, -1, ..} are left out; other numbers
 * outside the pool raise FLUX_DEV_BAD_PAGE.  A page that is copied to must stand in no other entry. */
int flux_page_copy(flux_ctx* ctx, const flux_paged_kv* kv, int n_kv_heads, int head_dim, const int32_t* copies,
                   const int32_t* n_copies, int max_copies, void* stream);

/* ---- Cross attention: every query row of sequence b sees all kv_len[b] keys of its cache (the states of an encoder, written by flux_kv_append or
 * flux_qkv_append), whatever the number of queries.  q dev bf16 [T, n_q_heads, head_dim], rows of sequence b are cu_q[b] .. cu_q[b+1]-1
 * (dev int32 [batch+1]); cu_q NULL: max_q_len rows each, one sequence behind the other.  out dev [T, n_q_heads, head_dim] in cfg->out_dtype; cfg->n_sink, window and
 * sa_block have to be valid and are not used.  max_q_len, max_kv_len: host upper bounds (rows and keys beyond them are left out and raise FLUX_DEV_BAD_LENGTH; looser ones cost idle
 * workgroups).  Rows without any key are zero; rows of no sequence are left as they were.  With cu_q NULL and max_q_len 1 (a decode step) the
 * call is worked on like flux_attn_decode and needs the workspace that flux_workspace_needed names (a length above the capacity counts as the capacity there,
 * and is reported only where max_kv_len is less); any other call takes what there is.
 * Weights are held to 2^-16 where max_q_len * group <= 32 (a decode step is such a call), and else rounded to bf16 as in flux_attn_prefill; cached rows below kv_len[b] must be finite, those of V up to 2^64.
 * Keys of a tile of rows may be shared out over workgroups, in a way that depends on the bounds and lengths of up to 64 sequences side by side.
 * n_q_heads / n_kv_heads <= 2^20, batch * max_q_len < 2^31 where cu_q is NULL; min(batch, 64) * (n_kv_heads * ceil(max_q_len * group / 64) + 8) <= 2^23 is always enough (FLUX_EINVAL). */
int flux_attn_cross(flux_ctx* ctx, const flux_attn_cfg* cfg, const void* q, const int32_t* cu_q, int max_q_len, int max_kv_len,
                    const flux_kv_cache* cache, void* out, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* FLUX_H_ */
