/*
 * hh.h -- C ABI of the MI355X (gfx950) decoder runtime for the "mouth" model
 * of the Horsehair runtime path.
 *
 * The paper's runtime phase ends with a 1B-class decoder-only model that
 * streams a rendered answer (Sec. 4, "Runtime phase"): one prompt evaluation,
 * whose latency is the time to first token, followed by token-by-token
 * streaming decode (the three speed quantities are defined in Sec. 6.2; the
 * KV cache's memory grows with the context window, Sec. 6.6).  The paper does
 * not describe the model's internals, so the library implements the standard
 * Llama-style decoder: RMSNorm, rotary embeddings (rotate-half pairing), grouped
 * query attention, SwiGLU MLP, tied or untied LM head, greedy argmax.
 *
 * Conventions for every call:
 *  - Every function returns an hh_status; HH_OK is 0, errors are negative.
 *    On any error the context's state (stream lengths, KV contents, pending
 *    tokens, loaded weights) is unchanged and hh_last_error() describes it.
 *    An error that an earlier HIP call left on the thread is not theirs, and
 *    stays; prompts, hh_load_weights (and steps without graphs) report and take
 *    it, with nothing done.
 *  - A context is not thread-safe: use it from one host thread at a time.
 *  - All GPU work of a context is enqueued on the HIP stream given to
 *    hh_create.  Calls whose outputs are host memory synchronize that stream
 *    before returning; calls whose outputs are device memory (or absent) only
 *    enqueue.
 *  - Pointer arguments documented "host or device" are classified with
 *    hipPointerGetAttributes; "host" arguments must be host memory.
 */
#ifndef HH_H_
#define HH_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef int32_t hh_status;

enum {
  HH_OK = 0,
  HH_ERR_INVALID_ARG = -1,   /* bad pointer, id, size or tensor count        */
  HH_ERR_OOM = -2,           /* arena smaller than hh_workspace_size()       */
  HH_ERR_CONTEXT_FULL = -3,  /* a stream would exceed max_context            */
  HH_ERR_NOT_LOADED = -4,    /* prefill/decode before hh_load_weights        */
  HH_ERR_HIP = -5,           /* a HIP runtime call failed                    */
  HH_ERR_UNSUPPORTED = -6    /* configuration outside what the kernels cover */
};

enum { HH_F32 = 0, HH_BF16 = 1 };                       /* weight / KV element type */
enum { HH_F16 = 2 };                                    /* a further row type of the hh_kv4 calls */
/*
 * Weight formats.  HH_WF_DTYPE: the weights are used as loaded (cfg.dtype).
 * HH_WF_Q4G32 (bf16 models only): the paper's mouth model runs 4-bit weights
 * (Sec. 4 "Runtime phase", Sec. 5) without naming the format; this library's
 * 4-bit format is symmetric per group of 32 consecutive elements of a row:
 * scale s = bf16(max|w| / 7) (fp32 division, round to nearest even), codes
 * q = clamp(rint(w / s), -8, 7) (fp32 division, ties to even), value q * s.
 * At load the bf16 matrices are quantized row by row (W_q, W_k, W_v, W_o,
 * W_gate, W_up along their input dimension, W_down along its output
 * dimension, i.e. the rows of W_down^T, and the LM head's copy of the
 * embedding); the token-embedding table stays bf16.  Every kernel then
 * computes with the values q * s.
 */
enum { HH_WF_DTYPE = 0, HH_WF_Q4G32 = 1 };
/*
 * Added to a weight format (either, of either dtype): the context keeps its
 * KV cache in 4 bits, in the pages of hh_kv4_append below, quantized as keys
 * (rotated) and values are produced.  72 bytes a position and kv head take the place of
 * fp16's 256 (fp32's 512).  Prompts and decode steps run as otherwise, batch-1 steps
 * through the kernels of the multi-stream ones (the first step past each power of
 * two of the longest stream's pages captures its graph); hh_decode_step_noalloc
 * gives HH_ERR_UNSUPPORTED.  A context is created with one or the other cache.
 */
enum { HH_KV_Q4 = 0x100 };
/*
 * The same with 8 bits, in the pages of hh_kv8_append below (136 bytes a position and kv
 * head).  A page's scale grows as its positions come and stays when a stream is cut, so a prompt
 * that is evaluated in other passes, or a stream that was longer, may differ by what its codes are
 * rounded again.
 * Either cache pays where streams are many or long; a single stream's steps are slower than with a
 * 16-bit one (1B decoder, 8 bits: 0.93 ms for 0.63 at 256 positions, 0.99 for 0.74 at 8,192; 32
 * streams at 4,000 1.34 for 1.68).
 */
enum { HH_KV_Q8 = 0x400 };
enum { HH_LOGITS_NONE = 0, HH_LOGITS_LAST = 1, HH_LOGITS_ALL = 2 };

/*
 * Model and capacity description.  Supported: head_dim == 64, page_size == 16,
 * n_heads / n_kv_heads in {1, 2, 4, 8}, d_model % 64 == 0, ffn_dim % 8 == 0,
 * vocab >= 2, max_context <= 131072; anything else gives HH_ERR_UNSUPPORTED.  rms_eps is added to the mean square inside the root;
 * rope_theta is the rotary base (frequencies theta^(-2i/head_dim)).
 */
typedef struct {
  int32_t n_layers, d_model, n_heads, n_kv_heads, head_dim, ffn_dim, vocab;
  float rms_eps, rope_theta;
  int32_t tied_embeddings;   /* 1: LM head is the embedding matrix           */
  int32_t dtype;             /* HH_F32 or HH_BF16: weights and KV cache      */
  int32_t max_streams;       /* independent sequences held at once (>= 1)    */
  int32_t max_context;       /* positions per stream (prompt + generated)    */
  int32_t page_size;         /* KV page length in tokens; must be 16         */
  int32_t max_prefill;       /* rows per prefill pass; 0 means max_context.
                                Longer prompts are processed in passes.      */
  int32_t weight_format;     /* HH_WF_DTYPE or HH_WF_Q4G32 (dtype HH_BF16,
                                d_model % 32 == 0); + HH_KV_Q4 or HH_KV_Q8   */
} hh_config;

typedef struct hh_ctx hh_ctx;

/* Bytes of device memory hh_create needs for this configuration. */
hh_status hh_workspace_size(const hh_config* cfg, size_t* bytes);

/*
 * Create a context inside a caller-owned device arena.
 *  arena       device pointer, 256-byte aligned, at least hh_workspace_size()
 *              bytes; it holds weights, KV pages, RoPE tables and scratch and
 *              must outlive hh_destroy.  The library never allocates device
 *              memory of its own.
 *  hip_stream  hipStream_t to enqueue on; must not be the legacy NULL stream
 *              (decode steps are replayed as HIP graphs captured on it).
 *  out         receives the context (host object owned by the library).
 * Errors: INVALID_ARG (NULL/unaligned arena, NULL stream), UNSUPPORTED, OOM.
 */
hh_status hh_create(const hh_config* cfg, void* arena, size_t arena_bytes, void* hip_stream,
                    hh_ctx** out);

/*
 * Copy the model weights into the arena (repacking them for the kernels).
 *  tensors    n_tensors pointers, host or device, element type cfg.dtype
 *             (float or bf16 bits), row-major [out, in] as in nn.Linear:
 *               embed[vocab, d];
 *               per layer: attn_norm[d], wq[Hq*64, d], wk[Hkv*64, d],
 *                          wv[Hkv*64, d], wo[d, Hq*64], mlp_norm[d],
 *                          w_gate[F, d], w_up[F, d], w_down[d, F];
 *               final_norm[d]; lm_head[vocab, d] only if untied.
 *  n_tensors  must be 1 + 9 * n_layers + 1 (+1 if untied).
 * The caller may free the sources after return (the call synchronizes).
 * Loading resets every stream.  Errors: INVALID_ARG, HIP.
 */
hh_status hh_load_weights(hh_ctx* ctx, const void* const* tensors, int32_t n_tensors);

/*
 * Prompt evaluation (the TTFT step): append n_tokens tokens to stream
 * stream_id, starting at its current length, and compute the greedy next
 * token from the last row.
 *  tokens       host, n_tokens ids in [0, vocab).
 *  logits_mode  HH_LOGITS_NONE, _LAST (logits = [vocab]) or _ALL
 *               (logits = [n_tokens, vocab]); fp32, host or device.
 *  next_token   NULL or one int32 (host or device): argmax of the last row,
 *               lowest index among ties.  The same token is kept on the
 *               device as the stream's pending token for hh_decode_step.
 * Errors: INVALID_ARG (id out of range, n_tokens <= 0, NULL logits with a
 * logits mode), CONTEXT_FULL, NOT_LOADED, HIP.
 */
hh_status hh_prefill(hh_ctx* ctx, int32_t stream_id, const int32_t* tokens, int32_t n_tokens,
                     int32_t logits_mode, float* logits, int32_t* next_token);

/*
 * Prompt evaluation for several streams together (several requests
 * arriving together, the paper's runtime phase at more than one user): the
 * prompts of n distinct streams are appended as one set of rows, every layer
 * runs over all of them (each row attends to its own stream's keys up to its
 * position), and the greedy next token of each stream comes from its last
 * row, as hh_prefill would give it.  Rows go through in passes of at most
 * max_prefill rows (max_context when 0, and at least max_streams), in
 * stream_ids order; a prompt that does not fit in what is left of a pass
 * continues in the next one.
 *  stream_ids   host, n distinct ids; lengths host, n counts >= 1.
 *  tokens       host, the prompts concatenated in stream_ids order
 *               (sum of lengths ids in [0, vocab)).
 *  next_tokens  NULL or n int32 (host or device), in stream_ids order.
 * The call waits for its passes to finish.  Errors: INVALID_ARG (n outside
 * 1..max_streams, an id out of range or repeated, a length < 1, a token out
 * of range), CONTEXT_FULL, NOT_LOADED, HIP.
 */
hh_status hh_prefill_batch(hh_ctx* ctx, int32_t n, const int32_t* stream_ids, const int32_t* lengths,
                           const int32_t* tokens, int32_t* next_tokens);

/*
 * One greedy decode step of n_streams streams in lockstep: each listed stream
 * consumes one token at its current length and advances by one.
 *  stream_ids   host, n_streams distinct ids; NULL means 0..n_streams-1.
 *  tokens       host, n_streams ids to consume (teacher forcing), or NULL to
 *               consume each stream's pending token (the previous argmax,
 *               kept on the device: no host round trip).
 *  logits       NULL or [n_streams, vocab] fp32, host or device.
 *  next_tokens  NULL or [n_streams] int32, host or device.
 * A stream with no tokens yet decodes at position 0 (its pending token must
 * then be given through tokens).  Errors: INVALID_ARG, CONTEXT_FULL,
 * NOT_LOADED, HIP.
 * Failure of a batch-1 step: every cross-workgroup wait of the single-kernel
 * step is bounded (about 1 s).  When one gives up, the step's token is -1
 * (pending token, next_tokens, and the history hh_read_argmax returns), and
 * so is the token of every later step of that stream, and of every step of
 * any stream until hh_reset; the first call with host outputs after the
 * failure returns HH_ERR_HIP.  Device-fed loops detect it by the -1.
 */
hh_status hh_decode_step(hh_ctx* ctx, int32_t n_streams, const int32_t* stream_ids,
                         const int32_t* tokens, float* logits, int32_t* next_tokens);

/*
 * For callers that cannot allocate device memory (code under HIP graph
 * capture, tight serving loops, harnesses that forbid allocation): one greedy
 * batch-1 decode step of stream_id, as hh_decode_step with n_streams == 1,
 * whose cross-workgroup exchange words live in a fixed array the library
 * keeps in each device's memory (9 MiB per device, held until the process
 * ends) instead of the context's arena.  The call allocates nothing and
 * captures no graph: it enqueues a small fill of the array's error word and
 * the single-kernel step on the context's stream.
 *  token        host, one id to consume, or NULL for the stream's pending
 *               token.
 *  logits       NULL or [vocab] fp32, host or device.
 *  next_token   NULL or one int32, host or device.
 * Every context on a device shares that device's array, and it keeps the
 * last step's contents: steps of different contexts that overlap in time on
 * one device (different streams, no ordering between them) race and give
 * wrong results.  Steps in one stream's order are safe.
 * Errors: as hh_decode_step; UNSUPPORTED when the configuration has no
 * single-kernel step or needs more exchange words than the array holds
 * (d_model 2048 with 32 query heads fits up to 256 workgroups); INVALID_ARG
 * when the context's device is not the current one.
 */
hh_status hh_decode_step_noalloc(hh_ctx* ctx, int32_t stream_id, const int32_t* token, float* logits,
                                 int32_t* next_token);

/* Drop a stream's KV pages and set its length to 0 (stream_id -1: all).
 * Also clears the context's record of a failed decode step (see
 * hh_decode_step). */
hh_status hh_reset(hh_ctx* ctx, int32_t stream_id);

/*
 * Fork a stream: each listed stream becomes a copy of stream src -- its
 * positions, pending token and argmax history -- and goes on by itself.  Full KV
 * pages are shared between the streams until each drops them; the partly
 * filled last page is copied.  What the listed streams held is dropped.  So
 * several answers to one prompt, or prompts with a common beginning, take one
 * prompt evaluation of it.
 *  dst  host, n distinct stream ids other than src.
 * Only enqueues.  Errors: INVALID_ARG (an id out of range, repeated or src, n
 * outside 1..max_streams - 1), OOM (host memory), HIP; after HIP each listed stream is
 * forked, or as it was, or empty.
 */
hh_status hh_fork(hh_ctx* ctx, int32_t src, int32_t n, const int32_t* dst);

/*
 * Cut a stream to its first `length` positions and free the KV pages behind
 * them (a page that another stream shares stays; one that this stream will
 * write to again is copied first).  The stream's pending token becomes the argmax recorded at
 * position length - 1; where none was (inside a prompt), the next
 * decode step of the stream must be given its token.  length 0 is as
 * hh_reset of the stream, but for the record of a failed step.
 * Only enqueues.  Errors: INVALID_ARG (an id out of range, length < 0 or past
 * the stream's), HIP; the stream is then as it was.
 */
hh_status hh_truncate(hh_ctx* ctx, int32_t stream_id, int32_t length);

/*
 * Move the KV pages that streams hold to the lowest page ids (hh_kv_compact's
 * rule), in every layer; results do not change.  After it the pages that are
 * in use, *pages_in_use of them (may be NULL), lie together at the start of each layer's
 * pool.  Only enqueues.  Errors: UNSUPPORTED (over 2^20 pages), OOM (host
 * memory), HIP.
 */
hh_status hh_compact(hh_ctx* ctx, int32_t* pages_in_use);

/* Current length (positions held in the KV cache) of a stream. */
hh_status hh_stream_length(const hh_ctx* ctx, int32_t stream_id, int32_t* length);

/*
 * Read back greedy outputs recorded on the device: out[i] is the argmax
 * computed at position first_pos + i of stream_id (i.e. the prediction of the
 * token at position first_pos + i + 1).  Positions must be < the stream's
 * length and must have been the last row of a prefill or a decode step.
 *  out  host, n int32.  Synchronizes the stream.
 */
hh_status hh_read_argmax(hh_ctx* ctx, int32_t stream_id, int32_t first_pos, int32_t n,
                         int32_t* out);

/*
 * The HH_WF_Q4G32 quantizer the loader runs, on its own: quantize rows of
 * bf16 values into the stored row format -- for each row, K / 2 bytes of
 * codes (n = q + 8; element 2k in the low nibble of byte k, 2k + 1 in the
 * high nibble) followed by the K / 32 scales as little-endian bf16, i.e.
 * K / 2 + K / 16 bytes per row.
 *  src         device, rows x K bf16 bits, row-major; finite values.
 *  K           a positive multiple of 32.
 *  dst         device, rows x (K / 2 + K / 16) bytes.
 *  hip_stream  hipStream_t the kernel is enqueued on (not synchronized).
 * Errors: INVALID_ARG (NULL pointer, rows < 1, K not a multiple of 32), HIP.
 */
hh_status hh_q4g32_quantize(const uint16_t* src, int64_t rows, int32_t K, uint8_t* dst, void* hip_stream);

/* Destroy the host context (the arena stays the caller's). NULL is a no-op. */
void hh_destroy(hh_ctx* ctx);

/* Measurement aid, not a step of the decoder: enqueue on hip_stream one pass
 * that reads `bytes` of device memory at src once (16-byte vector loads from
 * every CU) and computes nothing visible.  Timed by the caller with events,
 * it gives the read bandwidth a kernel can reach on the device, the
 * reference the decode kernel's HBM fraction is also reported against.
 * src must be device memory, 16-byte aligned, bytes a positive multiple of
 * 16; otherwise HH_ERR_INVALID_ARG. */
hh_status hh_read_probe(const void* src, size_t bytes, void* hip_stream);

/* ------------------------------------------------------------------------
 * A paged cache in 4 bits: its operators on the caller's own device memory.
 *
 * The KV cache's memory grows with the window (Sec. 6.6); held in 4 bits it
 * is 72 bytes a position and kv head where fp16 takes 256.  Pages hold 16
 * positions, heads have 64 dimensions, as in a context's cache.
 *
 * Values.  Keys and values are quantized in groups of 32 consecutive
 * dimensions of one position and head (two groups a row): the scale s is
 * max|x| / 7 (fp32 division), rounded to nearest even to 8 significant bits
 * and to a multiple of 2^-24, at most 2720; the code is
 * c = clamp(rint(x / s), -7, 7) (fp32 division, ties to even; 0 where s is
 * 0); the value is c * s, which fp16 holds exactly.  Magnitudes above 19,040
 * saturate.  A key or value row (64 dimensions) with an infinity or NaN has
 * NaN as both its scales: what attends it is NaN, as it would be unquantized.
 *
 * Pages.  One page of one kv head is a block of 1,152 bytes; a page is
 * n_kv_heads blocks in head order, a pool n_pages pages.  With n = c + 8 the
 * block's nibbles (j = 0 the lowest of a 16-bit word) and fp16 scales are:
 *   keys    bytes 0 .. 511: the code of (slot, dimension 32 t + 8 g + 2 j + h)
 *           is nibble j of the 16-bit word 4 (16 g + slot) + 2 t + h;
 *   values  bytes 512 .. 1023: the code of (slot, dimension 4 r + j) is
 *           nibble j of the word 4 (16 (slot / 4) + r) + slot % 4;
 *   scales  bytes 1024 .. 1087: keys, at [slot][group];
 *           bytes 1088 .. 1151: values, at [group][slot].
 *
 * All calls enqueue on hip_stream (NULL: the null stream), which must belong
 * to the current device, as must all memory; none of them synchronizes,
 * allocates or keeps anything, so a caller may capture them into a graph.
 * Pointers of the two descriptions below are read by the device when the
 * call's kernels run, the descriptions themselves during the call.
 * ------------------------------------------------------------------------ */

typedef struct {
  void* pool;                 /* device, 16-byte aligned: n_pages * n_kv_heads * 1152 bytes */
  const int32_t* page_table;  /* device [table_rows][max_pages]: page ids in [0, n_pages)   */
  int32_t n_pages, n_kv_heads;
  int32_t max_pages;          /* columns of the page table                                  */
  int32_t table_rows;
} hh_kv4_pool;

/* Rows of one or more sequences, each sequence's consecutive: sequence s has
 * rows row_start[s] .. row_start[s + 1] - 1, at positions first_pos[s],
 * first_pos[s] + 1, ...  A row at a negative position is padding: it has no
 * key, and nothing to attend to. */
typedef struct {
  const int32_t* row_start;   /* device [n_seqs + 1], or NULL: one row each, row s          */
  const int32_t* first_pos;   /* device [n_seqs]                                            */
  const int32_t* table_row;   /* device [n_seqs] rows of the page table, or NULL: row s     */
  int32_t n_seqs;
  int32_t n_rows;             /* rows of the buffers                                        */
  int32_t max_rows;           /* at least the longest sequence's rows (1 without row_start) */
} hh_kv4_rows;

/*
 * Quantize key and value rows into their pages.
 *  k, v      device, 16-byte aligned, [n_rows][n_kv_heads][64] of `dtype`
 *            (HH_F32, HH_F16, HH_BF16) with k_stride and v_stride elements
 *            from row to row (multiples of 16 bytes, at least n_kv_heads * 64),
 *            so rows may be columns of a wider matrix.
 *  rope      NULL, or device [rope_len][32][2] fp32, 16-byte aligned: cos and
 *            sin of position and pair; keys are then rotated at their positions
 *            (pairs i, i + 32), in 64 bits rounded once to fp32, before they
 *            are quantized.
 * Only the slots of the given positions are written.  Rows whose position is
 * negative, or past the page table's max_pages * 16 or rope_len, are skipped.
 * Two rows of one call must not have the same place in the cache.
 * Errors: INVALID_ARG (NULL or misaligned pointers, a size < 1, n_kv_heads over
 * 1,024, max_pages over 2^26, n_rows or max_rows from 2^30 on, a stride, an
 * element type), UNSUPPORTED (max_rows near 2^28 and above), HIP.
 */
hh_status hh_kv4_append(const hh_kv4_pool* pool, const hh_kv4_rows* rows, const void* k, const void* v, int32_t dtype,
                        int64_t k_stride, int64_t v_stride, const float* rope, int32_t rope_len, void* hip_stream);

/* The values that the pages hold for the given rows, into k and v (as in
 * hh_kv4_append; c * s rounded to nearest even to `dtype`).  Rows at
 * positions that have no page are set to 0.  Errors as hh_kv4_append's. */
hh_status hh_kv4_read(const hh_kv4_pool* pool, const hh_kv4_rows* rows, void* k, void* v, int32_t dtype,
                      int64_t k_stride, int64_t v_stride, void* hip_stream);

/* Bytes of device memory that hh_kv4_attention needs for these sizes (their
 * pointers are not read; row_start counts as given or NULL): 0 to
 * HH_KV4_WORKSPACE_MOST.  Fewer sequences or rows may need more, so a caller of
 * calls of several sizes takes the largest or the bound. */
enum { HH_KV4_WORKSPACE_MOST = 16 << 20 };
hh_status hh_kv4_attention_workspace(const hh_kv4_pool* pool, const hh_kv4_rows* rows, int32_t n_heads, size_t* bytes);

/*
 * Causal grouped-query attention over the pages: the row at position p attends
 * to the keys at positions 0 .. p of its sequence's page table row (its own
 * included: append first), query head j to kv head j / (n_heads / n_kv_heads).
 *   out = sum_t w_t v_t,  w = softmax_t(scale * q . k_t)
 *  q, out    device, 16-byte aligned, [n_rows][n_heads][64] of q_dtype and
 *            out_dtype, strides as above (at least n_heads * 64); out must not
 *            overlap q.  n_heads is a multiple of n_kv_heads.
 *  scale     finite, > 0.
 *  rope      NULL, or as above: queries are rotated at their positions first
 *            (in fp32; those from rope_len on as at rope_len - 1).
 *  workspace device, 256-byte aligned, hh_kv4_attention_workspace() bytes (NULL
 *            if that is 0); its contents need not be kept or cleared, and calls
 *            that may run at the same time need one each.
 * Rows at negative positions give 0; rows of `out` in no sequence are left as
 * they are.  Positions past max_pages * 16 - 1 are taken as that.  Sums and
 * softmax are fp32.  In the products, whatever the types and sizes of a call,
 * weights are fp16 pairs (22 bits), and so are queries, scaled by a power of two
 * (16-bit ones that are not rotated are single fp16 numbers, exactly); a weight
 * is 2^-37 of its row's largest off at most, so that smaller ones may count as 0.
 * Scores past fp32 are no error: the largest takes all.  A query with an infinity
 * or NaN gives NaN where its row sees a key.  Equal calls give equal bits.
 * Errors: INVALID_ARG (as above; a workspace that is too small; scale),
 * UNSUPPORTED (max_rows * n_heads near 2^30 and above, n_heads from 2^25 on), HIP.
 */
hh_status hh_kv4_attention(const hh_kv4_pool* pool, const hh_kv4_rows* rows, const void* q, int32_t q_dtype,
                           int64_t q_stride, int32_t n_heads, float scale, const float* rope, int32_t rope_len,
                           void* out, int32_t out_dtype, int64_t out_stride, void* workspace, size_t workspace_bytes,
                           void* hip_stream);

/* ------------------------------------------------------------------------
 * A paged cache in 8 bits, and attention over selected blocks of it, on the
 * caller's own device memory.
 *
 * 136 bytes a position and kv head (fp16 takes 256, the 4-bit cache 72), at a
 * tenth of the 4-bit cache's error where a page's rows are of like magnitude (1.0% of normal
 * values; 1.6%, a sixth, where rows differ by factors of e^(0.3 n), n normal).  A
 * block (the 16 positions of a page of one kv head) has one scale for its keys and one for
 * its values, and a summary of its keys, by which a step over a long stream can choose the
 * blocks that it reads.
 *
 * Values.  A scale is 2^e, e the least integer from -20 to 9 with max|x| <=
 * 127 * 2^e over the block's keys (or values); a code is
 * c = clamp(rint(x / 2^e), -127, 127) (ties to even), the value c * 2^e.
 * Magnitudes above 65,024 saturate.  A key or value row (64 dimensions of a position)
 * with an infinity or NaN is marked, counts for no scale, and is NaN: what attends it
 * is NaN, as it would be unquantized.
 * While a page fills, its scales grow and never shrink: where rows come behind kept ones
 * whose scale is 2^d, e is at least d, and kept codes become rint(c * 2^(d - e)).
 * The summary of a block is m = rint(S / 2^j), S the sum of the key codes over the
 * slots and j the least of 0 .. 4 with max|S| <= 127 * 2^j; m * 2^(e + j - 4) is its
 * mean key.
 *
 * Pages.  One page of one kv head is a block of HH_KV8_BLOCK bytes; a page is
 * n_kv_heads blocks in head order, a pool n_pages pages.  Codes are bytes c + 128:
 *   keys    bytes 0 .. 1023: the code of (slot, dimension 32 h + 8 g + j) is
 *           byte 256 g + 16 slot + 8 h + j;
 *   values  bytes 1024 .. 2047: the code of (slot 4 g + i, dimension 4 r + j)
 *           is byte 1024 + 256 g + 16 r + 4 j + i;
 *   summary bytes 2048 .. 2111: m, int8, by dimension;
 *   scales  fp16 at byte 2112 (keys), 2114 (values), 2120 (summary);
 *   marks   16-bit sets of slots at 2116 (keys), 2118 (values);
 *   bytes 2122 .. 2127 are 0, those from 2128 on neither read nor written.
 *
 * The descriptions are those of the 4-bit cache, with these blocks, and so is what
 * is said there of streams, devices, captures and pointers.
 * Positions live on the device, so that how a call over all keys, or a selection, is cut up goes by
 * max_pages, as if every sequence filled its row of the page table. A table that is as
 * wide as the longest sequence of a call is the fastest: behind one of 8,192 columns a selection for
 * 4,000 rows of 437 blocks takes 458 us (44 behind 438 columns), for 32 rows of 1,400 22 (19), and
 * attention of 32 tokens at 4,000 30 (27), of 6 at 200 9 (5.4). Lists do not depend on it.
 * ------------------------------------------------------------------------ */

enum { HH_KV8_BLOCK = 2176 };
typedef hh_kv4_pool hh_kv8_pool;  /* pool: n_pages * n_kv_heads * 2176 bytes */
typedef hh_kv4_rows hh_kv8_rows;

/*
 * Quantize key and value rows into their pages: arguments, rotation and skipped
 * rows as in hh_kv4_append.
 * A page that rows go to is written whole: its slots in front of the call's first
 * row of that sequence stay (requantized where the scale grows), those behind
 * its last are dropped and hold zeros.  So a sequence ends with its last
 * row, and one that was cut is appended to at its new end.  Sequences of one call must
 * not have rows in the same page, nor may a page be shared that rows go to.
 * Errors as hh_kv4_append's.
 */
hh_status hh_kv8_append(const hh_kv8_pool* pool, const hh_kv8_rows* rows, const void* k, const void* v, int32_t dtype,
                        int64_t k_stride, int64_t v_stride, const float* rope, int32_t rope_len, void* hip_stream);

/* The values that the pages hold for the given rows, into k and v (c * 2^e
 * rounded to nearest even to `dtype`, NaN for marked rows).  Rows at positions that
 * have no page are set to 0.  Errors as hh_kv4_append's. */
hh_status hh_kv8_read(const hh_kv8_pool* pool, const hh_kv8_rows* rows, void* k, void* v, int32_t dtype,
                      int64_t k_stride, int64_t v_stride, void* hip_stream);

/* Bytes of device memory that hh_kv8_attention needs for these sizes: as
 * hh_kv4_attention_workspace. */
enum { HH_KV8_WORKSPACE_MOST = 16 << 20 };
hh_status hh_kv8_attention_workspace(const hh_kv8_pool* pool, const hh_kv8_rows* rows, int32_t n_heads, size_t* bytes);

/*
 * Causal grouped-query attention over the pages: arguments, masks and errors as in
 * hh_kv4_attention (scale at most 2^100).  Sums, softmax and weights are as there too, and so
 * are the queries of calls with max_rows * (n_heads / n_kv_heads) over 16; those of others are
 * whole numbers of 23 bits in the products, each element off by 2^-22 of the query's largest
 * at most.  Scores past fp32 are no error: the largest takes all.  A query with an infinity or
 * NaN gives NaN where its row sees a key.
 */
hh_status hh_kv8_attention(const hh_kv8_pool* pool, const hh_kv8_rows* rows, const void* q, int32_t q_dtype,
                           int64_t q_stride, int32_t n_heads, float scale, const float* rope, int32_t rope_len,
                           void* out, int32_t out_dtype, int64_t out_stride, void* workspace, size_t workspace_bytes,
                           void* hip_stream);

/* Bytes of device memory that hh_kv8_select needs for these sizes: 0 to
 * HH_KV8_WORKSPACE_MOST, as above. */
enum { HH_KV8_MOST_BLOCKS = 1 << 15 };
hh_status hh_kv8_select_workspace(const hh_kv8_pool* pool, const hh_kv8_rows* rows, int32_t n_heads, int32_t n_blocks,
                                  size_t* bytes);

/*
 * For each row and kv head, the n_blocks blocks that score highest.  A row at position
 * p has the blocks 0 .. p / 16 of its sequence (at most max_pages).  The first keep_first
 * and the last keep_last of them are selected, and then those between with the largest
 *   score(b) = (sum_d a_d m_b,d) * 2^(e + j - 4),
 * the block's mean key against the queries of the kv head's group: a_d = rint(Q_d / 2^f),
 * f the least integer with max|Q| <= 127 * 2^f, Q the sum of the group's queries
 * (rotated), in 64 bits.  Scores are exact; among equal ones the lowest block wins.
 * Queries with an element that is not finite score 0 everywhere.
 *  q, rope   as in hh_kv4_attention (rotated in 64 bits).
 *  blocks    device int32 [n_rows][n_kv_heads][n_blocks]: in ascending order, -1
 *            behind the last where a row has fewer; rows at negative positions
 *            get -1 alone, and rows in no sequence are left as they are.
 * Every block but a row's last ones must be full, as appending leaves them
 * (keep_last >= 1 covers its own).
 * Errors: INVALID_ARG (as above; keep_first < 0, keep_last < 1, their sum over
 * n_blocks), UNSUPPORTED (n_blocks or max_pages over 32,768; max_rows * n_kv_heads near 2^22
 * and above), HIP.
 */
hh_status hh_kv8_select(const hh_kv8_pool* pool, const hh_kv8_rows* rows, const void* q, int32_t q_dtype,
                        int64_t q_stride, int32_t n_heads, const float* rope, int32_t rope_len, int32_t n_blocks,
                        int32_t keep_first, int32_t keep_last, int32_t* blocks, void* workspace, size_t workspace_bytes,
                        void* hip_stream);

/* Bytes of device memory that hh_kv8_attention_blocks needs for these sizes: 0 to
 * HH_KV8_WORKSPACE_MOST, as above. */
hh_status hh_kv8_attention_blocks_workspace(const hh_kv8_pool* pool, const hh_kv8_rows* rows, int32_t n_heads,
                                            int32_t n_blocks, size_t* bytes);

/*
 * Attention over listed blocks: a row at position p attends, for each kv head, to the
 * positions 0 .. p that lie in the blocks it lists.
 *  blocks  device int32 [n_rows][n_kv_heads][n_blocks], in any order; entries that
 *          are no block of the row (negative, or past p / 16) are skipped, and one
 *          that is listed twice counts twice.  A row without any gives 0.
 * Otherwise as hh_kv8_attention, queries as in its smaller calls.  Errors: as there, INVALID_ARG (blocks NULL or
 * misaligned, n_blocks < 1), UNSUPPORTED (n_blocks over 32,768).
 */
hh_status hh_kv8_attention_blocks(const hh_kv8_pool* pool, const hh_kv8_rows* rows, const int32_t* blocks,
                                  int32_t n_blocks, const void* q, int32_t q_dtype, int64_t q_stride, int32_t n_heads,
                                  float scale, const float* rope, int32_t rope_len, void* out, int32_t out_dtype,
                                  int64_t out_stride, void* workspace, size_t workspace_bytes, void* hip_stream);

/* ------------------------------------------------------------------------
 * Pages of any paged cache: n_layers pools of n_pages pages of page_bytes, a
 * pool every layer_stride bytes from `pool` (device, 16-byte aligned;
 * page_bytes and layer_stride multiples of 16, page_bytes at most 64 MiB;
 * layer_stride at least n_pages * page_bytes where there are several layers).
 * Streams, devices and captures as above; hh_kv_copy_pages takes n_pages bytes
 * of host memory for its checks while it runs.
 * ------------------------------------------------------------------------ */

/*
 * Copy page src[i] to page dst[i] in every layer, i < n: a fork's last page, a
 * stream's pages to another pool position.
 *  src, dst  host, page ids, read during the call.  A page may be the source of
 *            several copies.
 * Errors: INVALID_ARG (NULL or misaligned pointers, sizes, an id out of range,
 * a destination that is listed twice or is a source), OOM (host memory), HIP.
 */
hh_status hh_kv_copy_pages(void* pool, int32_t n_layers, int64_t layer_stride, int64_t page_bytes, int32_t n_pages,
                           int32_t n, const int32_t* src, const int32_t* dst, void* hip_stream);

/* Bytes of device memory hh_kv_compact needs for a pool of n_pages pages. */
hh_status hh_kv_compact_workspace(int32_t n_pages, size_t* bytes);

/*
 * Move the live pages to the lowest ids, on the device, so that what lies
 * behind them can be given back.  A page is live if an entry
 * page_table[r][i], i < ceil(lengths[r] / 16), names it (several may: shared
 * pages stay shared).  With L live pages, the live pages with ids >= L go, in
 * ascending order, to the free ids < L in ascending order; no other page is
 * touched, and the entries are rewritten.  Entries past a row's length stay as
 * they are; entries out of range name no page and stay as well.
 *  page_table  device [table_rows][max_pages].
 *  lengths     device [table_rows], positions held by each row.
 *  live        device, receives L.
 *  workspace   device, 256-byte aligned, hh_kv_compact_workspace() bytes, one
 *              for each call that may run at the same time; contents as above.
 * Errors: INVALID_ARG, UNSUPPORTED (n_pages over 2^20), HIP.
 */
hh_status hh_kv_compact(void* pool, int32_t n_layers, int64_t layer_stride, int64_t page_bytes, int32_t n_pages,
                        int32_t* page_table, int32_t table_rows, int32_t max_pages, const int32_t* lengths,
                        int32_t* live, void* workspace, size_t workspace_bytes, void* hip_stream);

/* Message of the last error on this context ("" if none); never NULL. */
const char* hh_last_error(const hh_ctx* ctx);

#ifdef __cplusplus
}
#endif

#endif /* HH_H_ */
