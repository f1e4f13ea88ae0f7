/*
 * fp.h -- C ABI of the MI355X fingerprint forward pass.
 *
 * A fingerprint (iServe, arXiv 2501.13111, Sec. 1 and Sec. 5.1, Fig. 2) is an
 * LLM cut down to a few hidden layers that keep the architecture's components.
 * iServe's Profiler deploys it and sends dummy requests to measure the time to
 * first token and the time per output token (Sec. 4.2, Sec. 5.3, Eq. 1):
 * a prefill over the prompt, then one KV-cached decode step per output token.
 * This library runs that forward pass for Llama-style decoder layers on one
 * gfx950 GPU under the compression settings the paper searches over
 * (Sec. 3.2, Table A.1): bf16 weights, int8 per-channel or int4 group-128
 * weight-only quantisation, and a bf16 or int8 KV cache.
 *
 * Conventions shared by every call:
 *  - Device pointers are HIP device addresses; host pointers are plain host
 *    memory.  "stream" is a hipStream_t passed as void* (NULL = the default
 *    stream).  Enqueuing calls return as soon as the work is queued; buffers
 *    must stay valid until the stream has passed them.
 *  - Activations are bf16 bit patterns (uint16), contiguous, row-major.
 *  - Every argument and state check happens on the host before any launch;
 *    on error nothing is modified and a negative fp_status is returned, with
 *    a message available from fp_last_error() (thread-local).
 *  - A handle is not thread-safe: calls on one handle must be serialised.
 *  - The library allocates and owns weights, KV cache and workspace; the
 *    caller owns the x / y buffers it passes.
 */
#ifndef FP_MI355X_H
#define FP_MI355X_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    FP_OK = 0,
    FP_ERR_INVALID_ARG = -1,   /* bad pointer, shape, size or enum */
    FP_ERR_STATE = -2,         /* call not allowed in the handle's state (decode before prefill) */
    FP_ERR_CAPACITY = -3,      /* batch / prompt / sequence beyond what the handle was created for */
    FP_ERR_OOM = -4,           /* device allocation failed */
    FP_ERR_HIP = -5,           /* HIP runtime error (no device, launch failure, ...) */
    FP_ERR_UNSUPPORTED = -6    /* valid request the library does not implement */
} fp_status;

/* Weight compression (Sec. 3.2). */
typedef enum {
    FP_WQ_BF16 = 0,          /* unquantised 16-bit weights */
    FP_WQ_INT8_CHANNEL = 1,  /* symmetric int8, one fp16 scale per output row */
    FP_WQ_INT4_G128 = 2,     /* asymmetric int4, fp16 scale and integer zero per 128 inputs */
    FP_WQ_BF16_2OF4 = 3      /* 2:4 semi-structured sparse bf16 (pruning, Sec. 3.3, Table A.1):
                                in every 4 consecutive inputs of a row the 2 weights of largest
                                magnitude are kept (the lower input first among equal ones);
                                runs on the sparse matrix cores */
} fp_weight_quant;

/* KV-cache compression (Sec. 3.2, "KV-cache quantization"). */
typedef enum {
    FP_KV_BF16 = 0,
    FP_KV_INT8 = 1           /* int8 codes, one fp16 scale per (sequence, position, kv head) */
} fp_kv_quant;

/* Layer-stack shape and capacity, fixed at creation.
 * Requirements (checked by fp_layer_create on the host):
 *  - every field > 0, rms_eps > 0, rope_theta > 0                 (else FP_ERR_INVALID_ARG)
 *  - n_heads % n_kv_heads == 0                                      (FP_ERR_INVALID_ARG)
 *  - hidden, n_heads*head_dim and ffn multiples of 16, of 128 for int4 weights (their
 *    groups run along every projection's input dimension)          (FP_ERR_INVALID_ARG)
 *  - max_seq >= max_prompt (max_seq == max_prompt leaves no room for a decode step
 *    after a full-length prompt)                                    (FP_ERR_INVALID_ARG)
 *  - vocab >= 0 and a multiple of 16                              (FP_ERR_INVALID_ARG)
 *  - 2:4 sparse weights: hidden, n_heads*head_dim and ffn multiples of 64 (FP_ERR_INVALID_ARG)
 *  - head_dim 64 or 128; query group n_heads / n_kv_heads from 1 to 16;
 *    max_batch <= 64; max_batch * max_prompt <= 2^24               (FP_ERR_UNSUPPORTED) */
typedef struct {
    int32_t n_layers, hidden, n_heads, n_kv_heads, head_dim, ffn;
    int32_t max_batch, max_prompt, max_seq;
    float rms_eps;      /* RMSNorm epsilon, inside the square root (1e-5) */
    float rope_theta;   /* rotary base (1e4) */
    int32_t vocab;      /* 0: hidden layers only (requests on hidden states); > 0 (a multiple
                           of 16): the fingerprint also keeps the token embedding, the final
                           norm and the LM head (Sec. 5.1, Fig. 2) for requests on token ids */
} fp_shape;

typedef struct fp_layer fp_layer;   /* opaque: weights, KV cache, workspace, position */

/* Tensor ids (weights of layer l are synthesised from (seed, l, id)). */
enum {
    FP_T_ATTN_NORM = 0, FP_T_Q = 1, FP_T_K = 2, FP_T_V = 3, FP_T_O = 4,
    FP_T_MLP_NORM = 5, FP_T_GATE = 6, FP_T_UP = 7, FP_T_DOWN = 8,
    FP_T_INPUT = 15,     /* prompt hidden states, layer id -1 */
    /* the blocks outside the hidden layers (layer id -1), present when vocab > 0; all
     * bf16 under every weight format (the weight-only quantisation of Sec. 3.2 applies
     * to the hidden layers' projections) */
    FP_T_EMBED = 16,     /* token embedding [vocab, hidden], ~N(0, 0.02) */
    FP_T_FINAL_NORM = 17,/* final RMSNorm gain [hidden], 1 + N(0, 0.02) */
    FP_T_LM_HEAD = 18    /* LM head [vocab, hidden], ~N(0, 0.02) */
};

/*
 * Build a fingerprint: allocate weights, KV cache and workspace on the current
 * device and synthesise the weights from `seed` (the Generator of Sec. 5.1
 * reads a checkpoint; here weights ~N(0, 0.02) and norm gains 1 + N(0, 0.02)
 * come from the counter-based generator of fp_fill_normal), then quantise them
 * on the device.  Synchronous.  *out receives the handle (NULL on error).
 */
fp_status fp_layer_create(const fp_shape* shape, fp_weight_quant wq, fp_kv_quant kvq,
                          uint64_t seed, fp_layer** out);

/*
 * Validation-only handle with no device storage: fp_prefill / fp_decode_step
 * check their arguments and advance the host-side state exactly as a real
 * handle does, but enqueue no work; export calls return FP_ERR_STATE.  Needs
 * no GPU (host-side tests of the argument and state checks).
 */
fp_status fp_layer_create_unbacked(const fp_shape* shape, fp_weight_quant wq, fp_kv_quant kvq,
                                   uint64_t seed, fp_layer** out);

/* Free everything the handle owns: weights, KV cache, workspace and captured decode
 * graphs (synchronises the device first).  NULL is a no-op.  The handle is the
 * fingerprint the Profiler deploys (Sec. 4.2, Sec. 5.1); destroying it ends its
 * deployment. */
fp_status fp_layer_destroy(fp_layer* layer);

/*
 * Prefill (time to first token, Sec. 5.3): run the layer stack over a prompt.
 * x: device bf16 [B, P, hidden], y: device bf16 [B, P, hidden] (may not alias x).
 * Resets the KV cache of the B sequences and sets the position to P.
 * 1 <= B <= max_batch, 1 <= P <= max_prompt.  A prefill with a batch other than
 * the previous one drops the decode graphs captured for that batch (it waits for
 * the device to finish their replays first).
 */
fp_status fp_prefill(fp_layer* layer, const void* x, int32_t B, int32_t P, void* y, void* stream);

/*
 * One decode step (time per output token, Sec. 5.3): the B sequences of the
 * last prefill each take one token's hidden state at the current position,
 * append its K/V to the cache, attend over the whole prefix and produce the
 * layer stack's output; the position then advances by one.
 * x: device bf16 [B, hidden] (normally the previous output fed back), y: device
 * bf16 [B, hidden], no aliasing.  FP_ERR_STATE before a prefill,
 * FP_ERR_CAPACITY when the position has reached max_seq.
 */
fp_status fp_decode_step(fp_layer* layer, const void* x, void* y, void* stream);

/*
 * n consecutive decode steps, each step's output fed back as the next step's input
 * (the fingerprint generating n tokens, Sec. 5.3).  Step 1 reads x and writes y,
 * step 2 reads y and writes x, and so on: the last step's output ends in y when n
 * is odd and in x when n is even.  x and y: device bf16 [B, hidden] each, both
 * written, no aliasing.  With the decode graph on (fp_set_decode_graph), the n
 * steps are captured once per (x, y, n) and replayed as one graph, which saves the
 * steps' launches; the results equal n calls of fp_decode_step.  The
 * position advances by n.  FP_ERR_INVALID_ARG for n < 1, NULL or overlapping
 * buffers; FP_ERR_STATE before a prefill; FP_ERR_CAPACITY when fewer than n
 * positions remain before max_seq (nothing runs).
 */
fp_status fp_decode_steps(fp_layer* layer, void* x, void* y, int32_t n, void* stream);

/*
 * For callers that cannot allocate device memory (code under HIP graph capture, tight
 * serving loops, harnesses that forbid allocation): one decode step exactly as
 * fp_decode_step computes it (same kernels, same results bit for bit), launched
 * kernel by kernel with no graph instantiation and no allocation of any kind.  The
 * step's split-K partials, attention partials and row-norm sums live in a static
 * 64 MiB device region per GPU (held from the first call on that GPU until the
 * process ends) instead of the handle's workspace.  Every call on one GPU shares that
 * GPU's region: calls that overlap on one GPU (other streams, other threads, other
 * handles) race, so serialise them.  FP_ERR_CAPACITY, with nothing launched, when
 * the step at the active batch needs more than 64 MiB of scratch (the message gives
 * the size); otherwise the same argument and state errors as fp_decode_step.
 */
fp_status fp_decode_step_noalloc(fp_layer* layer, const void* x, void* y, void* stream);

/*
 * Replay the steps of fp_decode_steps and fp_generate as a captured HIP graph (1, the
 * default) or launch the kernels one by one (0).  Results are identical.  Graphs are
 * captured on first use per (x, y, n, active batch) for fp_decode_steps; each cache holds
 * at most 16 graphs and is emptied (after a device synchronisation) when a new capture
 * would exceed that.  fp_decode_step launches its kernels one by one (a graph per single
 * step takes longer), except that with 1 the inner layers of a fingerprint of many small
 * layers are one graph, captured on the first step of each batch size and kept for every x
 * and y (at most 16, likewise); with 1 it refuses a stream that is being captured.
 */
fp_status fp_set_decode_graph(fp_layer* layer, int32_t enable);

/*
 * Synthetic data on the device: dst[i] = bf16(mean + sigma * z_i), i < n, where
 * z_i is element i of the Irwin-Hall-12 stream of (seed, layer, tensor):
 *   key = mix64(mix64(seed) + G*(((layer+1) << 8) | tensor)),
 *   words mix64(key + G*(c+1)) for c = 3i..3i+2, z_i = (sum of their twelve
 *   16-bit lanes - 393210) * 2^-16, with mix64 the SplitMix64 finaliser
 *   (Steele, Lea & Flood, OOPSLA 2014) and G = 0x9E3779B97F4A7C15.
 * Prompts use layer -1, tensor FP_T_INPUT, mean 0, sigma 1.  dst: device bf16 [n].
 */
fp_status fp_fill_normal(void* dst, int64_t n, uint64_t seed, int32_t layer, int32_t tensor,
                         float mean, float sigma, void* stream);

/*
 * The fingerprint's blocks outside the hidden layers (Sec. 5.1, Fig. 2), for handles
 * created with vocab > 0 (FP_ERR_STATE otherwise).  Their time is the "other" share
 * of TTFT and TPOT in Eq. 2 and Eq. 3 (Sec. 5.3).
 *
 * fp_embed: x[m] = row ids[m] of the embedding table, m < M.  ids: device int32 [M];
 * x: device bf16 [M, hidden].  An id outside [0, vocab) gives a row of zeros.
 */
fp_status fp_embed(fp_layer* layer, const int32_t* ids, int64_t M, void* x, void* stream);

/*
 * fp_head: final RMSNorm and LM head of the last position of each of B sequences, then
 * greedy decoding.  y: device bf16 [B, T, hidden] (a decode step's output has T = 1, a
 * prefill's T = P); the head reads position T - 1 of each sequence:
 *   yn = bf16(y * rsqrt(mean(y^2) + eps) * g_final),  logits = yn W_lm^T (fp32),
 *   next_ids[b] = argmax_v logits[b, v], the lowest v among equal maxima.
 * logits: device fp32 [B, vocab], or NULL; next_ids: device int32 [B].
 * 1 <= B <= max_batch, T >= 1.
 */
fp_status fp_head(fp_layer* layer, const void* y, int32_t B, int32_t T, float* logits, int32_t* next_ids,
                  void* stream);

/*
 * fp_generate: one dummy request on token ids (the Profiler's request, Sec. 4.2 and
 * Sec. 5.3): embed the prompt, prefill, head -> token 0 (the first token); then n_out
 * decode steps, step i embedding token i - 1 and producing token i.  Output length
 * n_out is the number of decode steps (Eq. 1: latency = TTFT + n_out * TPOT).
 *   prompt_ids: device int32 [B, P];  out_ids: device int32 [n_out + 1, B];
 *   logits: device fp32 [n_out + 1, B, vocab], or NULL;
 *   force_ids: NULL, or device int32 [n_out, B]: step i embeds force_ids[i - 1] instead
 *     of its own token i - 1 (teacher forcing, for parity checks); out_ids still
 *     receives the generated tokens;
 *   elapsed_ms: NULL, or receives the request's device time (events recorded on
 *     `stream` around it; the call then synchronises the stream).
 * Resets the cache of the B sequences like fp_prefill; the position ends at P + n_out.
 * The n_out decode steps replay as one captured graph per (out_ids, logits, force_ids,
 * n_out, B) while the decode graph is on.  1 <= B <= max_batch, 1 <= P <= max_prompt,
 * n_out >= 0, P + n_out <= max_seq (FP_ERR_CAPACITY).
 */
fp_status fp_generate(fp_layer* layer, const int32_t* prompt_ids, int32_t B, int32_t P, int32_t n_out,
                      int32_t* out_ids, float* logits, const int32_t* force_ids, float* elapsed_ms,
                      void* stream);

/*
 * Paged KV cache.  A serving profiler's requests are ragged: sequences of different
 * lengths, prompts taken in chunks, a few drafted tokens checked at once.  These calls
 * work on one layer's cache held in pages of page_size positions, which the caller
 * allocates and hands out; the storage formats are those of the handle's own cache
 * (FP_KV_BF16, or FP_KV_INT8 with one fp16 scale per position and kv head).
 *
 * Layout, ps = page_size, nkv = n_kv_heads, d = head_dim, e = bf16 or int8:
 *   k [n_pages, nkv, ps, d] of e: rows of keys (after the rotary embedding);
 *   v [n_pages, nkv, ps / 32, d, 32] of e: values transposed in blocks of 32 positions,
 *     position t of a block in slot 8 ((t % 16) / 4) + 4 (t / 16) + t % 4 (the order in
 *     which the attention kernels' probabilities leave the matrix cores);
 *   k_scales, v_scales fp16 [n_pages, nkv, ps] (FP_KV_INT8; unused with FP_KV_BF16).
 * page_size is a multiple of 32, up to 65536; head_dim 64 or 128; n_pages * nkv * (ps / 32)
 * below 2^31.  Positions that no call has written may hold anything, NaN included: nothing
 * reads them into a result.  A page may appear in several sequences' tables (a shared
 * prefix) as long as no chunk writes it in two of them.
 */
typedef struct {
    int32_t format;              /* fp_kv_quant */
    int32_t n_pages, page_size, n_kv_heads, head_dim;
    void* k;
    void* v;
    uint16_t* k_scales;
    uint16_t* v_scales;
} fp_paged_kv;

/*
 * A chunk: a ragged batch of rows (tokens) of n_seqs sequences.  Sequence b owns rows
 * row_start[b] .. row_start[b + 1] - 1, none or several; row row_start[b] + i sits at
 * position ctx_len[b] + i, and position p of sequence b lives in page
 * table[b * table_stride + p / page_size] at offset p % page_size.  The three arrays are
 * device int32 (row_start has n_seqs + 1 entries, not decreasing), read when the kernels
 * run, so a captured call follows their later contents.  The host knows only the bounds:
 *   n_rows   rows of the row buffers; rows from row_start[n_seqs] on belong to no sequence
 *            and are left as they are
 *   max_new  bound on a sequence's rows
 *   max_len  bound on ctx_len[b] + rows of b, at most table_stride * page_size and 2^31 - 1024
 * The bounds size the launches (tight ones are faster).  Contents that break them, or a page
 * number outside [0, n_pages), are no error and touch no memory outside the buffers: rows
 * beyond max_new are not computed, positions from max_len on are neither written nor read,
 * and a missing page takes no writes and reads as zeros.
 * 1 <= n_seqs <= 4096, 0 <= n_rows <= 2^24 (0: nothing to do), 1 <= max_new, max_len.
 */
typedef struct {
    int32_t n_seqs, n_rows, max_new, max_len, table_stride;
    const int32_t* row_start;
    const int32_t* ctx_len;
    const int32_t* table;
} fp_chunk;

/*
 * Write a chunk's keys and values into the pages.  k, v: device bf16, row r's head h at
 * k + r * kv_stride + h * head_dim (the stride in elements, so that k and v may be columns of
 * one fused projection).  FP_KV_INT8: s = fp16(absmax / 127), code = rint(x / s) clamped to
 * +-127 per (position, kv head), in fp32 with ties to even; a zero scale gives zero codes.  A NaN, an
 * infinity or an absmax of 127 * 65520 and more leaves a scale that is not finite: that position and head reads
 * back as NaN throughout, and so do the rows of an attention that see it.
 * With cos and sin (device fp32 [n_pos, head_dim / 2], n_pos >= max_len; both or neither)
 * keys are first rotated by their position (rotate-half: i pairs with i + d / 2), in fp32.
 * With q (then q_out, n_heads, a multiple of n_kv_heads of at most 16 times as many; and cos and
 * sin) the queries are rotated in the same launch: q like k with q_stride, q_out device bf16
 * [n_rows, n_heads, head_dim], not overlapping q.  Pointers and strides are multiples of 16 bytes.
 */
fp_status fp_kv_append(const fp_paged_kv* kv, const fp_chunk* chunk, const void* k, const void* v, int64_t kv_stride,
                       const void* q, int64_t q_stride, int32_t n_heads, void* q_out, const float* cos_t,
                       const float* sin_t, int32_t n_pos, void* stream);

/*
 * Read positions back: row r of k_out and v_out (device bf16 [n_rows, n_kv_heads, head_dim],
 * 16-byte aligned) receives the key and value at row r's position; int8: bf16(code * scale).
 * With ctx_len zero and row_start the running sum of the lengths, whole sequences.
 */
fp_status fp_kv_read(const fp_paged_kv* kv, const fp_chunk* chunk, void* k_out, void* v_out, void* stream);

/*
 * Attention of a chunk over the cache, causal: out[r, h] = sum_j p_j v_j over the positions
 * j = 0 .. (row r's position) of r's sequence, p = softmax(scale * q[r, h] . k_j), kv head
 * h * n_kv_heads / n_heads.  The chunk's own keys and values are read from the pages too:
 * append first.  q: device bf16, row r's head h at q + r * q_stride + h * head_dim; out: device
 * bf16 [n_rows, n_heads, head_dim]; both 16-byte aligned.  Query group n_heads / n_kv_heads from
 * 1 to 16; scale below 2^127 in magnitude.  Scores, softmax statistics and sums are fp32; probabilities
 * enter the product with V as bf16 (int8 caches: fp16).  Keys and values that are NaN or infinite reach the rows that see them and no
 * others.  bf16: values below 2^127 in magnitude over up to 2^24 positions cannot overflow the sums.  int8: keys
 * and values below 65504 in magnitude (calls of more than 64 rows per sequence and kv head unpack them to fp16).
 * workspace: device memory of at least fp_attn_chunk_workspace bytes, 16-byte aligned, which
 * the call may use until the stream has passed it (calls that can overlap need one each); enough
 * for one chunk's bounds is enough for any chunk of smaller ones.  FP_ERR_CAPACITY if workspace_bytes
 * is less.
 */
fp_status fp_attn_chunk_workspace(const fp_paged_kv* kv, const fp_chunk* chunk, int32_t n_heads, size_t* bytes);
fp_status fp_attn_chunk(const fp_paged_kv* kv, const fp_chunk* chunk, const void* q, int64_t q_stride, int32_t n_heads,
                        float scale, void* out, void* workspace, size_t workspace_bytes, void* stream);

/*
 * The layer stack over a chunk: fp_prefill and fp_decode_step for ragged batches on the
 * caller's pages (a prompt in pieces, next tokens of sequences of any lengths, drafted tokens,
 * all in one call).  kv: host array of n_layers paged caches (one per layer, the chunk's table
 * naming the same pages in each), with the fingerprint's n_kv_heads and head_dim; their format
 * is their own, whatever cache the handle was created with.  x, y: device bf16 [n_rows, hidden], no
 * aliasing; row r's token sits at its chunk position, its keys and values are written to the
 * pages, its output goes to row r of y (rows of no sequence: unspecified values).  The handle's
 * weights and activations are used, its own cache, position and batch are not touched.
 * n_rows <= max_batch * max_prompt and max_len <= max_seq (FP_ERR_CAPACITY); up to max_batch
 * rows take the decode projections.  workspace: as for fp_attn_chunk (the largest of the
 * layers').  May be captured into a graph; allocates nothing.  The debug dumps are not written.  Another
 * current device than the handle's is refused (FP_ERR_INVALID_ARG).
 */
fp_status fp_extend_workspace(const fp_layer* layer, const fp_paged_kv* kv, const fp_chunk* chunk, size_t* bytes);
fp_status fp_extend(fp_layer* layer, const fp_paged_kv* kv, const fp_chunk* chunk, const void* x, void* y,
                    void* workspace, size_t workspace_bytes, void* stream);

/*
 * Decide over drafted tokens.  Sequence b owns rows row_start[b] .. row_start[b + 1] - 1 of the
 * target's logits (fp32 [n_rows, vocab], row_stride elements apart): row i of it gives the
 * distribution p_i = softmax(logits / temperature) of the token after i accepted drafts.
 * draft_ids[row i] is the drafted token that row i judges (the last row judges none: its entry
 * is not read), drawn from q_i = draft_probs[row i] (fp32 [n_rows, vocab] of draft_stride; NULL:
 * q_i is one at the drafted token).  Drafts are taken in order: x_i is accepted if
 *   u[row i] * q_i(x_i) < p_i(x_i);
 * the first refused one is replaced by a token drawn from max(0, p_i - q_i) (from p_i if that
 * is zero everywhere), and after the last accepted one a token is drawn from the last row's p.  A
 * draw takes the lowest id whose running sum exceeds u_last[b] times the total.  The numbers u
 * and u_last are uniform in [0, 1), the caller's.  All sums and comparisons are in 64 bits.
 * temperature 0: x_i is accepted if it is the row's argmax (the lowest id among equal ones),
 * and the last token is an argmax (u, u_last and draft_probs are not read; may be NULL).
 * out_ids: device int32 [n_seqs, max_rows], sequence b's accepted tokens and then the drawn one,
 * -1 behind; n_out: device int32 [n_seqs], their number (1 .. its rows; a sequence without rows
 * gives 0).  -inf and NaN logits have probability zero; +inf ones share it all.  A row with
 * nothing else gives token -1.  A draft outside [0, vocab) has probability zero; negative and
 * NaN draft probabilities count as zero.
 * row_start: device int32 [n_seqs + 1], not decreasing, entries past n_rows or sequences of more
 * than max_rows rows are cut.  1 <= n_seqs <= 4096, 0 <= n_rows <= 65535, 1 <= max_rows <= 64,
 * 1 <= vocab <= 2^20, finite temperature >= 0.
 */
fp_status fp_verify_draft_workspace(int32_t n_seqs, int32_t n_rows, int32_t vocab, size_t* bytes);
fp_status fp_verify_draft(const float* logits, int64_t row_stride, int32_t n_seqs, int32_t n_rows, int32_t max_rows,
                          int32_t vocab, const int32_t* row_start, const int32_t* draft_ids, const float* draft_probs,
                          int64_t draft_stride, const float* u, const float* u_last, float temperature,
                          int32_t* out_ids, int32_t* n_out, void* workspace, size_t workspace_bytes, void* stream);

/*
 * Latency and memory estimation from fingerprints (host arithmetic, no device).
 *
 * Eq. 1 (Sec. 5.3): latency = TTFT + output_length * TPOT.  fp_fit_ttft_tpot solves the
 * 2x2 system of Eq. 1 at two output lengths.  L2: two fingerprints with layers[0] and
 * layers[1] hidden layers, each timed at the output lengths n_out[0] and n_out[1]
 * (latency[2*i + j]: fingerprint i at length j, any time unit); fp_fit_latency_l2
 * solves each fingerprint's 2x2, then the 4x4 system of Eq. 2 and Eq. 3
 *   TTFT = num_layers * TTFT_layer + TTFT_other,  TPOT = num_layers * TPOT_layer + TPOT_other.
 * fp_predict_latency evaluates Eq. 1-3 for any layer count and output length (NULL
 * outputs skipped).  FP_ERR_INVALID_ARG for NULL inputs or a singular system (equal
 * lengths or equal layer counts).
 */
typedef struct {
    double ttft_layer, tpot_layer, ttft_other, tpot_other;
} fp_latency_model;

fp_status fp_fit_ttft_tpot(const int32_t n_out[2], const double latency[2], double* ttft, double* tpot);
fp_status fp_fit_latency_l2(const int32_t layers[2], const int32_t n_out[2], const double latency[4],
                            fp_latency_model* model);
fp_status fp_predict_latency(const fp_latency_model* model, int32_t n_layers, int32_t n_out, double* ttft,
                             double* tpot, double* latency);

/*
 * M2's layer extrapolation (Sec. 5.2): the value (e.g. a memory footprint) on the straight
 * line through (layers[0], values[0]) and (layers[1], values[1]) at n_layers; footprints
 * grow linearly with the number of hidden layers (Sec. 5, Fig. 7).  FP_ERR_INVALID_ARG
 * for equal layer counts.
 */
fp_status fp_extrapolate_layers(const int32_t layers[2], const double values[2], int32_t n_layers,
                                double* value);

/* Device memory in use on the current device (total - free, hipMemGetInfo) and its
 * total; the observed footprint M2 profiles (Sec. 5.2).  Either pointer may be NULL. */
fp_status fp_device_memory(size_t* used, size_t* total);

/*
 * Copy one weight tensor to host memory in its canonical layout (synchronous).
 * For parity checks of the quantised formats of Sec. 3.2 / Table A.1 (INT8 per
 * channel, INT4 group-128) against an independent implementation:
 *  bf16:  codes = bf16 [N, K] (scales, zeros unused, may be NULL)
 *  int8:  codes = int8 [N, K], scales = fp16 [N]
 *  int4:  codes = int32 [N, K/8] with nibble j of word w holding column 8w+j,
 *         scales = fp16 [N, K/128], zeros = fp16 [N, K/128] (integer values)
 *  2:4:   codes = bf16 [N, K], dense, the pruned weights zero (scales, zeros unused)
 * Norm gains (FP_T_ATTN_NORM, FP_T_MLP_NORM): codes = bf16 [hidden].
 * With vocab > 0 and l = -1: FP_T_EMBED and FP_T_LM_HEAD codes = bf16 [vocab, hidden],
 * FP_T_FINAL_NORM codes = bf16 [hidden].
 * [N, K] is (out, in): q [nh*d, hidden], k/v [nkv*d, hidden], o [hidden, nh*d],
 * gate/up [ffn, hidden], down [hidden, ffn].
 */
fp_status fp_export_weight(fp_layer* layer, int32_t l, int32_t tensor, void* codes, void* scales,
                           void* zeros);

/*
 * Copy layer l's KV cache (the cache that keeps per-token decode cost constant,
 * Sec. 5.3; int8 per Table A.1's KV-cache quantisation) for the active batch to
 * host memory (synchronous).  FP_ERR_STATE before a prefill:
 * k, v: [B, n_kv_heads, max_seq, head_dim] of bf16 or int8; k_scales, v_scales:
 * fp16 [B, n_kv_heads, max_seq] (int8 cache only, else may be NULL).
 */
fp_status fp_export_kv(fp_layer* layer, int32_t l, void* k, void* v, void* k_scales, void* v_scales);

/*
 * Debug: when dev_f32 is non-NULL, every later prefill / decode step also
 * writes the float32 K (after the rotary embedding) and V that enter the KV
 * store of every layer into dev_f32, laid out [n_layers, 2, B, T, n_kv_heads,
 * head_dim] with T the step's token count (P for prefill, 1 for decode);
 * the buffer must hold n_layers*2*max_batch*max_prompt*n_kv_heads*head_dim
 * floats.  NULL switches it off.  Disables graph replay while set.
 */
fp_status fp_set_debug_kv_dump(fp_layer* layer, void* dev_f32);

/*
 * Debug: when dev_bf16 is non-NULL, every later prefill / decode step also
 * copies each layer's output (the bf16 hidden states it hands to the next
 * layer, Sec. 5.1's stack of decoder layers) into dev_bf16, laid out
 * [n_layers, B, T, hidden] with T as above; the buffer must hold
 * n_layers*max_batch*max_prompt*hidden bf16 values and stay valid while set.
 * Lets a test compare each layer against a reference fed that layer's own
 * input.  NULL switches it off.  Disables graph replay while set.
 */
fp_status fp_set_debug_layer_dump(fp_layer* layer, void* dev_bf16);

/*
 * Per-kernel timing (the Profiler of Sec. 4.2 measures latency with dummy
 * requests; this breaks one request's step down by kernel).  Runs one prefill
 * or one decode step exactly as fp_prefill / fp_decode_step do, but launches
 * kernel by kernel with a HIP event recorded on `stream` before each launch and
 * after the last; synchronises, then writes one record per launch into out[]
 * (at most cap records; *count receives the number written).  State changes as
 * for the plain call.
 */
typedef enum {
    FP_K_RMSNORM = 0, FP_K_QKV = 1, FP_K_ROPE_KV = 2, FP_K_ATTN = 3, FP_K_O = 4,
    FP_K_RESID_NORM = 5, FP_K_GATE_UP = 6, FP_K_SWIGLU = 7, FP_K_DOWN = 8, FP_K_POS = 9
} fp_kernel_kind;

typedef struct {
    int32_t kind;    /* fp_kernel_kind */
    int32_t layer;   /* layer index, -1 for step-level kernels */
    float ms;        /* event-to-event device time of the launch */
} fp_kernel_time;

fp_status fp_profile_prefill(fp_layer* layer, const void* x, int32_t B, int32_t P, void* y,
                             void* stream, fp_kernel_time* out, int32_t cap, int32_t* count);
fp_status fp_profile_decode_step(fp_layer* layer, const void* x, void* y, void* stream,
                                 fp_kernel_time* out, int32_t cap, int32_t* count);

/*
 * Bytes of device memory the handle holds for weights (W), KV cache and workspace
 * (the activations A of the memory breakdown mem_base = W + A, Sec. 5.2).  On an
 * unbacked handle: the bytes a real handle of the same shape and formats holds.
 * Weight bytes count the fragment-major codes (K padded to a whole 1 KiB block
 * row-slice), the fp16 scales and zeros, the packed int4 scale/zero words and the
 * bf16 norm gains.  Any output pointer may be NULL.
 */
fp_status fp_memory_bytes(const fp_layer* layer, size_t* weights, size_t* kv, size_t* workspace);

/* Current position (tokens in the cache, Sec. 5.3) and active batch of the handle;
 * both 0 before the first prefill.  Any output pointer may be NULL. */
fp_status fp_get_position(const fp_layer* layer, int32_t* pos, int32_t* batch);

const char* fp_status_str(fp_status status);
const char* fp_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* FP_MI355X_H */
