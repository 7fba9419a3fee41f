/*
 * mixkvq.h — C ABI of the MixKVQ decode hot path for NVIDIA B200 (sm_100a).
 *
 * MixKVQ (arxiv 2512.19206) keeps the KV cache of a decoder in three stores per (layer, batch element,
 * KV head) "stream" (Appendix D, "Storage Layout"): bit-packed low-precision codes, the critical key
 * channels in BF16, and a full-precision residual window of the newest <= R tokens.  This library
 * implements the three data-parallel steps of one decode step on that cache:
 *
 *   mixkvq_select_channels   query-aware key-channel scoring and three-tier assignment (Section 4.2)
 *   mixkvq_quantize_append   append to the residual window and, every R tokens, quantize and pack
 *                            (Section 4.2 workflow, Eq. 2; Appendix D.1 lazy update, D.2 accumulator)
 *   mixkvq_decode_attention  softmax(q K~^T * scale) V~ over the mixed-precision cache (Eq. 1, Eq. 3)
 *
 * Conventions
 *   - Every pointer named *_dev is DEVICE memory, owned by the caller, 16-byte aligned.  The library
 *     allocates no device memory and frees none.  `mixkvq_cache*` is a small HOST object.
 *   - bf16 tensors are passed as `const void*` (raw 16-bit bfloat16, row-major, innermost dim = head_dim).
 *   - `stream` is a `cudaStream_t` passed as `void*` (NULL = default stream).  All work is enqueued on
 *     it; only mixkvq_query_status synchronizes.
 *   - Every function returns MIXKVQ_OK (0) or a negative MIXKVQ_E_* code.  Nothing aborts, traps or
 *     throws.  Conditions discovered on the device (extras arena full, a staged copy that never arrived)
 *     set a sticky device status word that mixkvq_query_status returns.
 *   - All sequences of the batch have the same length (the library tracks it per layer on the host).
 *   - head_dim must be 128.
 */
#ifndef MIXKVQ_H_
#define MIXKVQ_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

enum {
  MIXKVQ_OK = 0,
  MIXKVQ_E_INVALID_ARG = -1,          /* null pointer, bad dimension, layer out of range            */
  MIXKVQ_E_UNSUPPORTED = -2,          /* head_dim != 128, v_bits not 2 or 4, unsupported R, G or layout */
  MIXKVQ_E_ALIGNMENT = -3,            /* a device pointer is not 16-byte aligned                     */
  MIXKVQ_E_BUFFER_TOO_SMALL = -4,     /* cache memory or attention workspace smaller than required   */
  MIXKVQ_E_CAPACITY = -5,             /* append would exceed max_tokens                              */
  MIXKVQ_E_CUDA = -6,                 /* a CUDA runtime call or kernel launch reported an error: an
                                         append may then have advanced part of the way (the handle
                                         counts what was enqueued before the failing launch), so the
                                         layer's contents are undefined until mixkvq_cache_reset      */
  MIXKVQ_E_EMPTY = -7,                /* attention or selection requested on a layer with no tokens  */
  MIXKVQ_E_BUILTIN_SCRATCH = -8       /* mixkvq_decode_attention_noalloc: batch * n_kv_heads exceeds
                                         MIXKVQ_NOALLOC_MAX_STREAMS                                  */
};

/* bits of the sticky device status word */
enum {
  MIXKVQ_DEV_EXTRAS_FULL = 1,         /* a block's promoted channels did not fit the stream's extras arena.  The
                                         block's base part is written as usual, but nothing goes to the arena and the
                                         block's table entry records no promoted channel (n16 = n4 = 0): its BF16-tier
                                         channels then read as 0 and its UINT4 channels lose their high plane, so the
                                         layer's attention is wrong from that block on, until the cache is reset
                                         (with a larger extras_budget_bytes).  Earlier blocks are unaffected            */
  MIXKVQ_DEV_BAD_POSITION = 4,        /* a rotation with several axes, of part of the head or of a paged append met a position beyond the tables: that
                                         token's rows were left alone (and it was not appended) */
  MIXKVQ_DEV_BAD_LENGTH = 8,          /* paged cache: a length or a count of a call was negative or beyond the page table or the call's tokens: it
                                         was taken as the nearest that is possible, and a token that has no place was left out */
  MIXKVQ_DEV_BAD_PAGE = 16,           /* paged cache: a page that a call needed is none of the pool's: its tokens were left out */
  MIXKVQ_DEV_COPY_TIMEOUT = 2         /* a bounded wait (for a staged bulk copy, or for the partner warp of a pair) ran out:
                                         the warps concerned contributed nothing to that call's output, which is
                                         therefore wrong (0 where no warp contributed); later calls are unaffected    */
};

typedef struct mixkvq_config {
  int32_t n_layers;
  int32_t batch;                      /* B                                                           */
  int32_t n_q_heads;                  /* Hq, a multiple of n_kv_heads, Hq/Hkv <= 8                   */
  int32_t n_kv_heads;                 /* Hkv                                                         */
  int32_t head_dim;                   /* D, must be 128                                              */
  int32_t max_tokens;                 /* capacity per sequence                                       */
  int32_t residual_len;               /* R (Section 5.1: 128): multiple of 32, <= 256, multiple of G */
  int32_t group_size;                 /* G (Section 5.1: 32): 32, 64 or 128                          */
  int32_t v_bits;                     /* value bit-width: 2 (Section 4.2), or 4 (fragment layout only; stored as
                                         two 2-bit planes, the value scale must then stay below 2^7)  */
  int32_t score_bits;                 /* B of the sensitivity score S_d (Section 4.2), 2 or 4        */
  float tau_bf16;                     /* A_d >  tau_bf16            -> BF16                          */
  float tau_u4;                       /* tau_u4 < A_d <= tau_bf16   -> UINT4, else UINT2             */
  int32_t importance_mode;            /* 0: |q| accumulated within the current window (Section 4.2);
                                         1: cumulative over the whole history (Appendix D.2);
                                         2: error-only ablation (Appendix E): I_d = 1, A_d = S_d     */
  int32_t block_layout;               /* 0: fragment layout (any R; mma.sync attention kernel), the default;
                                         1: tile layout (R must be 128; tcgen05 attention kernel)        */
  uint64_t extras_budget_bytes;       /* per stream, for promoted channels; 0 = library default
                                         (1/8 of the bf16 size of max_tokens keys)                   */
  int32_t budget_bf16;                /* fixed-budget form of the tier rule of Section 4.2: when budget_bf16 +     */
  int32_t budget_u4;                  /* budget_u4 > 0 the thresholds are ignored; the budget_bf16 channels of highest
                                         salience A_d of a window go to BF16, the next budget_u4 to UINT4, the rest to
                                         UINT2 (equal saliences: lower channel first).  Every block then has the same
                                         tier counts.  Sum <= 128                                       */
  int32_t sink_len;                   /* sink tokens (the "sink length" of the settings in Appendix E): the first sink_len
                                         tokens of every sequence stay in bf16 for good, outside the residual window, the
                                         importance accumulator and the quantized blocks.  0, or a multiple of 32 <= 256 */
  int32_t reserved;                   /* must be 0                                                    */
} mixkvq_config;

typedef struct mixkvq_cache mixkvq_cache;

/* Byte offsets (from the start of the cache memory) and strides of one layer's arrays, for tools
 * and tests that inspect the cache.  The element formats are part of the library's documentation. */
typedef struct mixkvq_layout_desc {
  uint64_t state_off, state_stride;       /* per stream: acc fp64[128], cnt u32, extras_used16 u32   */
  uint64_t table_off, table_stride;       /* per stream: max_blocks entries of 8 bytes               */
  uint64_t resk_off, resk_stride;         /* per stream: [R][128] bf16                               */
  uint64_t resv_off, resv_stride;         /* per stream: [R][128] bf16                               */
  uint64_t base_off, base_stride;         /* per stream: max_blocks blocks of base_bytes             */
  uint64_t extras_off, extras_stride;     /* per stream: extras arena                                */
  uint64_t base_bytes;                    /* size of one block's fixed part                          */
  uint32_t max_blocks, n_streams;
  uint32_t n_blocks, residual_tokens;     /* current fill of sequence 0 (mixkvq_sequence_fill: any)  */
  uint64_t sink_off, sink_stride;         /* per stream: [sink_len][128] bf16 keys, then the same for values */
  uint32_t sink_tokens, sink_len;         /* sink rows filled so far, and their capacity              */
} mixkvq_layout_desc;

/* Sizes the caller must provide: the cache memory for all layers and the workspace of one
 * mixkvq_decode_attention call (split partials).  Host-only, no CUDA call. */
int mixkvq_cache_bytes(const mixkvq_config* cfg, size_t* cache_bytes, size_t* attn_workspace_bytes);

/* Creates the host handle over caller-owned device memory and enqueues the zeroing of the per-stream
 * state on `stream`.  cache_dev must hold at least the size reported by mixkvq_cache_bytes. */
int mixkvq_cache_init(const mixkvq_config* cfg, void* cache_dev, size_t bytes, void* stream, mixkvq_cache** out);

/* Frees the host handle only. */
int mixkvq_cache_destroy(mixkvq_cache* cache);

/* Empties one layer (layer >= 0) or all layers (layer < 0): lengths to zero, state re-zeroed on `stream`. */
int mixkvq_cache_reset(mixkvq_cache* cache, int layer, void* stream);

/* (1) Section 4.2: I_d (mean |q| over the window and the GQA group), S_d (key range over the window
 * divided by 2^score_bits - 1), A_d = I_d * S_d, and the tier of every key channel for the CURRENT
 * residual window of `layer`; a pure function of the cache state.
 *   tiers_dev    [B, Hkv, 128] uint8: 0 = UINT2, 1 = UINT4, 2 = BF16
 *   salience_dev [B, Hkv, 128] double A_d, or NULL */
int mixkvq_select_channels(mixkvq_cache* cache, int layer, uint8_t* tiers_dev, double* salience_dev, void* stream);

/* Stateless form of (1) on explicit windows: q_dev [B, Hq, Lq, 128] bf16, k_dev [B, Hkv, Lk, 128] bf16. */
int mixkvq_select_channels_raw(const void* q_dev, const void* k_dev, int batch, int n_q_heads, int n_kv_heads,
                               int lq, int lk, int score_bits, float tau_bf16, float tau_u4,
                               uint8_t* tiers_dev, double* salience_dev, void* stream);

/* (2) Appends n_tokens (1 = decode step, > 1 = prefill / bulk) post-RoPE tokens to `layer`, in token order:
 * for each token, if the residual window already holds R tokens it is first scored, quantized (keys per
 * channel at the tier's bit-width, values per token at 2 bits, groups of G, Eq. 2) and packed; then the
 * token is stored in the window and |q| is added to the importance accumulator.
 * Complete windows of a long append are quantized straight from the tensors (the prefill path); the result is byte for
 * byte that of n_tokens single appends.
 *   k_dev, v_dev [B, Hkv, n_tokens, 128] bf16;  q_dev [B, Hq, n_tokens, 128] bf16 */
int mixkvq_quantize_append(mixkvq_cache* cache, int layer, const void* k_dev, const void* v_dev, const void* q_dev,
                           int n_tokens, void* stream);

/* (3) Eq. 1 for one decode step of `layer` over [packed blocks, residual window], keys and values
 * dequantized on the fly (Eq. 3).
 *   q_dev [B, Hq, 128] bf16  ->  out_dev [B, Hq, 128] float
 *   workspace_dev: at least attn_workspace_bytes (mixkvq_cache_bytes); contents are scratch
 * Numeric range: the tensor-core operands are fp16, so |q| must stay below 4094, a stored key scale below 2^11 and a
 * stored value scale below 2^9 (value ranges up to about 1500); beyond that the output overflows to inf or NaN.
 * The kernels are launched with programmatic stream serialization and wait on the device for all earlier work of
 * the stream before they read q_dev or write anything, so stream order holds as for any other launch.  One access comes
 * before that wait: the first packed blocks of the layer are requested early unless the call this library enqueued last
 * on this handle wrote packed blocks of this layer (a flush; initialisation and reset count for all layers) or went to
 * another stream.  Cache
 * memory is written through this library only; a caller that writes it by other means (restoring saved cache bytes with
 * a kernel of its own, say) calls mixkvq_cache_written_externally before the next attention call.
 * No wait inside the kernels is unbounded: a staged copy or a hand-over between two warps that has not arrived after
 * 2^21 polls (each poll suspends the thread for up to about a microsecond: two seconds at most, milliseconds if the
 * polls return at once) sets MIXKVQ_DEV_COPY_TIMEOUT and the call returns. */
int mixkvq_decode_attention(mixkvq_cache* cache, int layer, const void* q_dev, float* out_dev, float softmax_scale,
                            void* workspace_dev, size_t workspace_bytes, void* stream);

/* (2) + (3) fused for one decode step of `layer`: appends the step's token (k_dev, v_dev [B, Hkv, 1, 128],
 * q_dev [B, Hq, 1, 128] bf16, flushing the residual window first if it is full) and attends with the same q_dev.
 * The cache state and out_dev are exactly those of mixkvq_quantize_append(n_tokens = 1) followed by
 * mixkvq_decode_attention; the attention kernel stores the token and updates the importance accumulator itself
 * (Appendix D.1, D.2), which saves a kernel launch per layer. */
int mixkvq_decode_step(mixkvq_cache* cache, int layer, const void* k_dev, const void* v_dev, const void* q_dev,
                       float* out_dev, float softmax_scale, void* workspace_dev, size_t workspace_bytes, void* stream);

/* (2) for a batch whose sequences differ in length (the serving setting of the efficiency experiment: requests of
 * unequal length share a batch).  Sequence b takes the first n_tokens_host[b] tokens (0 <= n_tokens_host[b] <=
 * n_tokens_max; 0 = the sequence takes no token in this call) of its rows of the tensors:
 *   k_dev, v_dev [B, Hkv, n_tokens_max, 128], q_dev [B, Hq, n_tokens_max, 128] bf16; n_tokens_host: HOST array [B].
 * Every sequence keeps its own number of packed blocks, residual tokens and sink rows; each is flushed when ITS window
 * is full, exactly as if it were alone in the batch (the bytes of its streams equal those of a batch-1 cache fed the
 * same tokens).  Neighbouring sequences with the same fill and the same count go through the kernels together, so a
 * batch of equal lengths costs what mixkvq_quantize_append costs (which is this call with equal counts).
 * The capacity check covers every sequence before anything is enqueued.
 * After sequences have diverged, mixkvq_decode_attention, mixkvq_decode_step and mixkvq_select_channels work per
 * sequence: the attention kernel reads every sequence's fill from a table in device memory (written on the stream as
 * kernel arguments, no copy) and splits the positions of all streams evenly over its CTAs; a sequence without tokens
 * gets an all-zero output.  Restrictions of a diverged batch: fragment layout, the default or the split-only
 * attention kernel, B <= 128 (MIXKVQ_E_UNSUPPORTED otherwise). */
int mixkvq_quantize_append_ragged(mixkvq_cache* cache, int layer, const void* k_dev, const void* v_dev, const void* q_dev,
                                  int n_tokens_max, const int32_t* n_tokens_host, void* stream);

/* Fill of sequence b of a layer (any pointer may be NULL). */
int mixkvq_sequence_fill(const mixkvq_cache* cache, int layer, int b, uint32_t* n_blocks, uint32_t* residual_tokens,
                         uint32_t* sink_tokens);

/* Decode attention for a context whose tokens are spread over several caches (one per GPU: a sequence split for
 * contexts beyond one GPU's memory).  Eq. 1 over this cache's tokens alone, in the form the merge needs:
 *   out_dev [B, Hq, 128] float: softmax-weighted values over this cache's tokens (normalised by this cache's own
 *   denominator);  lse_dev [B, Hq] float: natural logarithm of that denominator sum_j exp(scale q.k_j).
 * A sequence (or a whole cache) without tokens gives zeros and lse = -inf.  Same kernels, workspace and queue
 * behaviour as mixkvq_decode_attention; fragment layout and the default kernel only (MIXKVQ_E_UNSUPPORTED otherwise). */
int mixkvq_decode_attention_partial(mixkvq_cache* cache, int layer, const void* q_dev, float* out_dev, float* lse_dev,
                                    float softmax_scale, void* workspace_dev, size_t workspace_bytes, void* stream);

/* Eq. 1 over the union of disjoint token sets from the per-set results of mixkvq_decode_attention_partial (the
 * log-sum-exp identity): out = sum_r w_r o_r / sum_r w_r, w_r = exp(lse_r - max_r lse_r).  Stateless.
 *   o_parts_dev [n_parts, rows, 128] float, lse_parts_dev [n_parts, rows] float (rows = B * Hq; the layout an
 *   all-gather of the ranks' results produces)  ->  out_dev [rows, 128] float.  Parts with lse = -inf weigh 0;
 *   rows whose parts are all empty come out as zeros.  1 <= n_parts <= 1024. */
int mixkvq_merge_partials(const float* o_parts_dev, const float* lse_parts_dev, int n_parts, int rows, float* out_dev,
                          void* stream);

/* The prefill phase of Section 4.2 for one layer: causal attention of the prompt over itself in full precision (Eq. 1,
 * position i sees positions 0..i), then the prompt's keys and values go into the cache exactly as
 * mixkvq_quantize_append(n_tokens) would put them (complete windows quantized, the last 1..R tokens in the residual
 * window).  The layer must be empty (MIXKVQ_E_UNSUPPORTED otherwise: a later chunk attends to a
 * dequantized cache, which is mixkvq_chunk_step).
 *   k_dev, v_dev [B, Hkv, n_tokens, 128], q_dev [B, Hq, n_tokens, 128] bf16 (post-RoPE)  ->  out_dev [B, Hq, n_tokens, 128] float
 *   scratch_dev: device memory of at least mixkvq_prefill_scratch_bytes(cfg, n_tokens) bytes, 16-byte aligned, owned by
 *   the caller and free for reuse once the work enqueued by this call has run (it holds K and V of the prompt
 *   rearranged into the tensor core's tile layout); too small -> MIXKVQ_E_CAPACITY.
 * The attention runs on the tcgen05 tensor cores (bf16 products for the logits, fp16 probabilities and values for the
 * output, fp32 accumulation in tensor memory); values must stay inside the fp16 range.  softmax_scale > 0.  A barrier
 * wait that runs out sets MIXKVQ_DEV_COPY_TIMEOUT in the status word and leaves the affected output rows unwritten.
 * Nothing is allocated and nothing synchronises with the host. */
size_t mixkvq_prefill_scratch_bytes(const mixkvq_config* cfg, int n_tokens);
int mixkvq_prefill(mixkvq_cache* cache, int layer, const void* k_dev, const void* v_dev, const void* q_dev, int n_tokens,
                   float* out_dev, float softmax_scale, void* scratch_dev, size_t scratch_bytes, void* stream);

/* Attention of a chunk of new tokens over a layer that may hold tokens already: the later chunks of a prompt, or drafted tokens whose
 * acceptance is decided afterwards.  Sequence b has n_tokens_host[b] new tokens (0 <= n_tokens_host[b] <= n_tokens_max; HOST array [B], or
 * NULL: n_tokens_max each), the first rows of
 *   k_dev, v_dev [B, Hkv, n_tokens_max, 128], q_dev [B, Hq, n_tokens_max, 128] bf16 (post-RoPE)  ->  out_dev [B, Hq, n_tokens_max, 128]
 * New token j attends to everything the sequence holds (sink, packed blocks dequantized by Eq. 3, residual window) and to the new tokens
 * 0 .. j in full precision.  out_type: MIXKVQ_OUT_FLOAT or MIXKVQ_OUT_BF16 (rounded once, to nearest).  Rows behind a sequence's count are neither
 * read nor written.  The sequences may hold different numbers of tokens.  An empty layer gives the causal attention of mixkvq_prefill (that
 * multiplies queries and keys in bf16 and so takes any magnitude; here they are fp16, see below).
 * mixkvq_chunk_attention appends nothing: accepted tokens go in with mixkvq_quantize_append_ragged, which takes the same tensors.
 * mixkvq_chunk_step is mixkvq_chunk_attention, then the chunk is appended as mixkvq_quantize_append_ragged does it; on
 * MIXKVQ_E_CAPACITY nothing was enqueued.
 *   scratch_dev: at least mixkvq_chunk_scratch_bytes(cfg, n_tokens_max) bytes, contents are scratch, free for reuse once the call's work has
 *   run (two calls that may overlap on the GPU need one each, two captured graphs too unless they never run at the same time).
 * The fills and the counts are parameters of the launches: a captured call is replayed with those of its capture.
 * Numeric range: products are fp16 with fp32 accumulation, so |q|, |k|, |v| and dequantized elements must stay below 65504.  A dequantized element is
 * rounded once, by 2^-11 of itself; below 2^-14 elements round to fp16 subnormals (2^-25), and those of a group whose scale is below 2^-15 by up to 2^-20
 * (2-bit codes) or 2^-18 (4-bit).  A key's weight is rounded by up to 2^-11 of itself (below 2^-10 of the row's largest one up to twice
 * that) or 2^-30 of the largest, in the sum and in its denominator alike.  A NaN or an infinity among the new tokens reaches the rows that attend to
 * it and no others.
 * The tensor core's sums are truncated, not rounded: about 3.5e-7 of the output per 128 tokens held, in one direction, up to 1.8e-4; what a key adds
 * below 2^-24 of the sum is lost.  65536 tokens are summed so at most; the sums of more are joined in fp32.
 * softmax_scale > 0; out_dev and scratch_dev overlap no other argument nor the cache's memory (MIXKVQ_E_INVALID_ARG); fragment layout, n_tokens_max <=
 * MIXKVQ_CHUNK_MAX_TOKENS (MIXKVQ_E_UNSUPPORTED otherwise); scratch too small: MIXKVQ_E_BUFFER_TOO_SMALL.  A wait that runs out sets
 * MIXKVQ_DEV_COPY_TIMEOUT; the rows concerned are then wrong.  Nothing is allocated and nothing synchronises with the host. */
enum { MIXKVQ_OUT_FLOAT = 0, MIXKVQ_OUT_BF16 = 1 };
#define MIXKVQ_CHUNK_MAX_TOKENS (1 << 24)
size_t mixkvq_chunk_scratch_bytes(const mixkvq_config* cfg, int n_tokens_max);
int mixkvq_chunk_attention(mixkvq_cache* cache, int layer, const void* k_dev, const void* v_dev, const void* q_dev, int n_tokens_max,
                           const int32_t* n_tokens_host, void* out_dev, int out_type, float softmax_scale, void* scratch_dev,
                           size_t scratch_bytes, void* stream);
int mixkvq_chunk_step(mixkvq_cache* cache, int layer, const void* k_dev, const void* v_dev, const void* q_dev, int n_tokens_max,
                      const int32_t* n_tokens_host, void* out_dev, int out_type, float softmax_scale, void* scratch_dev,
                      size_t scratch_bytes, void* stream);

/* Appendix D ("saliency evaluation is performed post-transformation"): for models with rotary position embeddings the
 * scores, the stored keys and the attention all use rotated queries and keys.  These two calls rotate before they
 * append.  k_dev [B, Hkv, n_tokens, 128] and q_dev [B, Hq, n_tokens, 128] (bf16) are rotated IN PLACE: afterwards q_dev
 * holds the rotated queries that mixkvq_decode_attention takes, k_dev the keys that were stored.  v_dev is not touched.
 *   cos_dev, sin_dev: float tables [n_positions, 64] of the caller's angles (row p = position p, entry i the angle of
 *   channel pair (i, i + 64): the "rotate-half" pairing); token j of the call uses row pos0 + j.  The caller owns them.
 *   Arithmetic: y[i] = x[i] c - x[i+64] s, y[i+64] = x[i+64] c + x[i] s, every product and the sum one fp32 operation
 *   rounded to nearest, the result rounded to bf16 (ties to even).  The cache then equals, byte for byte, that of
 *   mixkvq_quantize_append on tensors rotated in this way.
 * Errors as for mixkvq_quantize_append / mixkvq_decode_step; on MIXKVQ_E_CAPACITY nothing was rotated. */
int mixkvq_rope_append(mixkvq_cache* cache, int layer, void* k_dev, const void* v_dev, void* q_dev, const float* cos_dev,
                       const float* sin_dev, int pos0, int n_tokens, void* stream);
/* The same for one decode step: rotates the step's k_dev [B, Hkv, 1, 128] and q_dev [B, Hq, 1, 128] with table row `pos`,
 * then does what mixkvq_decode_step does. */
int mixkvq_rope_decode_step(mixkvq_cache* cache, int layer, void* k_dev, const void* v_dev, void* q_dev,
                            const float* cos_dev, const float* sin_dev, int pos, float* out_dev, float softmax_scale,
                            void* workspace_dev, size_t workspace_bytes, void* stream);

/* The rotation for tokens with several coordinates (time, height, width of an image patch or a video frame; up to MIXKVQ_ROPE_MAX_AXES axes, and a
 * position of its own for every sequence): channel pair (i, i + 64) of token j of sequence b turns by row positions_dev[axis_of_pair_host[i]][b][j] of the
 * tables.  Arithmetic, pairing and tables as for mixkvq_rope_append; n_positions is the tables' number of rows.
 *   positions_dev [n_axes, B, n_tokens] int32, DEVICE.  A token with a negative coordinate on an axis that some pair uses is none (padding of
 *   a ragged batch): its rows of the outputs are left as they are.  So are those of a token with a coordinate of n_positions or more, and that sets
 *   MIXKVQ_DEV_BAD_POSITION.
 *   axis_of_pair_host [64]: HOST array, every entry below n_axes.
 * mixkvq_rope_axes is stateless but for the status word: from q_dev, k_dev (and v_dev, which is copied; NULL with v_out_dev NULL: left out) in any
 * layout whose last dimension is contiguous, the fused projection's [B, n, Hq + 2 Hkv, 128] included, to head-major
 * q_out_dev [B, Hq, n, 128], k_out_dev, v_out_dev [B, Hkv, n, 128]: what the append, prefill and chunk calls take.
 *   strides_host [9]: HOST array, the distances in elements from one batch element, head and token to the next, for q, k, v in turn (0 or more,
 *   multiples of 8); NULL: head-major.  An output may be its own input where that is head-major; no output may overlap anything else,
 *   the tables, the positions and the cache's memory included (MIXKVQ_E_INVALID_ARG).
 * mixkvq_rope_axes_append and mixkvq_rope_axes_decode_step rotate k_dev and q_dev in place and then do what mixkvq_quantize_append and
 * mixkvq_decode_step do (one more launch than mixkvq_rope_decode_step); v_dev overlaps neither (MIXKVQ_E_INVALID_ARG); on MIXKVQ_E_CAPACITY and
 * MIXKVQ_E_UNSUPPORTED nothing was rotated or appended.  They append every row of the call, those that the rotation leaves alone (a negative
 * coordinate, one beyond the tables) as they came: a ragged batch takes mixkvq_rope_axes, then mixkvq_quantize_append_ragged with its counts. */
#define MIXKVQ_ROPE_MAX_AXES 4
int mixkvq_rope_axes(mixkvq_cache* cache, const void* q_dev, const void* k_dev, const void* v_dev, const int64_t* strides_host, int n_tokens,
                     const float* cos_dev, const float* sin_dev, int n_positions, const int32_t* positions_dev, int n_axes,
                     const uint8_t* axis_of_pair_host, void* q_out_dev, void* k_out_dev, void* v_out_dev, void* stream);
int mixkvq_rope_axes_append(mixkvq_cache* cache, int layer, void* k_dev, const void* v_dev, void* q_dev, const float* cos_dev, const float* sin_dev,
                            int n_positions, const int32_t* positions_dev, int n_axes, const uint8_t* axis_of_pair_host, int n_tokens, void* stream);
int mixkvq_rope_axes_decode_step(mixkvq_cache* cache, int layer, void* k_dev, const void* v_dev, void* q_dev, const float* cos_dev, const float* sin_dev,
                                 int n_positions, const int32_t* positions_dev, int n_axes, const uint8_t* axis_of_pair_host, float* out_dev,
                                 float softmax_scale, void* workspace_dev, size_t workspace_bytes, void* stream);

/* Rotary positions of part of the head.  Channels 0 .. rotary_dim - 1 of a row turn, the others stay: pairs (i, i + rotary_dim / 2), or (2 i, 2 i + 1) where
 * `interleaved` is 1.  Tables as mixkvq_rope_tables makes them: float [n_positions, rotary_dim / 2], 16-byte aligned.  Arithmetic as for mixkvq_rope_append:
 * y0 = x0 c - x1 s, y1 = x1 c + x0 s, every product and the sum one fp32 operation rounded to nearest, the result rounded to bf16. */
typedef struct mixkvq_rotation {
  const float *cos_dev, *sin_dev;
  const int32_t* positions_dev;       /* [B, n] int32, DEVICE: the table row of every token */
  int32_t n_positions;                /* rows of the tables */
  int32_t rotary_dim;                 /* a multiple of 16 up to 128 */
  int32_t interleaved;
  int32_t reserved;
} mixkvq_rotation;
/* Rotates q_dev, k_dev (and copies v_dev; NULL with v_out_dev NULL: left out) from any layout whose last dimension is contiguous into the head-major
 * q_out_dev [B, Hq, n, 128], k_out_dev, v_out_dev [B, Hkv, n, 128] that the append, prefill and chunk calls take.  Strides, overlaps, tokens with a negative
 * position (none: their rows of the outputs are left alone) and with one beyond the tables (MIXKVQ_DEV_BAD_POSITION) as for mixkvq_rope_axes. */
int mixkvq_rope_partial(mixkvq_cache* cache, const void* q_dev, const void* k_dev, const void* v_dev, const int64_t* strides_host, int n_tokens,
                        const mixkvq_rotation* rotation, void* q_out_dev, void* k_out_dev, void* v_out_dev, void* stream);

/* The tables of a rotation: entry [p - start][i] is m cos(p f_i) and m sin(p f_i) for p = start .. start + n_positions - 1, f_i the frequency of channel pair i,
 * d = rotary_dim, computed in 64 bits and rounded to float once.  Frequencies base^(-2 i / d), and for contexts beyond the one trained on:
 *   PLAIN   as they are
 *   LINEAR  divided by factor
 *   NTK     base * factor^(d / (d - 2)) for base: the lowest is divided by factor, the highest stays
 *   BANDS   those with at least `high` turns in `original` positions stay, those with at most `low` are divided by factor, between them a linear mix
 *   YARN    the same with the mix linear in i, between the pairs (rounded outwards) that turn `high` and `low` times in `original` positions; m = 0.1 ln factor + 1
 * attention_factor: m; 0: the kind's own (1 but for YARN with a factor above 1).  Stateless, enqueued on the current device. */
enum { MIXKVQ_ROPE_PLAIN = 0, MIXKVQ_ROPE_LINEAR = 1, MIXKVQ_ROPE_NTK = 2, MIXKVQ_ROPE_BANDS = 3, MIXKVQ_ROPE_YARN = 4 };
typedef struct mixkvq_rope_scaling {
  int32_t kind, rotary_dim;           /* rotary_dim: a multiple of 16 up to 128 */
  double base, factor, original, low, high, attention_factor;
  int32_t reserved;                   /* must be 0 */
} mixkvq_rope_scaling;
int mixkvq_rope_tables(const mixkvq_rope_scaling* scaling, int64_t start, int n_positions, float* cos_dev, float* sin_dev, void* stream);

/* ---- A cache held in 4 bits, in pages (no counterpart in the paper): for servers that give sequences memory page by page, share
 * pages between them and capture their steps into graphs.  Keys and values are both quantized token by token when they come (Eq. 2 with 16 levels,
 * groups of G channels of one token, scale and zero-point bf16 as everywhere: reading of the stored scale included), so there is no window, no flush and no
 * state but the pages.  (The paper quantizes keys per channel, as do the methods it compares with: an outlier channel then costs the others nothing.  Here it widens the
 * step of its group of G channels.)  Which pages belong to a sequence and how many tokens it has is the caller's, in DEVICE memory: nothing about a call but its shape is
 * known to the host.
 *
 * Pool: `n_layers` times `n_pages` pages of page_tokens tokens of all KV heads, behind a header of 256 bytes with the status word; page p of a layer is one contiguous piece
 * of Hkv * page_tokens * (128 + 1024 / G) bytes.  A page has the same number in all layers. */
typedef struct mixkvq_paged_config {
  int32_t n_layers, n_q_heads, n_kv_heads;   /* Hq a multiple of Hkv, Hq / Hkv <= 8 */
  int32_t head_dim;                   /* must be 128 */
  int32_t n_pages;                    /* per layer */
  int32_t page_tokens;                /* 16, 32, 64, 128 or 256 */
  int32_t group_size;                 /* G: 32, 64 or 128 */
  int32_t reserved;                   /* must be 0 */
} mixkvq_paged_config;
typedef struct mixkvq_paged mixkvq_paged;

/* The sequences of a call.  Token t of sequence b lies on page pages_dev[b * pages_stride + t / page_tokens], slot t % page_tokens.  Pages beyond those that a call's tokens need
 * are not looked at.  Lengths and counts that are impossible set MIXKVQ_DEV_BAD_LENGTH, pages that are none MIXKVQ_DEV_BAD_PAGE (see there). */
typedef struct mixkvq_paged_sequences {
  int32_t batch;                      /* B */
  int32_t n_tokens;                   /* n: tokens of the call per sequence, at most */
  const int32_t* pages_dev;           /* [B, max_pages] int32, rows pages_stride apart */
  int32_t max_pages, pages_stride;    /* max_pages * page_tokens <= MIXKVQ_PAGED_MAX_TOKENS */
  const int32_t* lens_dev;            /* [B] int32: tokens of each sequence (what each call says) */
  const int32_t* counts_dev;          /* [B] int32 or NULL (n each): tokens of the call in each sequence, its first rows of the tensors */
} mixkvq_paged_sequences;
#define MIXKVQ_PAGED_MAX_TOKENS (1 << 28)
#define MIXKVQ_PAGED_MAX_BATCH 4096

int mixkvq_paged_bytes(const mixkvq_paged_config* cfg, size_t* pool_bytes);
/* Workspace of an attention call of this batch, number of tokens and columns of the page table, and of every call of a smaller batch, number and table: it never falls as they
 * grow, so that one workspace serves all calls up to the largest.  Contents are scratch and need not be anything; two calls that may overlap on the GPU
 * need one each, two captured graphs too unless they never run at the same time. */
size_t mixkvq_paged_workspace_bytes(const mixkvq_paged_config* cfg, int batch, int n_tokens, int max_pages);
/* The handle over caller-owned memory (256-byte aligned); the pages are left as they are, the status word is cleared on `stream`. */
int mixkvq_paged_init(const mixkvq_paged_config* cfg, void* pool_dev, size_t bytes, void* stream, mixkvq_paged** out);
int mixkvq_paged_destroy(mixkvq_paged* cache);

/* Stores tokens: token i < counts[b] of sequence b becomes token lens[b] + i of the sequence (lens: tokens before the call).
 *   k_dev, v_dev [B, Hkv, n, 128], q_dev [B, Hq, n, 128] bf16 with strides_host [9] (q, k, v: batch, head, token; NULL: head-major) as for mixkvq_rope_axes.
 *   rotation: NULL (keys are stored as they are), or keys and queries turn on the way; its positions_dev may be NULL: a token turns by its place in
 *   its sequence.  A token with a negative position is none: its slot stays as it was (and a step reckons with lens + counts all the same).
 *   q_dev, q_out_dev: both NULL, or the queries and where they go, rotated, head-major; q_out_dev may be q_dev itself where that is head-major.
 * A NaN is held as the least value of its group, whose other channels are as they are without it (no quantizer of this library has a code for one); a group of nothing else
 * reads back as NaN, and one with an infinity is finite in no channel.
 * Rows of q_out_dev behind a sequence's count are left as they are.  Two tokens of a call in the same slot (a page used twice) leave
 * a mix of both. */
int mixkvq_paged_append(mixkvq_paged* cache, int layer, const mixkvq_paged_sequences* seqs, const void* k_dev, const void* v_dev, const void* q_dev,
                        const int64_t* strides_host, const mixkvq_rotation* rotation, void* q_out_dev, void* stream);
/* The values that tokens lens[b] .. lens[b] + counts[b] - 1 of every sequence are held as (Eq. 3, rounded to bf16): k_out_dev, v_out_dev [B, Hkv, n, 128] bf16.  Other rows
 * are left as they are. */
int mixkvq_paged_read(mixkvq_paged* cache, int layer, const mixkvq_paged_sequences* seqs, void* k_out_dev, void* v_out_dev, void* stream);
/* Eq. 1 over the pages: the newest counts[b] tokens of sequence b, which has lens[b] tokens, these included; query row i sees tokens 0 .. lens[b] - counts[b] + i.
 *   q_dev [B, Hq, n, 128] bf16 (rotated), out_dev [B, Hq, n, 128] of out_type (MIXKVQ_OUT_*), rounded once.
 * A row that sees no token is zeros; rows behind a sequence's count are left as they are.  Nothing is read of tokens that no row sees: freed pages and the rest of a last
 * page may hold anything.  softmax_scale > 0 and finite.
 * Logits and sums are fp32; weights are fp16 numbers (2^-11), and calls that unpack the pages (MIXKVQ_PAGED_UNPACKED) round keys and values to fp16 once more.  Which calls do follows
 * from batch, heads, n_tokens and max_pages, not from the lengths (mixkvq_paged_last_attention).  Queries, keys and values are scaled by powers of two on the way, so that those
 * bits are kept at any magnitude, within two limits: what a token adds is held no finer than 2^-28 of the row's largest weight times the largest value of the sequence and KV head,
 * and values below 2^-110 lose bits.  What is not finite in the pages or a query reaches the rows that see it only. */
int mixkvq_paged_attention(mixkvq_paged* cache, int layer, const mixkvq_paged_sequences* seqs, const void* q_dev, void* out_dev, int out_type, float softmax_scale,
                           void* workspace_dev, size_t workspace_bytes, void* stream);
/* mixkvq_paged_append, then mixkvq_paged_attention of the tokens appended: a decode step, or a chunk of a prompt.  lens: tokens before the call.
 * q_out_dev is written (as the append does) and may be q_dev; out_dev and the workspace lie over none of the inputs. */
int mixkvq_paged_step(mixkvq_paged* cache, int layer, const mixkvq_paged_sequences* seqs, const void* k_dev, const void* v_dev, const void* q_dev,
                      const int64_t* strides_host, const mixkvq_rotation* rotation, void* q_out_dev, void* out_dev, int out_type, float softmax_scale,
                      void* workspace_dev, size_t workspace_bytes, void* stream);
/* As their counterparts of mixkvq_cache; the status word stays until it is cleared. */
int mixkvq_paged_test_arm_copy_timeout(mixkvq_paged* cache, uint32_t extra_bytes, uint32_t max_polls);
int mixkvq_paged_query_status(mixkvq_paged* cache, int* device_status, void* stream);
int mixkvq_paged_clear_status(mixkvq_paged* cache, void* stream);
uint64_t mixkvq_paged_launch_count(const mixkvq_paged* cache);
/* Which kernel the last attention on this handle enqueued (diagnostic), 0 before the first. */
enum {
  MIXKVQ_PAGED_DIRECT = 1,            /* a thread block per KV head and block of query rows, which wrote the output */
  MIXKVQ_PAGED_PIECES = 2,            /* pieces of streams, joined by a second kernel                */
  MIXKVQ_PAGED_UNPACKED = 4           /* the pages unpacked once into fp16 tiles, tcgen05            */
};
int mixkvq_paged_last_attention(const mixkvq_paged* cache);

/* (The paper has no counterpart of this entry point; it exists for integration reasons only.)
 * Same computation and same results as mixkvq_decode_attention, for callers that have no way to hand
 * over a workspace: code that runs inside a serving engine's pre-sized memory pool, a plugin that may
 * not call cudaMalloc (or any allocating library routine) once the engine has started, or a host
 * program written in a language binding that exposes no device allocator.  The split partials go to a
 * scratch array that is compiled into the library (static device storage of
 * (1184 + 2 * MIXKVQ_NOALLOC_MAX_STREAMS) * 4160 bytes, about 6.7 MiB, which every GPU that loads the
 * library holds until the process exits).  The call allocates and frees nothing.
 *   - batch * n_kv_heads of the cache must be <= MIXKVQ_NOALLOC_MAX_STREAMS, else
 *     MIXKVQ_E_BUILTIN_SCRATCH is returned and nothing is launched.
 *   - The first call on each device looks up the device address of the scratch array (with that device
 *     current, which must be the device that owns the cache memory: MIXKVQ_E_INVALID_ARG otherwise).  Make
 *     that first call before any stream capture begins, and from one thread: the look-up is not guarded
 *     against concurrent first calls.  The address is kept for the life of the process; it does not
 *     survive a cudaDeviceReset.
 *   - All calls on a device share the one array.  Nothing in it has to start at zero (every partial a
 *     call reads was written by that same call), so stale contents of earlier calls are harmless; but
 *     two calls whose kernels overlap on the GPU (different streams, no ordering between them) race on
 *     it and both results are undefined.  Calls on one stream are ordered and safe. */
#define MIXKVQ_NOALLOC_MAX_STREAMS 256
int mixkvq_decode_attention_noalloc(mixkvq_cache* cache, int layer, const void* q_dev, float* out_dev,
                                    float softmax_scale, void* stream);

/* Tells the library that cache memory was written by other means than its own calls since the last call on this
 * handle: the next decode attention of every layer then waits for all earlier work of the stream before its first read. */
int mixkvq_cache_written_externally(mixkvq_cache* cache);

/* Test hook for the give-up paths of the decode-attention kernel (fragment layout), the prefill and the chunk attention.  While
 * extra_bytes > 0 (a multiple of 16), the barrier of the first staged copy of every warp pair (decode) or of every
 * CTA's first key tile (prefill) is armed for extra_bytes more than the copy delivers, so it never completes, and every
 * wait gives up after max_polls polls (0: the default): the call returns, the device status word carries
 * MIXKVQ_DEV_COPY_TIMEOUT, the decode output rows are zero and the prefill output is left unwritten.  In the chunk attention
 * the CTAs leave out the announcement of their first key tile instead; its output is then undefined.  Nothing faults or
 * hangs: the copies themselves are the normal ones.  (0, 0) restores normal operation. */
int mixkvq_test_arm_copy_timeout(mixkvq_cache* cache, uint32_t extra_bytes, uint32_t max_polls);

/* The same in the prefill attention for the barrier of a CTA's last value tile where that tile's number is odd or it is the
 * prompt's last: the rows whose last product is missing are left unwritten, the others are as usual. */
int mixkvq_test_arm_value_copy_timeout(mixkvq_cache* cache, uint32_t extra_bytes, uint32_t max_polls);

/* Selects the decode-attention kernel: 0 = tensor-core kernel (default), 1 = plain-ALU kernel
 * (kept for comparison; same results within tolerance, much slower), 2 = the tensor-core split kernel
 * alone: the split partials stay in the workspace and out_dev is NOT written (for timing that kernel). */
int mixkvq_set_attention_kernel(mixkvq_cache* cache, int kind);

/* Synchronizes `stream`, then returns the sticky device status word (MIXKVQ_DEV_* bits). */
int mixkvq_query_status(mixkvq_cache* cache, int* device_status, void* stream);

/* Where one layer's arrays live inside the cache memory, and how full the layer is. */
int mixkvq_cache_describe(const mixkvq_cache* cache, int layer, mixkvq_layout_desc* out);

/* Which kernel the last decode-attention call on this handle enqueued (diagnostic): the sum of these, 0 before the first. */
enum {
  MIXKVQ_ATTN_ONE_UNIT = 1,           /* the tensor-core split kernel, one 32-token unit per step    */
  MIXKVQ_ATTN_TWO_UNITS = 2,          /* ... two units per step                                      */
  MIXKVQ_ATTN_DIRECT = 4,             /* one thread block per stream, which wrote the output: no merge */
  MIXKVQ_ATTN_EARLY = 8,              /* packed blocks were requested before the wait for earlier work */
  MIXKVQ_ATTN_OTHER = 16,             /* the plain-ALU kernel or the tile layout's                   */
  MIXKVQ_ATTN_EIGHT_PAIRS = 32        /* ONE_UNIT | DIRECT with eight instead of four pairs of warps per thread block */
};
int mixkvq_last_attention(const mixkvq_cache* cache);
/* Thread blocks of that call's split kernel (0: none, or MIXKVQ_ATTN_OTHER).  With fewer streams than thread blocks a number that
 * is no multiple of batch * n_kv_heads means that thread blocks straddle two streams. */
int mixkvq_last_attention_ctas(const mixkvq_cache* cache);

/* Number of kernels launched by this handle since it was created (diagnostic). */
uint64_t mixkvq_launch_count(const mixkvq_cache* cache);

const char* mixkvq_status_string(int status);

#ifdef __cplusplus
}
#endif
#endif /* MIXKVQ_H_ */
