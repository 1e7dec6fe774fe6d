/*
 * kl — one decode step of a Llama-style decoder-only transformer on one
 * AMD MI355X (gfx950), with kernel looping (arXiv 2410.23668).
 *
 * The paper's token step is Embedding -> L x Decoder -> Classifier (Sec. 2).
 * Each decoder layer is RMSNorm, the Q/K/V projections, RoPE, GQA attention
 * over the KV cache, the O projection with a residual add, RMSNorm, a SwiGLU
 * MLP and a second residual add.  The step runs in one of three schedules:
 *
 *   KL_MODE_PER_LAYER  one kernel launch per decoder layer (the layer-level
 *                      fusion baseline of Sec. 2, K0 called L times), plus one
 *                      launch for the embedding and one for the classifier:
 *                      L + 2 dispatches.
 *   KL_MODE_LOOPED     kernel looping (Sec. 2 and Sec. 3.2): the L chained
 *                      layer calls become one call of a kernel with an outer
 *                      loop over layers; the embedding and classifier run in
 *                      the same launch: 1 dispatch.  Kernel boundaries are
 *                      replaced by device-scope counters.
 *   KL_MODE_PER_OP     one launch per operator group of a layer (the many-
 *                      kernels-per-layer GPU schedule of Sec. 2, Fig. 3 (i)):
 *                      5 L + 2 dispatches.
 *   KL_MODE_PER_LAYER_GRAPH
 *                      the per-layer schedule's L + 2 launches recorded once as
 *                      a HIP graph and replayed (the graph alternative of the
 *                      related work, Sec. 5): rebuilt when the caller's
 *                      buffers (tokens, positions, batch, cache, outputs,
 *                      trace) differ from the last call's; one graph per
 *                      state.  Not available to kl_decode_step_noalloc or
 *                      kl_decode_greedy.
 *
 * All modes run the same device code with the same work partition, so for the
 * same inputs they produce bit-identical logits, hidden states and KV writes.
 *
 * Conventions.  All tensors are row-major.  "dev" pointers are device memory
 * of the current HIP device; "host" pointers are host memory.  bf16 values are
 * passed as their 16-bit patterns.  Streams are hipStream_t passed as void*
 * (NULL = the default stream).  Functions returning kl_status return KL_OK or
 * a negative code; on a negative code nothing was enqueued and kl_last_error()
 * describes the problem.  The library is built for gfx950 only.
 */
#ifndef KL_H
#define KL_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    KL_OK = 0,
    KL_ERR_INVALID_ARGUMENT = -1,  /* null / misaligned pointer, bad size, bad mode  */
    KL_ERR_UNSUPPORTED = -2,       /* a shape this build does not implement           */
    KL_ERR_OUT_OF_MEMORY = -3,     /* device allocation failed                        */
    KL_ERR_HIP = -4,               /* a HIP runtime call failed (message has details) */
    KL_ERR_DEVICE_FAULT = -5       /* reported by kl_get_device_error                 */
} kl_status;

typedef enum {
    KL_MODE_PER_LAYER = 0,
    KL_MODE_LOOPED = 1,
    KL_MODE_PER_OP = 2,
    KL_MODE_PER_LAYER_GRAPH = 3
} kl_mode;

/* Bits of the device error word (kl_get_device_error).  A sequence with a bad
 * token or position is skipped: none of its K/V slots is written and its
 * logits (and hidden state) are NaN; the other sequences of the step are
 * computed normally. */
#define KL_DEVERR_TOKEN    1   /* a token id outside [0, vocab)                              */
#define KL_DEVERR_POSITION 2   /* a position outside [0, capacity) or >= max_seq             */
#define KL_DEVERR_BARRIER  4   /* a grid barrier waited longer than its watchdog allows      */
#define KL_DEVERR_PAGE     8   /* a page table entry outside [0, n_pages)                    */

/* Model shape.  Supported: head_dim 64 or 128, n_heads a multiple of
 * n_kv_heads with n_heads / n_kv_heads one of 1, 2, 4, 8 (and 3 with
 * head_dim 128), n_heads at most the GPU's compute units, every dimension
 * >= 1 and hidden, ffn_dim multiples of 8.  max_batch bounds the batch of a
 * step; max_seq bounds positions (the RoPE table covers [0, max_seq)).
 * qkv_bias: 1 if the Q/K/V projections carry biases (the Qwen2.5 variant of
 * Table 2), else 0.  Tied embeddings (Llama 3.2) need no flag: pass the
 * embedding table as the LM head.
 * n_experts, top_k: a mixture of experts in place of the SwiGLU MLP (the
 * Mixtral 8x7B variant of Table 2): 2..8 experts per layer, top_k 1 or 2
 * of them per token, chosen by a router and weighted by the softmax of the
 * chosen router logits (the lowest index first among equal logits); 0 (or
 * 1) experts: the dense MLP.  With experts, steps run with batch < 8 and not
 * in KL_MODE_PER_OP (KL_ERR_UNSUPPORTED otherwise). */
typedef struct {
    int32_t n_layers, hidden, n_heads, n_kv_heads, head_dim, ffn_dim, vocab;
    float rope_theta, rms_eps;
    int32_t max_batch, max_seq;
    int32_t qkv_bias;
    int32_t n_experts, top_k;
} kl_config;

/* One decoder layer's weights: dev bf16, nn.Linear layout [out][in].
 *   attn_norm, ffn_norm [hidden]
 *   wq [n_heads*head_dim][hidden], wk, wv [n_kv_heads*head_dim][hidden]
 *   wo [hidden][n_heads*head_dim]
 *   w_gate, w_up [ffn_dim][hidden], w_down [hidden][ffn_dim]
 *   bq [n_heads*head_dim], bk, bv [n_kv_heads*head_dim]: the Q/K/V biases,
 *   required with cfg.qkv_bias and ignored (may be NULL) without
 *   with n_experts > 1: w_gate, w_up [n_experts][ffn_dim][hidden],
 *   w_down [n_experts][hidden][ffn_dim] (the experts' MLPs, stacked) and
 *   w_router [n_experts][hidden]; w_router is ignored (may be NULL) without */
typedef struct {
    const void *attn_norm, *wq, *wk, *wv, *wo, *ffn_norm, *w_gate, *w_up, *w_down;
    const void *bq, *bk, *bv;
    const void *w_router;
} kl_layer_ptrs;

/* Whole model: dev bf16 embed [vocab][hidden], final_norm [hidden],
 * lm_head [vocab][hidden] (untied); layers is a host array of n_layers. */
typedef struct {
    const void *embed, *final_norm, *lm_head;
    const kl_layer_ptrs *layers;
} kl_weight_ptrs;

/* Caller-owned KV cache: dev bf16 k and v, each
 * [n_layers][batch][n_kv_heads][capacity][head_dim], holding post-RoPE keys.
 * 'batch' is the allocated batch extent (>= the step's batch), 'capacity'
 * the allocated positions per sequence.  16-byte aligned. */
typedef struct {
    void *k, *v;
    int32_t batch, capacity;
} kl_kv_cache;

typedef struct kl_state kl_state;

/* Read-only facts about a loaded model (for benches and tests). */
typedef struct {
    int32_t n_workgroups;       /* persistent grid size used by every mode        */
    int32_t threads_per_group;
    int32_t lds_bytes;          /* dynamic LDS per workgroup                       */
    int32_t attn_chunks_b1;     /* KV chunks per (sequence, KV head) at batch 1, at
                                   most (a chunk has 4 KiB of keys or more)        */
    int32_t mfma_min_batch;     /* steps with batch >= this run the weight products
                                   on the matrix cores                             */
    int64_t arena_bytes;        /* packed weights + gains                          */
    int64_t scratch_bytes;      /* activations, partials, counters                 */
    int64_t noalloc_scratch_bytes;  /* scratch a kl_decode_step_noalloc call at
                                       max_batch needs (besides a fixed reserve of
                                       the library for hand-off words)             */
    int64_t noalloc_scratch_limit;  /* bytes of the static scratch                  */
} kl_info;

/* Load a model: validates cfg, allocates the packed weight arena, the RoPE
 * table and the step scratch on the current device, and repacks the caller's
 * weights into the gfx950 layout with kernels on 'stream'.  Returns after the
 * stream has finished the packing, so the caller may free the source weights.
 * The grouped weights of all layers are laid out linearly in one arena (the
 * grouping rule of Sec. 3.2, Eq. 3, with the linear layout it suggests).
 * On success *out owns every allocation; release with kl_free_model. */
kl_status kl_load_model(const kl_config *cfg, const kl_weight_ptrs *weights, void *stream,
                        kl_state **out);

/* Incremental loading, for models whose source weights cannot sit in device
 * memory beside the packed copy (e.g. the 70B shape on one GPU): the same
 * result as kl_load_model, one layer at a time.
 *   kl_model_create      validates cfg and allocates everything kl_load_model
 *                        allocates; the weights start as zeros.
 *   kl_model_set_layer   packs layer 'layer' (0 <= layer < n_layers) from the
 *                        caller's device pointers (layout of kl_layer_ptrs);
 *                        returns after the packing finished on 'stream', so
 *                        the caller may free the source right away.
 *   kl_model_set_globals packs the embedding, final norm and LM head (layouts
 *                        of kl_weight_ptrs), likewise synchronously.
 * Steps may run once every layer and the globals are set (earlier steps
 * compute with zero weights).  Errors as for kl_load_model; a failed set call
 * leaves the model usable for another attempt. */
kl_status kl_model_create(const kl_config *cfg, kl_state **out);
kl_status kl_model_set_layer(kl_state *st, int32_t layer, const kl_layer_ptrs *weights,
                             void *stream);
kl_status kl_model_set_globals(kl_state *st, const void *embed, const void *final_norm,
                               const void *lm_head, void *stream);

/* Enqueue one decode step on 'stream' (asynchronous): the token step of the
 * paper's Sec. 2 and Fig. 3 (Embedding -> L x Decoder -> Classifier), for
 * every sequence of the batch.  In KL_MODE_LOOPED the L decoder-layer calls
 * are collapsed into one call of the looped kernel (Sec. 3.2: the grouped
 * per-layer arguments become one linearly laid-out argument, the call sites
 * collapse into one); the other modes issue one launch per layer or per
 * operator group.  Every mode computes the same bits.
 *   token_ids  dev int32 [batch]   token of each sequence
 *   positions  dev int32 [batch]   position p of the new token; the step writes
 *                                  K/V slot p of every layer and attends over
 *                                  slots 0..p
 *   batch      1 <= batch <= min(max_batch, kv->batch)
 *   kv         caller's cache (layout above); capacity <= max_seq
 *   logits_out dev fp32 [batch][vocab]
 *   hidden_out dev fp32 [batch][hidden] or NULL: the residual stream after the
 *              last layer (before the final norm)
 *   mode       a kl_mode
 * Host-checkable errors (NULL or misaligned pointers, batch or capacity out
 * of range, an unknown mode, the wrong current device) return a negative
 * status with nothing enqueued.  Out-of-range token ids or positions can only
 * be seen on the device: they set bits in the device error word, and that
 * sequence is skipped as described with the bits.  One step may be in flight
 * per state; the caller's buffers are borrowed until the step completes in
 * stream order. */
kl_status kl_decode_step(kl_state *st, const int32_t *token_ids, const int32_t *positions,
                         int32_t batch, const kl_kv_cache *kv, float *logits_out,
                         float *hidden_out, void *stream, int32_t mode);

/* Greedy token loop: n_steps decode steps in a row on 'stream', each one's
 * sampled tokens feeding the next on the device (the Sampling block, executed
 * once per output token, Sec. 2 and Fig. 3; the paper does not fix the
 * sampler: greedy, the largest logit, the lowest index on ties).  Step n runs
 * at positions[b] + n on the tokens step n - 1 sampled (step 0 on token_ids),
 * writes K/V slot positions[b] + n of every layer, and samples in the LM
 * head's epilogue (no separate kernel, no host round trip).
 *   token_ids, positions, batch, kv, mode   as for kl_decode_step
 *   n_steps     >= 1
 *   tokens_out  dev int32 [n_steps][batch]: the token sampled at each step
 *   logits_out  dev fp32 [batch][vocab]: every step's logits in turn (the last
 *               step's remain)
 * A sequence whose token or position is out of range at some step is skipped
 * from then on (error bits as for kl_decode_step; it samples token -1).  Same
 * host-side errors as kl_decode_step, plus n_steps < 1 or a NULL or
 * misaligned tokens_out; nothing is enqueued then. */
kl_status kl_decode_greedy(kl_state *st, const int32_t *token_ids, const int32_t *positions,
                           int32_t batch, int32_t n_steps, const kl_kv_cache *kv,
                           int32_t *tokens_out, float *logits_out, void *stream, int32_t mode);

/* kl_decode_step for callers that cannot allocate device memory (code under
 * HIP graph capture, tight serving loops, harnesses that forbid allocation):
 * the same arguments, results and errors, bit-identical outputs, and it calls
 * no allocating routine.  Its step scratch is not the state's but a static
 * array of the library, one per device, of kl_info.noalloc_scratch_limit bytes
 * (32 MiB), held until the process ends; a step that needs more (see
 * kl_info.noalloc_scratch_bytes: e.g. the 70B shape on the matrix-core path) returns
 * KL_ERR_UNSUPPORTED with nothing enqueued.  Each call first clears the
 * scratch it uses with a fill kernel on 'stream' (one extra launch), so no
 * state carries over from an earlier call.  Every call on a device shares
 * that device's array: calls that may overlap in time on one device (other
 * streams, other threads, other states) race and must be serialized by the
 * caller. */
kl_status kl_decode_step_noalloc(kl_state *st, const int32_t *token_ids,
                                 const int32_t *positions, int32_t batch, const kl_kv_cache *kv,
                                 float *logits_out, float *hidden_out, void *stream,
                                 int32_t mode);

/* ---------------------------------------------------------------- paged cache
 *
 * A KV cache in pages: sequences of any length share one pool, and an 8-bit
 * pool holds twice the positions of a bf16 one and halves what the attention
 * reads.  Three operators work on one layer of a pool: kl_paged_append writes
 * rows (a decode step's or a prompt's, quantised as they are written),
 * kl_paged_read reads rows back, kl_paged_attention attends one new token per
 * sequence over its cached positions.  All are asynchronous on 'stream',
 * allocate nothing, synchronise nothing and may be captured into a graph.
 *
 * Conditions only the device can see set bits of the caller's device error
 * word (int32, 4-byte aligned; NULL: not reported), with an atomic or; it is
 * never cleared by these calls. */
typedef enum {
    KL_DTYPE_BF16 = 0,
    KL_DTYPE_FP16 = 1,
    KL_DTYPE_FP32 = 2,
    KL_DTYPE_E4M3 = 3    /* OCP 8-bit float (4 exponent, 3 mantissa bits, largest 448) */
} kl_dtype;

/* The pool.  Entry (layer, page, head, offset) of k and v is a row of
 * head_dim values: dev [n_layers][n_pages][n_kv_heads][page_size][head_dim],
 * 16-byte aligned.  dtype KL_DTYPE_BF16: the values.  KL_DTYPE_E4M3: codes,
 * value = code * 2^(s - 127) with the row's byte s (1..254) in k_scale,
 * v_scale: dev [n_layers][n_pages][n_kv_heads][page_size], 8-byte aligned
 * (NULL with KL_DTYPE_BF16).  A power of two costs an 8-bit float no
 * precision (the significand is scaled by nothing), every product with it is
 * exact in fp32, and from s = 3 on in bf16 (at 1 and 2 the smallest codes are
 * multiples of 2^-135 and 2^-134, bf16's least step is 2^-133).
 * page_size: a power of two, 8..4096.  head_dim: 64 or 128.  device: the HIP
 * device of the pool, current in every call. */
typedef struct {
    void *k, *v;
    uint8_t *k_scale, *v_scale;
    int32_t dtype;
    int32_t n_layers, n_pages, n_kv_heads, page_size, head_dim;
    int32_t device;
} kl_paged_cache;

/* Which pages hold a sequence: position p of sequence b is in page
 * pages[b * stride + p / page_size] at offset p % page_size (dev int32,
 * stride >= max_pages elements).  Entries of positions not in use may hold
 * anything.
 * max_pages * page_size <= 2^30. */
typedef struct {
    const int32_t *pages;
    int32_t batch, max_pages, stride;
} kl_page_table;

/* Rows of heads: element i of head h of row r at data + r * row_stride +
 * h * head_stride + i (strides in elements, >= 0; of outputs, where there is
 * more than one row or head, >= head_dim).  dtype: KL_DTYPE_BF16, _FP16 or
 * _FP32.  data is aligned to its element. */
typedef struct {
    void *data;
    int32_t dtype;
    int64_t row_stride, head_stride;
} kl_rows;

/* Writes rows 0..rows-1 of k and v (n_kv_heads heads each) to the slots of
 * (seq[r], positions[r]); seq NULL: row r is sequence r's.
 *   seq        dev int32 [rows] or NULL (then rows <= table->batch)
 *   positions  dev int32 [rows]; a negative position: a padding row, skipped
 * bf16 pool: values rounded to nearest even.  e4m3 pool, per row and head
 * with a = max |x|: e = the smallest integer >= -126 with a <= 448 2^e, scale
 * byte e + 127, code = x 2^-e rounded to nearest even; a row with an infinity
 * or NaN reads back as NaN throughout.  Every other slot stays as it was.  Two
 * rows with the same slot in one call leave it unspecified.
 * Device error bits: KL_DEVERR_POSITION for a sequence outside [0, batch) or
 * a position >= max_pages * page_size, KL_DEVERR_PAGE for a bad table entry;
 * such a row is skipped. */
kl_status kl_paged_append(const kl_paged_cache *cache, int32_t layer, const kl_page_table *table,
                          const int32_t *seq, const int32_t *positions, int64_t rows,
                          const kl_rows *k, const kl_rows *v, int32_t *error, void *stream);

/* Reads the slots of (seq[r], positions[r]) into rows of k and v, rounded to
 * their type (nearest even).  Arguments and error bits as for
 * kl_paged_append; a padding row's output stays as it was, a bad row's is
 * NaN.  With strides of a kl_kv_cache's layer and sequence as output, a
 * sequence moves from pages to the contiguous cache of kl_decode_step. */
kl_status kl_paged_read(const kl_paged_cache *cache, int32_t layer, const kl_page_table *table,
                        const int32_t *seq, const int32_t *positions, int64_t rows,
                        const kl_rows *k, const kl_rows *v, int32_t *error, void *stream);

/* Bytes of the workspace of kl_paged_attention calls of up to 'batch'
 * sequences (at most 4096) over this pool, with any number of heads (0 if an
 * argument is invalid). */
size_t kl_paged_attention_workspace(const kl_paged_cache *cache, int32_t batch);

/* Attention of one new token per sequence (sequence b is row b of q and out)
 * over its first lengths[b] cached positions, the new one's among them:
 *   out_h = sum_j p_j v_j / sum_j p_j,  p_j = exp(scale q_h . k_j),
 * j in [lengths[b] - window, lengths[b]) and >= 0 (window 0: from 0), query
 * head h with KV head h / (n_heads / n_kv_heads).
 *   lengths    dev int32 [batch]; 0: no position (a padded batch): the output
 *              row is zero and its lse -infinity
 *              (batch * n_kv_heads * max_pages * page_size <= 2^35)
 *   q, out     n_heads heads; n_heads a multiple of n_kv_heads, at most 16
 *              times as many
 *              (out overlaps neither q nor the pool)
 *   scale      at most 2^127 in magnitude (scores are taken times log2 e)
 *   lse        dev fp32 [batch][n_heads] or NULL: max_j + ln sum_j of scale q.k
 *              (what joins this result with one over other positions)
 *   workspace  dev, 16-byte aligned, at least kl_paged_attention_workspace()
 *              bytes, zeroed by the caller before its first use; every call
 *              leaves it ready for the next one.  Calls that may run at the
 *              same time (other streams, graphs replayed side by side) need a
 *              workspace each.
 * Keys and values are taken as bf16: those of an e4m3 pool exactly from scale
 * byte 3 on, below it rounded to multiples of 2^-133.  Scores, softmax and sums
 * are held in 32 bits, and a sequence's result does not depend on timing (parts
 * are joined in a fixed order).  Slots outside the attended positions do not
 * affect the result, whatever they hold; with a NaN or an infinity in an attended
 * slot the outputs of its KV head's query heads may be NaN.  A score that
 * overflows downwards has no weight, whatever the type of q; with one that
 * overflows upwards the head's outputs are NaN.
 * Device error bits: KL_DEVERR_POSITION for a length outside [0, max_pages *
 * page_size], KL_DEVERR_PAGE for a bad table entry of an attended position;
 * the sequence's output row and lse are then NaN. */
kl_status kl_paged_attention(const kl_paged_cache *cache, int32_t layer,
                             const kl_page_table *table, const int32_t *lengths, const kl_rows *q,
                             int32_t n_heads, float scale, int32_t window, const kl_rows *out,
                             float *lse, void *workspace, size_t workspace_bytes, int32_t *error,
                             void *stream);

/* kl_decode_step over a paged cache: sequence b's row of the page table says
 * where its positions are; the step writes the new token's K/V to position
 * positions[b]'s slot of every layer (as kl_paged_append) and attends over
 * positions 0..positions[b] (as kl_paged_attention), so an e4m3 pool halves
 * the cache that a step reads.  It runs on the matrix-core path at every batch,
 * two launches per layer with the two operators' between them (4 L + 1
 * dispatches).  It may be captured into a graph, whose replays take about 37 us
 * less per layer than the call.
 *   cache    of the model's n_layers, n_kv_heads, head_dim and device
 *   table    batch >= the step's; positions are < max_pages * page_size and
 *            < max_seq (batch * n_kv_heads * the smaller of the two <= 2^35)
 * The other arguments, results and errors as for kl_decode_step; a bad table
 * entry up to the position's sets KL_DEVERR_PAGE, and its sequence is skipped
 * as one with a bad position (KL_DEVERR_POSITION).  KL_ERR_UNSUPPORTED for a
 * mixture of experts, and for a model loaded with a max_batch below
 * kl_info.mfma_min_batch. */
kl_status kl_decode_step_paged(kl_state *st, const int32_t *token_ids, const int32_t *positions,
                               int32_t batch, const kl_paged_cache *cache,
                               const kl_page_table *table, float *logits_out, float *hidden_out,
                               void *stream);

/* Bytes of ONE of the K or V buffers for the given batch and capacity
 * (0 if cfg is invalid). */
size_t kl_kv_cache_bytes(const kl_config *cfg, int32_t batch, int32_t capacity);

/* Synchronizes the device, returns the device error word in *code (KL_DEVERR_*
 * bits, 0 = none) and clears it.  Returns KL_ERR_DEVICE_FAULT when *code != 0. */
kl_status kl_get_device_error(kl_state *st, int32_t *code);

kl_status kl_get_info(const kl_state *st, kl_info *info);

/* Timeline of the phases, for profiling the schedules (the kind of
 * synchronization-cost breakdown of Sec. 2, Fig. 5).  While a buffer is set,
 * every later launch writes, for phase i < max_phases of the launch (in the
 * order embed, then qkv, attn, oproj, gateup, down per layer, then head) and
 * workgroup w, s_memrealtime stamps (100 MHz ticks) into
 *   dev_buffer[(i * n_workgroups + w) * 4 + {0: phase end (every wave of the
 *   workgroup done; its writes complete where the phase ends on a barrier,
 *   issued where it hands tagged words to the next phase), 1: start of the
 *   wait for its inputs, 2: end of that wait, 3: inputs staged (in LDS on the
 *   per-sequence path; matrix-core path: the workgroup's share of the
 *   grid-wide step before the product, RMSNorm or SwiGLU fold, done; an
 *   attention phase: its chunk result published)}]
 * (slots a workgroup does not reach keep their old contents; a launch
 * overwrites the previous launch's entries).  The buffer (dev, uint64,
 * max_phases * n_workgroups * 4 entries) stays owned by the caller; pass NULL
 * to stop tracing. */
kl_status kl_set_trace(kl_state *st, uint64_t *dev_buffer, int32_t max_phases);

/* Measurement helper (no model involved): reads every byte of the device
 * buffer buf (bytes, both 16-byte aligned) once with the step kernel's
 * 16-byte non-temporal loads, 16 in flight per lane, on a grid of workgroups
 * x 512 lanes (1..65536 workgroups), and writes nothing the caller relies on
 * (dev_out, one device uint32, is at most written with an unspecified value).
 * Timed by the caller, it gives the read-stream rate this load pattern
 * reaches: the practical ceiling of a kernel whose traffic is one pass over
 * its weights (the roofline of Sec. 4.4's bandwidth comparison is the
 * nominal peak).  Asynchronous on stream; invalid arguments return
 * KL_ERR_INVALID_ARGUMENT with nothing enqueued. */
kl_status kl_read_stream(const void *buf, size_t bytes, int32_t workgroups, uint32_t *dev_out,
                         void *stream);

/* Frees everything the state owns (synchronizes the device first). NULL is a no-op. */
void kl_free_model(kl_state *st);

/* Message describing the last failing call on this thread ("" if none). */
const char *kl_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* KL_H */
