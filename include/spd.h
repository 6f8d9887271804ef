/*
 * libspd -- Superposed Decoding (arXiv 2405.18400) hot path for AMD MI355X (gfx950).
 *
 * One SPD timestep (Section 3; Algorithm 1, else-branch), entirely on the GPU:
 *   superposition weights (Section 3.1, Eq. 2) -> superposed input embedding (Eq. 1) ->
 *   batch-1 decoder forward over one shared key/value cache (Section 3, "Next Timesteps")
 *   -> full-vocabulary log-softmax with temperature and KeepTopK (Algorithm 1) ->
 *   k x k draft options -> n-gram mixture (Section 3.2, Eq. 3) -> interpolation (Eq. 4)
 *   or the no-overlap penalty form (Eq. 5) -> keep the k most probable options and update
 *   their probabilities (Section 3, Eq. for D and P).
 * Around it: the pass over the prefix (Section 3, "First Timestep"; spd_prefill), one pass of
 * nucleus sampling on the same forward (the comparison decoder of Section 4.3;
 * spd_nucleus_step), and committing one draft to restart from it (resets, Section 5.3; a
 * nucleus-sampled opening in front of Superposed Decoding, Section 4.5; spd_commit).
 *
 * Conventions
 *   - Every function returns SPD_OK (0) or a negative spd_status.  No exceptions, no global
 *     state.  spd_last_error() gives a human-readable reason for the last failure on a ctx.
 *   - "device" pointers are HIP device memory owned by the CALLER (the library never
 *     allocates or frees device memory); "host" pointers are ordinary host memory.
 *   - All GPU work is enqueued on the hipStream_t given to spd_create (passed as void*;
 *     NULL = the default stream).  A call that fills host outputs synchronises that stream
 *     before returning; a call with no host outputs does not synchronise.
 *   - Scores cross this boundary as natural-log probabilities.
 *   - Matrices are row-major [out_features, in_features], contiguous, 16-byte aligned,
 *     stored in cfg.dtype (fp32, or bf16 bit patterns).  Norm gains use the same dtype.
 *   - One ctx serves one generation at a time; calls on one ctx must not overlap.
 */
#ifndef SPD_H
#define SPD_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define SPD_K_MAX 16      /* compile-time ceiling on the number of drafts k            */
#define SPD_MIN_ORDER 2   /* n-gram orders n = 2..6 (Section 3.2)                      */
#define SPD_MAX_ORDER 6
#define SPD_N_ORDERS 5
#define SPD_TAIL 5        /* tokens of history an order-6 context needs                */

typedef enum {
    SPD_OK = 0,
    SPD_EINVAL = -1,        /* bad argument (null pointer, shape, alignment, range)      */
    SPD_ESTATE = -2,        /* call out of order (e.g. step before prefill)              */
    SPD_ECTX_OVERFLOW = -3, /* the key/value cache would exceed cfg.max_ctx              */
    SPD_EWORKSPACE = -4,    /* workspace / table buffer too small or misaligned          */
    SPD_ETABLE = -5,        /* n-gram table rejected (duplicate key, id >= vocab, ...)   */
    SPD_EHIP = -6           /* a HIP runtime call failed                                 */
} spd_status;

typedef enum {
    SPD_DTYPE_FP32 = 0, SPD_DTYPE_BF16 = 1, SPD_DTYPE_FP16 = 2 /* key/value cache only */,
    SPD_DTYPE_INT8 = 3 /* paged cache of codes and scales only, where an operator says so */
} spd_dtype;

/* Decoder-only transformer f_theta: RMSNorm, rotary on adjacent pairs (x_2i, x_2i+1) with
 * angle pos * rope_theta^(-2i/d_head), causal attention scaled by 1/sqrt(d_head), SwiGLU
 * feed-forward, untied embedding / LM head, no biases.  d_head = d_model / n_heads. */
typedef struct {
    int32_t n_layers, d_model, n_heads, n_kv_heads, d_ffn, vocab;
    int32_t max_ctx;   /* key/value cache capacity in positions (prefix + generated)        */
    int32_t k_max;     /* largest k any spd_step will use, 1..SPD_K_MAX                     */
    int32_t dtype;     /* spd_dtype of the weights: SPD_DTYPE_FP32 or SPD_DTYPE_BF16        */
    float rms_eps, rope_theta;
    int32_t kv_dtype;  /* element type of the key/value cache: SPD_DTYPE_FP32 (0, the default: every
                        * cached key and value keeps the fp32 result of its projection) or, with
                        * bf16 weights only, SPD_DTYPE_FP16 (rounded to nearest even on the way in:
                        * half the cache bytes per step and per position; adds about 3e-3 of the
                        * logit scale over 32 layers, within the 2e-2 of a bf16 model's rounding) */
} spd_model_cfg;

typedef struct {
    const void *attn_norm; /* [d_model]                                                    */
    const void *wqkv;      /* [(n_heads + 2 n_kv_heads) d_head, d_model]: q rows, k, v      */
    const void *wo;        /* [d_model, n_heads d_head]                                     */
    const void *ffn_norm;  /* [d_model]                                                    */
    const void *w_gate;    /* [d_ffn, d_model]                                              */
    const void *w_up;      /* [d_ffn, d_model]                                              */
    const void *w_down;    /* [d_model, d_ffn]                                              */
} spd_layer_weights;

/* Borrowed device pointers; they must stay valid until spd_destroy. `layers` is a HOST
 * array of n_layers structs (copied by spd_create). */
typedef struct {
    const void *embed;      /* [vocab, d_model] token embeddings z (Section 3.1)            */
    const spd_layer_weights *layers;
    const void *final_norm; /* [d_model]                                                   */
    const void *lm_head;    /* [vocab, d_model]                                             */
} spd_weight_ptrs;

/* N-gram frequency tables (Section 4: every unique n-gram with its count), HOST memory.
 * Order n uses index n-2.  keys[n-2] is int32 [n_entries[n-2], n] row-major (oldest token
 * first, predicted token last); counts[n-2] is uint32 [n_entries[n-2]].  An order may be
 * empty (n_entries 0, pointers may be NULL).  lambda[n-2] is that order's mixture weight
 * (Eq. 3); the paper's values are 0.01, 0.04, 0.15, 0.18, 0.12 (Appendix B). */
typedef struct {
    const int32_t *keys[SPD_N_ORDERS];
    const uint32_t *counts[SPD_N_ORDERS];
    int64_t n_entries[SPD_N_ORDERS];
    float lambda[SPD_N_ORDERS];
} spd_ngram_host_tables;

/* Per-call decoding parameters (Appendix B): number of drafts k, interpolation weight
 * alpha in [0,1] (0 = n-gram smoothing disabled), temperature tau > 0 applied to the logits
 * of the full-vocabulary softmax, no-overlap penalty delta > 0 (Eq. 5). */
typedef struct {
    int32_t k;
    float alpha, tau, delta;
} spd_decode_cfg;

typedef struct spd_ctx spd_ctx;

/* Bytes of device workspace spd_create needs for this shape (KV cache, activations,
 * attention partials, draft state, token history). Host-only; touches no GPU. */
int spd_workspace_bytes(const spd_model_cfg *cfg, size_t *out_bytes);

/* Create a decoding context.  `workspace` is caller-owned DEVICE memory of at least
 * spd_workspace_bytes() bytes, 256-byte aligned, untouched by the caller until
 * spd_destroy.  `hip_stream` is a hipStream_t (or NULL).  Validates shapes and alignment
 * before any GPU work.  *out is set only on success and is freed by spd_destroy. */
int spd_create(const spd_model_cfg *cfg, const spd_weight_ptrs *weights, void *workspace,
               size_t workspace_bytes, void *hip_stream, spd_ctx **out);
void spd_destroy(spd_ctx *ctx);

/* Bytes of DEVICE memory spd_load_ngrams needs for these tables (exact-key hash table of
 * all n-grams plus one context-total entry per distinct context).  Host-only. */
int spd_ngram_table_bytes(const spd_ngram_host_tables *tables, size_t *out_bytes);

/* Build the device-resident n-gram store (Section 3.2; the paper keeps these in host
 * dictionaries, Section 4.3) in `dev_buf` (caller-owned DEVICE memory, 256-byte aligned,
 * kept alive while in use) and attach it to ctx.  Rejects (SPD_ETABLE) a duplicate key, a
 * token id outside [0, vocab) or a zero count.  May be called again at any time outside a
 * step to swap tables.  Synchronises the stream.  Without tables only alpha = 0 is legal. */
int spd_load_ngrams(spd_ctx *ctx, const spd_ngram_host_tables *tables, void *dev_buf,
                    size_t dev_bytes);

/* First-timestep forward (Section 3, "First Timestep"): reset the generation, run the
 * model over prefix[0..m-1] (HOST int32 ids in [0, vocab), 1 <= m < max_ctx), fill cache
 * positions 0..m-1 and keep the last position's logits.  Does not synchronise. */
int spd_prefill(spd_ctx *ctx, const int32_t *prefix, int32_t m);

/* Advance every draft by one token.  The first call after spd_prefill gives draft i the
 * i-th most probable token of p_theta(. | M) with that token's log-probability as its
 * score (no n-gram term); later calls run one full SPD timestep.  dc->k must stay the same
 * between a prefill and the end of its generation.  Outputs are HOST arrays of k entries,
 * best draft first, each may be NULL: the newest token of each surviving draft, the index
 * (0..k-1, in the previous step's order; -1 at the first step) of the draft it extends,
 * and its log-score.  If all three are NULL the call does not synchronise. */
int spd_step(spd_ctx *ctx, const spd_decode_cfg *dc, int32_t *out_last_tokens,
             int32_t *out_parents, float *out_logscores);

/* Algorithm 1 end to end: spd_prefill + n_tokens spd_steps, then rebuild the drafts from
 * the per-step parent indices.  out_drafts is HOST int32 [k, n_tokens] row-major, best
 * draft first; out_logscores HOST float [k].  Synchronises. */
int spd_generate(spd_ctx *ctx, const int32_t *prefix, int32_t m, const spd_decode_cfg *dc,
                 int32_t n_tokens, int32_t *out_drafts, float *out_logscores);

/* ---- state access: resets (Section 5.3) and step-by-step comparison with a reference ---- */

/* Read the k drafts' bookkeeping (HOST outputs, any may be NULL): tails int32 [k, SPD_TAIL]
 * = the last 5 tokens of (prefix, draft), oldest first, -1 where the history is shorter;
 * logscores float [k]; gamma float [k] = the superposition weights (Eq. 2) of the current
 * scores.  Synchronises. */
int spd_get_state(spd_ctx *ctx, int32_t *out_k, int32_t *out_tails, float *out_logscores,
                  float *out_gamma);
/* Overwrite the drafts' bookkeeping (HOST inputs) between steps; the KV cache is untouched.
 * Legal once the first step after a prefill has run.  Synchronises. */
int spd_set_state(spd_ctx *ctx, int32_t k, const int32_t *tails, const float *logscores);
/* Copy the logits [vocab] of the most recent forward pass to HOST memory.  Synchronises. */
int spd_read_logits(spd_ctx *ctx, float *out_logits);

/* What the most recent step decided (HOST outputs, any may be NULL): the kept token ids
 * int32 [k] and their log p_theta float [k] (Algorithm 1, KeepTopK); for each option
 * (i, j) = draft i + kept token j, row-major [k, k]: its score log p_i + log p_f (float),
 * whether it was an option at all (int32 0/1; options outside the overlap set are not,
 * Section 3.2) and the n-gram mixture value p_ngram (float, Eq. 3).  Synchronises. */
int spd_get_step_info(spd_ctx *ctx, int32_t *out_top_ids, float *out_top_logp,
                      float *out_cand_scores, int32_t *out_cand_valid, float *out_cand_pngram);

/* Run only the post-forward part of a timestep (KeepTopK, expansion, n-gram probes,
 * interpolation, prune, state update) on caller-supplied DEVICE logits float [vocab], as
 * if the forward pass had produced them.  `first` != 0 performs the first-timestep
 * initialisation instead.  Requires a prior spd_prefill (it provides the history).  Does
 * not touch the KV cache or the position.  Does not synchronise. */
int spd_expand_prune(spd_ctx *ctx, const spd_decode_cfg *dc, const float *dev_logits, int32_t first);

/* Commit one draft and restart (Section 5.3, "Superposed Decoding Resets": every s timesteps
 * one of the k drafts is sampled and draft generation restarts; Section 4.5: a nucleus-sampled
 * generation of any length serves as the prefix of a Superposed Decoding run).
 * Draft i is sampled with its superposition weight gamma_i (Eq. 2) by inverse CDF over the
 * drafts in rank order with the caller's draw u in [0, 1); its tokens since the last
 * spd_prefill / spd_commit are appended to the text, the cache positions they occupy are
 * recomputed from the tokens themselves (with one draft, k = 1, only the newest token's), and
 * the context is left as after spd_prefill of the extended text: the next spd_step (any k) or
 * spd_nucleus_step starts a generation from it.  Outputs are HOST, each may be NULL: the
 * sampled draft's index, its tokens (cap entries available) and their number.  Synchronises. */
int spd_commit(spd_ctx *ctx, float u, int32_t *out_chosen, int32_t *out_tokens, int32_t cap, int32_t *out_n);

/* ---- the comparison decoder: one pass of nucleus (top-p) sampling ----
 * Section 4.3 times Superposed Decoding against k independent passes of nucleus sampling;
 * Section 2 describes the sampler: the next-token distribution is cut to the smallest set of
 * most probable tokens whose cumulative probability reaches top_p and renormalised.  Here:
 * probabilities are the full-vocabulary softmax of logits / tau; tokens are ordered by
 * probability, the lower id first among equals; the nucleus is the shortest prefix of that
 * order whose mass reaches top_p; the draw u in [0, 1) (supplied by the caller, who owns the
 * random number generator) selects the first token whose cumulative probability in that
 * order exceeds u times the nucleus mass. */
typedef struct spd_sample_cfg {
    float top_p; /* in (0, 1] */
    float tau;   /* > 0 */
} spd_sample_cfg;

/* One token of one pass.  The first call after spd_prefill samples from the prefix pass's
 * logits; every later call feeds the previously sampled token's embedding through the
 * transformer (one more cached position) and samples from the new logits.  out_token /
 * out_logprob: HOST, may be NULL (then the call does not synchronise); the log-probability
 * is that of the sampled token under the full-vocabulary softmax.  A pass and an SPD
 * generation with k > 1 cannot be interleaved on one context (SPD_ESTATE); spd_prefill
 * starts either. */
int spd_nucleus_step(spd_ctx *ctx, const spd_sample_cfg *sc, float u, int32_t *out_token, float *out_logprob);

/* Run only the sampler (not the transformer) on caller-supplied DEVICE logits float [vocab],
 * as if the forward pass had produced them; `first` != 0 starts a pass (as the first
 * spd_nucleus_step after spd_prefill does).  Does not touch the KV cache or the position.
 * Does not synchronise; read the result with spd_get_state / spd_get_nucleus_info. */
int spd_nucleus_sample(spd_ctx *ctx, const spd_sample_cfg *sc, float u, const float *dev_logits, int32_t first);

/* Size and probability mass of the nucleus of the most recent sampling call, and the sum
 * of the log-probabilities of the tokens sampled so far in this pass.  HOST outputs, any may
 * be NULL.  Synchronises. */
int spd_get_nucleus_info(spd_ctx *ctx, int32_t *out_size, float *out_mass, float *out_sum_logprob);

/* Current position (= number of cached positions) as tracked by the host. */
int spd_position(const spd_ctx *ctx, int32_t *out_pos);

/* Turn the captured-graph replay of spd_step on (default) or off (plain launches).  It applies to the forward of one kernel per
 * matrix-vector product; a timestep of the persistent forward is two or three launches, which are made plainly either way. */
int spd_set_graph(spd_ctx *ctx, int32_t enable);

/* The transformer forward of a timestep runs either as one persistent kernel ("fused": the
 * default wherever an instantiation exists for the model shape) or as one kernel per
 * matrix-vector product.  Both compute the same thing; spd_set_fused switches between them
 * (SPD_EINVAL when asked for a fused kernel the shape has none for), spd_get_fused tells
 * which one runs. */
int spd_set_fused(spd_ctx *ctx, int32_t enable);
int spd_get_fused(const spd_ctx *ctx, int32_t *out_enabled);

/* spd_prefill runs the prefix either one token at a time through the timestep's forward, or
 * ("dense": the default for bf16 models whose widths allow it, for prefixes of 8 tokens or
 * more; spd_commit uses the same pass) up to 1024 prefix tokens at a time as matrix-matrix
 * products on the matrix cores, reading the weights once per chunk.  Both fill the same cache
 * and leave the same logits up to fp32 rounding.  A dense pass exists for bf16 weights,
 * d_head <= 128, d_model <= 8192 and d_model, d_ffn, n_heads * d_head divisible by 128; it adds
 * 1024 rows of activations to spd_workspace_bytes.
 * fp32 models with heads of 64 or 128 and d_model, d_ffn divisible by 16 take prefixes of three tokens or more the same
 * way (two where that is the faster pass), with every product and sum in fp32 (1024 rows, or max_ctx if that is less, in
 * spd_workspace_bytes; a workspace without them is taken too, and such a context has no dense pass).
 * spd_set_dense_prefill switches between the passes, back and forth (SPD_EINVAL when asked for a dense pass the model has
 * none for); spd_get_dense_prefill says whether the dense one is in use. */
int spd_set_dense_prefill(spd_ctx *ctx, int32_t enable);
int spd_get_dense_prefill(const spd_ctx *ctx, int32_t *out_enabled);

/* Per-kernel timing for profiling runs: when enabled, spd_step launches kernels one by one
 * with a HIP event pair around each and accumulates the elapsed time per kernel class.
 * spd_get_kernel_timing fills HOST arrays of up to `cap` entries (class name pointers valid
 * for the ctx lifetime, total milliseconds, launch counts), sets *out_n, and synchronises.  "expand_prune" includes the
 * selection from the logits' slices where one launch does both ("topk_partial" then has none); a dense prefix pass is not
 * timed. */
int spd_set_kernel_timing(spd_ctx *ctx, int32_t enable);
int spd_get_kernel_timing(spd_ctx *ctx, int32_t cap, const char **out_names, float *out_ms,
                          int64_t *out_launches, int32_t *out_n);

/* While kernel timing is on, every block of the fused forward kernel records a 100 MHz clock
 * stamp before and after each of its device-wide barriers (and at its end):
 * stamp[2i] = arrival at barrier i, stamp[2i+1] = release, i = 0 .. 5 n_layers (barrier 0
 * follows the input phase; each layer then has QKV, attention, O, gate/up, down).  Copies the
 * stamps of the most recent fused forward to HOST memory as [*out_blocks][*out_n] (the first
 * 512 blocks at most) with
 * *out_n = 2 (5 n_layers + 2); `cap` counts int64 elements of out_stamps.  SPD_ESTATE when
 * the model shape has no fused kernel. */
int spd_get_phase_clock(spd_ctx *ctx, int32_t cap, int64_t *out_stamps, int32_t *out_n,
                        int32_t *out_blocks);

/* ---- stand-alone operators (the kernels of one timestep, callable one at a time) ---- */

/* y = W x (+ residual), optionally with x first RMS-normalised (x * rsqrt(mean x^2 + eps) *
 * gain).  W is DEVICE [rows, cols] in `dtype`; x, residual, y are DEVICE float; gain is
 * DEVICE [cols] in `dtype` or NULL (no normalisation); residual may be NULL or equal y. */
int spd_op_gemv(int32_t dtype, const void *W, const void *gain, float eps, const float *x,
                const float *residual, float *y, int32_t rows, int32_t cols, void *hip_stream);
/* u = silu(Wg xn) * (Wu xn) with xn = RMS-normalised x (gain may be NULL: xn = x). */
int spd_op_swiglu(int32_t dtype, const void *Wg, const void *Wu, const void *gain, float eps,
                  const float *x, float *u, int32_t rows, int32_t cols, void *hip_stream);
/* Single-query attention over n_ctx cached positions: out[h] = softmax(q[h] . K / sqrt(d_head)) V
 * with K, V DEVICE [n_kv_heads, cap_ctx, d_head] in `dtype` (head-major, as the library's
 * cache, which is fp32 or fp16: SPD_DTYPE_FP16 is accepted here too), q and out DEVICE float
 * [n_heads, d_head]; `partials` is DEVICE scratch of spd_op_attention_scratch_bytes() bytes. */
size_t spd_op_attention_scratch_bytes(int32_t n_heads, int32_t d_head, int32_t cap_ctx);
int spd_op_attention(int32_t dtype, const float *q, const void *K, const void *V, float *out,
                     void *partials, int32_t n_heads, int32_t n_kv_heads, int32_t d_head,
                     int32_t n_ctx, int32_t cap_ctx, void *hip_stream);

/* spd_op_attention for callers that cannot allocate device memory (code under HIP graph
 * capture, tight serving loops, harnesses that forbid hipMalloc): the same computation with
 * the scratch in a static device array of SPD_STATIC_SCRATCH_BYTES inside the library instead
 * of a caller-supplied buffer.  The call allocates nothing.  Shapes whose
 * spd_op_attention_scratch_bytes(n_heads, d_head, cap_ctx) exceeds SPD_STATIC_SCRATCH_BYTES are
 * refused with SPD_EWORKSPACE before any GPU work.  Each GPU holds one such array for the life
 * of the process and every call on that GPU uses it: calls on one stream are ordered, calls that
 * overlap on one GPU (other streams, other threads) race and must be serialised by the caller.  Does not synchronise. */
#define SPD_STATIC_SCRATCH_BYTES (4u << 20)
int spd_op_attention_static(int32_t dtype, const float *q, const void *K, const void *V, float *out,
                            int32_t n_heads, int32_t n_kv_heads, int32_t d_head, int32_t n_ctx,
                            int32_t cap_ctx, void *hip_stream);

/* ---- several sequences over one prompt: operators of the step of k independent passes or of a beam search ----
 * Section 4.3 holds Superposed Decoding against k independent passes and against beam search: n_seq sequences that
 * agree in their first positions.  These operators take such a batch through a step on a PAGED cache, for programs
 * that run those decoders' products themselves (and, for k independent passes, sample from several rows themselves).  The attention here
 * takes one new token per sequence; several at once (a prompt, drafts) are the next section's.
 *   K, V   DEVICE [n_pages, n_kv_heads, page_size, d_head] in `dtype` (fp32, fp16 or bf16), 16-byte aligned; page_size a
 *          power of two from 4 to 1024, d_head a power of two from 8 to 256;
 *   table  DEVICE int32 [n_seq, table_stride]: position p of sequence s is row p % page_size of page
 *          table[s][p / page_size].  Entries no call needs may hold anything.
 * Sequences come in groups of `width` consecutive ones (one prompt each).  Lengths and page numbers live on the device,
 * so that a captured step can be replayed; what the host cannot check is bounded by the kernels: a page number outside
 * [0, n_pages), a row of the table or a length out of range is never followed, and *err (DEVICE int32, may be NULL) is
 * set to 1 (and never cleared).  Calls do not synchronise and allocate nothing; those that need scratch take it from the caller, 256-byte
 * aligned and of the size the function beside them gives (0: none, NULL will do; SPD_EWORKSPACE if less), and leave nothing in it for a
 * later call: calls that may overlap need scratch of their own.  What a call writes (results, scratch, the pools it appends to or copies in) lies apart from
 * everything else that it is given, but where an operator says otherwise; SPD_EINVAL if not. */

/* New tokens' keys and values into the cache, rotated on the way: token i, at position pos[i] of sequence seq[i] (DEVICE int32
 * [n_tokens]), has k and v rows DEVICE float [n_kv_heads, d_head] at k + i kv_stride, v + i kv_stride; k (and q) are rotated on adjacent
 * pairs by pos * rope_theta^(-2i/d_head).  q (may be NULL, then n_heads is 0): rows [n_heads, d_head] at q + i q_stride; q_out
 * [n_tokens, n_heads, d_head] gets them rotated, in fp32 (it may be q where q_stride is n_heads d_head).  Strides are in elements and
 * multiples of 4, so that the parts of one product's rows can be passed as they lie; pointers 16-byte aligned.  seq[i] < 0:
 * padding, nothing of that token is read or written.  A token whose position or page is out of range is left out whole, *err is set.  No two tokens of a
 * call may name the same position of the same page. */
int spd_op_append_paged(int32_t dtype, void *K, void *V, const int32_t *table, int32_t n_pages, int32_t n_kv_heads, int32_t page_size,
                        int32_t d_head, int32_t n_seq, int32_t table_stride, const float *q, int64_t q_stride, const float *k, const float *v,
                        int64_t kv_stride, const int32_t *seq, const int32_t *pos, int32_t n_tokens, int32_t n_heads, float rope_theta,
                        float *q_out, int32_t *err, void *hip_stream);

/* One query per sequence and head: out[s][h] = softmax(q[s][h] . K / sqrt(d_head)) V over positions [0, len[s]) of
 * sequence s.  Positions below shared[g] are the same in all sequences of group g: they are read once, through the table of
 * the group's first sequence.  q, out DEVICE float [n_seq, n_heads, d_head]; shared DEVICE int32 [n_seq / width], len DEVICE int32 [n_seq].
 * max_shared >= every shared[g] and max_own >= every len[s] - shared[g] size the launch (host values; neither more than a row of
 * the table holds): the call is cut by these bounds, not by the lengths, so one whose bounds are far above them costs the launch of what they might need
 * (a step of 74 positions 7.3 us at bounds of 64 + 10, 10.8 at 8192 + 2048).  len[s] may be less than shared[g]; such a sequence is read by
 * itself, in as many pieces as max_own is cut into (sixteen over 65537 positions, one of them a position shorter: 1009 us at a max_own of 33, 317 at 1024, 157 at
 * 65537, where all behind them take 91, 90 and 103).  A sequence of length 0 gets zeros; so does one whose lengths are out of these bounds
 * (*err is set).  A position on a page out of range does not count (*err is set).  Keys and values that count have to be finite for a finite result.  Nothing behind a sequence's last position gets into its result,
 * whatever it holds. */
size_t spd_op_attention_shared_scratch_bytes(int32_t n_seq, int32_t width, int32_t n_heads, int32_t n_kv_heads, int32_t d_head, int32_t max_shared,
                                             int32_t max_own);
int spd_op_attention_shared(int32_t dtype, const float *q, const void *K, const void *V, const int32_t *table, int32_t n_pages, int32_t n_kv_heads,
                            int32_t page_size, int32_t d_head, int32_t n_seq, int32_t table_stride, const int32_t *shared, const int32_t *len,
                            int32_t width, int32_t n_heads, int32_t max_shared, int32_t max_own, float *out, void *scratch, size_t scratch_bytes,
                            int32_t *err, void *hip_stream);

/* The n_out best continuations of each group's n_in beams (both 1..SPD_K_MAX; n_in 1 at a search's first step): continuation (b, v)
 * scores scores[g][b] + log softmax(logits[g][b] / tau)[v], and the lower b, then the lower v goes first among equals.  (The sum of
 * exponentials is an fp32 sum, which is some 1e-7 in a score: continuations of different beams that are nearer to each other than that may change places.)  logits
 * DEVICE [n_groups n_in rows of row_stride elements] in `dtype` (a logit that is no number counts as -inf, +inf as the largest finite
 * number; -inf is no continuation); scores DEVICE float [n_groups, n_in] (-inf or no number: no such beam).  ended (DEVICE int32
 * [n_groups, n_in], may be NULL): a beam with a value other than 0 has one continuation, itself, with token end_token and its score
 * unchanged; neither its logits nor those of an absent beam count.  Outputs DEVICE [n_groups, n_out], best first: scores, tokens (in
 * [0, vocab)), parents (in [0, n_in)) and, unless NULL, whether the beam has ended (its parent had, or the token is end_token).
 * Where there are fewer continuations, the others have score -inf, token 0, not ended, and as parent their own place (0 where that is no beam).  With
 * n_out = n_in an output may be the buffer of scores or ended. */
size_t spd_op_beam_select_scratch_bytes(int32_t n_groups, int32_t n_in, int32_t n_out, int32_t vocab);
int spd_op_beam_select(int32_t dtype, const void *logits, int64_t row_stride, int32_t n_groups, int32_t n_in, int32_t n_out, int32_t vocab,
                       const float *scores, const int32_t *ended, int32_t end_token, float tau, float *out_scores, int32_t *out_tokens,
                       int32_t *out_parents, int32_t *out_ended, void *scratch, size_t scratch_bytes, void *hip_stream);

/* The cache follows a selection: beam j of group g goes on from beam parents[g][j] (DEVICE int32 [n_seq / width, width], width <=
 * SPD_K_MAX).  len DEVICE int32 [n_seq]: positions cached so far, the same for all beams of a group; entry e = len / page_size of a
 * row is the page being filled, which like those behind it must be the row's own.  A row's first child keeps the whole row; each
 * further child, in order, takes its parent's entries before e and, from e on, those of a row without a child (in order), into
 * whose page e the rows filled so far are copied in all n_layers (layer l's pools start l * layer_stride elements after K and V).  So
 * every beam has pages of its own to write into and none has to be found.  table_out [n_seq, table_stride] is a table of its own.
 * A group with a parent outside [0, width), unequal lengths or, where a page is to be copied, a row whose page e is out of range or page e of another
 * row of the group too is left as it was (its table copied unchanged) and *err is set.  That is all that is looked at: pages that are not a row's own in
 * other ways (an entry of another group, or another entry of the same) are overwritten.
 * Any row may come first afterwards.  So every row has to hold all positions up to len itself: also those that spd_op_attention_shared reads through a group's first
 * row, whole pages of them by number, and on the page where they end, which is the row's own, as copies. */
int spd_op_beam_reorder(int32_t dtype, void *K, void *V, const int32_t *table, int32_t n_pages, int32_t n_kv_heads, int32_t page_size,
                        int32_t d_head, int32_t n_seq, int32_t table_stride, int32_t n_layers, int64_t layer_stride, int32_t width,
                        const int32_t *parents, const int32_t *len, int32_t *table_out, int32_t *err, void *hip_stream);

/* The same where only a group's first row has to hold its shared positions (shared DEVICE int32 [n_seq / width], as for spd_op_attention_shared; those behind len do not
 * count): all rows get its entries of whole pages of them, and where the first beam goes on from another row, the shared positions on the page where
 * they end are copied to that row's page.  A group whose shared[g] is out of range, or one of these two pages where there is something to copy, is left as it was and *err is set. */
int spd_op_beam_reorder_shared(int32_t dtype, void *K, void *V, const int32_t *table, int32_t n_pages, int32_t n_kv_heads, int32_t page_size,
                               int32_t d_head, int32_t n_seq, int32_t table_stride, int32_t n_layers, int64_t layer_stride, int32_t width,
                               const int32_t *parents, const int32_t *len, const int32_t *shared, int32_t *table_out, int32_t *err, void *hip_stream);

/* ---- chunks of new tokens: prompts and drafted tokens through a paged cache ----
 * A step of a program that runs a model's products itself feeds sequence s the new tokens first[s] .. first[s + 1] - 1 of a call's n_tokens (first DEVICE
 * int32 [n_seq + 1], ascending): a piece of its prompt, one token, or its newest token and drafts of the next ones (those that Superposed Decoding keeps, for
 * one).  Their keys and values go into the cache, their queries attend over it, and of drafts it is found out which stand.  The cache is the paged one of
 * the operators above, with their conventions (device-side lengths, *err, scratch, overlaps, nothing synchronised or allocated), and may also hold 8 bits per value:
 *   K, V              DEVICE int8 [n_pages, n_kv_heads, page_size, d_head], SPD_DTYPE_INT8;
 *   K_scale, V_scale  DEVICE float [n_pages, n_kv_heads, page_size], 16-byte aligned: a value is its code times its row's scale.
 * Both are NULL for the other types.  (spd_op_append_paged, spd_op_attention_shared and spd_op_beam_reorder take no 8-bit cache.) */

/* spd_op_append_paged into a cache of 8 bits: scale = fp32(max |x| / 127) over the d_head values x of a row, rotated where they are keys, and code = x / scale rounded
 * to the nearest whole number, to even between two; rotation, scale and code are formed in 64 bits.  A row of zeros has scale 0.  A k or v that is no number counts as 0, an
 * infinite one as the largest finite number. */
int spd_op_append_paged_q8(int8_t *K, int8_t *V, float *K_scale, float *V_scale, const int32_t *table, int32_t n_pages, int32_t n_kv_heads, int32_t page_size,
                           int32_t d_head, int32_t n_seq, int32_t table_stride, const float *q, int64_t q_stride, const float *k, const float *v, int64_t kv_stride,
                           const int32_t *seq, const int32_t *pos, int32_t n_tokens, int32_t n_heads, float rope_theta, float *q_out, int32_t *err, void *hip_stream);

/* Cached rows back: k_out, v_out [n_tokens, n_kv_heads, d_head] in `out_dtype` (fp32, fp16 or bf16), 16-byte aligned, get the keys (as cached: rotated) and values at
 * position pos[i] of sequence seq[i] of a cache in `dtype` (fp32, fp16, bf16 or int8: code x scale in fp32), rounded to nearest.  seq[i] < 0: padding, the row is left as it was; so is one whose position or
 * page is out of range (*err is set).  The same position may be named more than once. */
int spd_op_read_paged(int32_t dtype, const void *K, const void *V, const float *K_scale, const float *V_scale, const int32_t *table, int32_t n_pages, int32_t n_kv_heads,
                      int32_t page_size, int32_t d_head, int32_t n_seq, int32_t table_stride, const int32_t *seq, const int32_t *pos, int32_t n_tokens, int32_t out_dtype,
                      void *k_out, void *v_out, int32_t *err, void *hip_stream);

/* Causal attention of the new tokens: len[s] (DEVICE int32 [n_seq]) positions of sequence s are cached, its n new ones, appended before, among them.  The query of its j-th new token sits at
 * position p = len[s] - n + j: out[t][h] = softmax(q[t][h] . K / sqrt(d_head)) V over positions 0 .. p.  Cache in `dtype` (fp32, fp16, bf16 or int8).  q rows [n_heads,
 * d_head] at q + t q_stride (elements; a multiple of 8) and out [n_tokens, n_heads, d_head] in `io_dtype`: fp32, or the cache's own type, or with an int8 cache
 * fp16 or bf16.  In fp32 queries and probabilities go into the products with 24 bits, in 16 bits with those of the type.  max_len >= every len[s] (a host
 * value; no more than a row of the table holds) and max_new, the most new tokens of a sequence, size the launch: a sequence with more of them is taken as well, only slower.
 * A sequence whose first and len do not fit (first negative or past n_tokens, len below its new tokens or over max_len) gets zeros for the rows that it has; where first descends anywhere no row
 * is written; *err is set, also for a sequence that has no row (no new tokens, or all of them outside of 0 .. n_tokens - 1).  Rows that are no sequence's are left as they were.  (Without tokens, n_tokens 0, nothing is looked at.)  n_seq is at most 65536, n_tokens n_heads at most 2^24.  A position on a page out of range does not count (*err is set).  Keys and values that count have to be finite for a finite result; nothing behind a
 * sequence's last position, or behind a token's own, gets into its result.  (Of an 8-bit cache, values whose
 * scale lies more than 2^64 below the largest one in front of them or at the next 64 positions may count as zero.) */
size_t spd_op_attention_paged_scratch_bytes(int32_t dtype, int32_t io_dtype, int32_t n_seq, int32_t n_tokens, int32_t n_heads, int32_t n_kv_heads, int32_t d_head,
                                            int32_t max_new, int32_t max_len);
int spd_op_attention_paged(int32_t dtype, int32_t io_dtype, const void *q, int64_t q_stride, const void *K, const void *V, const float *K_scale, const float *V_scale,
                           const int32_t *table, int32_t n_pages, int32_t n_kv_heads, int32_t page_size, int32_t d_head, int32_t n_seq, int32_t table_stride, const int32_t *first,
                           const int32_t *len, int32_t n_tokens, int32_t n_heads, int32_t max_new, int32_t max_len, void *out, void *scratch, size_t scratch_bytes,
                           int32_t *err, void *hip_stream);

/* Which drafted tokens stand.  tokens (DEVICE int32 [n_tokens]): of sequence s its newest token, at first[s], then its m = first[s + 1] - first[s] - 1 >= 0 drafts.  Row t of logits
 * (DEVICE, `dtype` fp32, fp16 or bf16, rows of row_stride elements) is what the target model expects behind token t, p = softmax(logits / tau); row t of draft_logits (draft_stride) what
 * the drafter drew token t + 1 from, q = softmax(draft_logits / draft_tau), not looked at for a sequence's last token.  draft_logits NULL: drafts that were chosen, not drawn, q
 * is 1 at the draft.  u (DEVICE float [n_tokens], in [0, 1), the caller's draws): draft x behind token t stands if all before it do and u[t] < p(x) / q(x), however small the two are (a
 * quotient below 2^-990 may count as 0; with p(x) = 0 it does not stand, with q(x) = 0 < p(x) it does); so a text has the target's distribution whatever the drafter's is.  Behind the drafts
 * that stand comes one token more, drawn with u at the sequence's last token: from p where all stand, else from max(p - q, 0), formed in 64 bits, at the first that does not (from p where that is zero
 * everywhere): the first token, in the order of ids, up to which more than u of the sum has gone by.  Tokens below 2^-1021 of the likeliest one's probability have none there, so one that is
 * masked with a large negative number is not drawn, with a u of 0 neither.  What is drawn, and whether a draft stands, goes by sums of 64
 * bits (of 32 where those could not turn it); the log p of a draft by sums of 32, off by less than 2^-15 of itself.  tau and draft_tau, in 64 bits (the draw falls between as many borders as there are tokens, and a temperature rounded to 32 bits moves one in two
 * thousand draws over 131072 logits to another token), lie between 2^-100 and 2^100; n_seq is at most 65536.
 * A logit that is no number counts as -inf, +inf as the largest finite number.  A draft outside [0, vocab) does not stand; *err is set.
 * Outputs, DEVICE: out_accepted int32 [n_seq], the number a of drafts that stand; at first[s] .. first[s] + a of out_tokens int32 [n_tokens] those drafts and the token
 * behind them, and of out_logprobs float [n_tokens] their log p; -1 and 0 at the sequence's other tokens.  A row without a finite logit gives token 0 with log p = -inf, *err is set.  A
 * sequence without tokens, or whose first is negative or past n_tokens, has a = 0 and nothing else written (*err is set in the second case); so have all where first descends anywhere.  Rows that
 * are no sequence's are left as they were. */
size_t spd_op_verify_drafts_scratch_bytes(int32_t n_seq, int32_t n_tokens, int32_t vocab);
int spd_op_verify_drafts(int32_t dtype, const void *logits, int64_t row_stride, const void *draft_logits, int64_t draft_stride, const int32_t *tokens, const int32_t *first,
                         const float *u, int32_t n_seq, int32_t n_tokens, int32_t vocab, double tau, double draft_tau, int32_t *out_tokens, float *out_logprobs,
                         int32_t *out_accepted, void *scratch, size_t scratch_bytes, int32_t *err, void *hip_stream);

/* ---- test hooks for the error path of the persistent kernel's bounded waits ----
 * A wait of the persistent forward kernel that gives up (its grid was not co-resident) sets an
 * error word in the device-side draft state; every entry point that copies that state back
 * (spd_step, spd_generate, spd_commit, spd_nucleus_step, spd_get_state, spd_get_step_info,
 * spd_get_nucleus_info) then returns SPD_EHIP.  spd_test_state_layout gives the size of that
 * state in 32-bit words and the index of the error word; spd_test_state_status applies the
 * library's check to a HOST copy of the state filled by the caller (host only, no GPU);
 * spd_test_poke_err writes the device-side error word (a fill kernel on the ctx's stream, no
 * synchronisation) so that the getters' mapping can be seen without any wait ever failing:
 * spd_prefill clears it again. */
int spd_test_state_layout(size_t *out_words, size_t *out_err_word);
int spd_test_state_status(const int32_t *state_words, size_t n_words);
int spd_test_poke_err(spd_ctx *ctx, int32_t value);

/* ---- test hook of the n-gram tables ----
 * What spd_load_ngrams would copy to the device (host only, no GPU): the slots, 32 bytes each, into HOST memory of at least
 * spd_ngram_table_bytes() bytes, and the longest displacement of an entry from its home slot. */
int spd_test_ngram_table(const spd_ngram_host_tables *t, int32_t vocab, void *out_slots, size_t out_bytes, int32_t *out_max_probe);

/* ---- test hooks of the dense prefix pass ----
 * How a product (0: QKV, 1: attention output, 2: gate and up, 3: down) of a chunk of n_tokens is cut up on a GPU of num_cu
 * compute units (host only, no GPU): out[4] = tokens and columns of a tile, blocks that share a tile's k range, 1 where the
 * product runs its epilogue itself.  SPD_EINVAL for models without a dense pass. */
int spd_test_prefill_cut(const spd_model_cfg *cfg, int32_t num_cu, int32_t n_tokens, int32_t product, int32_t *out);
/* From now on this context cuts `product` with the tile shape `tile` (0 .. 6, for gate and up 0 .. 13; -1: by estimate again) and `splits` blocks per k
 * range, wherever partial sums of that size have room; out[4] as above, for a chunk of n_tokens. */
int spd_test_force_prefill_cut(spd_ctx *ctx, int32_t product, int32_t tile, int32_t splits, int32_t n_tokens, int32_t *out);
/* From now on this context's dense pass takes the last layer's query rows with the key and value rows (mode 1), in a product of their own for
 * the last token (2), or as measured (0); *out_own: whether a chunk of n_tokens has that product. */
int spd_test_force_last_query(spd_ctx *ctx, int32_t mode, int32_t n_tokens, int32_t *out_own);
/* The chunk's causal attention alone: DEVICE float queries [n_tokens, n_heads, d_head] at positions pos .., DEVICE cache
 * [n_kv_heads, cap_ctx, d_head] (fp32 or fp16) filled up to them, result [n_tokens, n_heads, d_head] as the sum of two bf16
 * numbers (DEVICE); everything 16-byte aligned, d_head a power of two from 8 to 128, n_tokens <= 1024. */
int spd_test_prefill_attention(int32_t kv_dtype, const float *q, const void *K, const void *V, uint16_t *out_hi, uint16_t *out_lo,
                               int32_t n_tokens, int32_t pos, int32_t n_heads, int32_t n_kv_heads, int32_t d_head, int32_t cap_ctx,
                               void *hip_stream);

/* ---- test hook of the attention over a paged cache ----
 * How spd_op_attention_shared cuts a call (host only, no GPU): out[7] = chunks of the shared positions, positions of one, chunks of each sequence's own, query rows of a
 * shared block, shared blocks in all, and where such a block's waves share out rows, keys of a stage and the stages that it holds (0, 0 elsewhere). */
int spd_test_attention_shared_cut(int32_t dtype, int32_t n_seq, int32_t width, int32_t n_heads, int32_t n_kv_heads, int32_t d_head, int32_t max_shared, int32_t max_own,
                                  int32_t *out);

/* ---- test hook of the selection ----
 * How spd_op_beam_select cuts a call (host only, no GPU): out[2] = logits per lane of a slice (0: one launch, no slices) and slices of a row. */
int spd_test_beam_select_cut(int32_t n_groups, int32_t n_in, int32_t n_out, int32_t vocab, int32_t *out);

const char *spd_last_error(const spd_ctx *ctx);
const char *spd_strerror(int status);

#ifdef __cplusplus
}
#endif
#endif /* SPD_H */
