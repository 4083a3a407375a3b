/*
 * sdlm.h - C ABI of the MI355X (gfx950) block-decode library for SDLM's Next
 * Sequence Prediction inference ("Sequential Diffusion Language Models").
 *
 * The library computes, entirely in hand-written HIP kernels, one decode step of
 * Longest Prefix Decoding (Sec. 3.2 and 3.4 of the paper):
 *
 *   - the block input X_T = [x_last, [m] x (D-1)] is appended after the cached
 *     prefix (block definition below the training objective, Sec. 3.2; Fig. 2(b));
 *   - a dense Qwen-2.5-shaped decoder (Sec. 4.1) runs on the block rows, which
 *     attend causally to the cache and bidirectionally inside the block (the
 *     attention-mask equation of Sec. 3.3, its operator read as OR);
 *   - per block position the arg-max token and its confidence are computed:
 *     softmax probability of the decoded token (Sec. 3.4 item (1)) or one minus
 *     the normalised entropy (Sec. 3.4 item (2));
 *   - gamma_tau = max({ j in 1..D : prod_{k<=j} p_k >= tau } U {1}) tokens are
 *     accepted (the gamma_tau equation, Sec. 3.4) and Decode() takes exactly those
 *     (the Decode equation, Sec. 3.2);
 *   - the cache only ever receives K/V of real, accepted tokens computed under
 *     causal attention: the tokens accepted in step t are fed in step t+1 as
 *     "pending" causal rows whose K/V land directly in their cache slots, next
 *     to the D block rows whose K/V are used inside the step and then dropped.
 *     This keeps the step a function of the token history alone (Sec. 3.2).
 *
 * Conventions
 *   Pointers marked [dev] are device (HBM) addresses, [host] are host addresses.
 *   The caller owns every buffer it passes in; the library allocates nothing on
 *   the device: all of its memory is the single workspace handed to sdlm_create.
 *   All work is enqueued on the HIP stream given to sdlm_create; outputs are
 *   valid once the caller has synchronised that stream.  Unless noted, calls do
 *   not synchronise.  Every call returns 0 on success or a negative sdlm_status;
 *   nothing throws or aborts across this boundary; sdlm_last_error() gives text.
 *   A context is not thread-safe.
 */
#ifndef SDLM_H
#define SDLM_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct sdlm_ctx sdlm_ctx; /* opaque */

typedef enum {
    SDLM_OK = 0,
    SDLM_EINVAL = -1,    /* bad argument or unsupported shape */
    SDLM_ECAPACITY = -2, /* sequence would outgrow max_seq_len, page pool or workspace too small */
    SDLM_ESTATE = -3,    /* call out of order (commit without step, step without prefill, ...) */
    SDLM_EHIP = -4       /* a HIP runtime call failed */
} sdlm_status;

/* Shape of the decoder (Qwen-2.5 family: pre-norm RMSNorm, rotate-half RoPE, GQA, SwiGLU, untied LM head). */
typedef struct {
    int32_t n_layers, hidden, n_q_heads, n_kv_heads, head_dim, ffn, vocab;
    float rope_theta, rms_eps;
    float logit_scale;     /* logits = logit_scale * (x_hat . W_lm[v]) */
    int32_t dtype;         /* 0: fp32 weights, cache and arithmetic (debug / tiny); 1: bf16 weights and cache,
                              bf16 matrix-core inputs, fp32 accumulation, fp32 residual stream and softmax */
    int32_t mask_token_id; /* the id of [m]; its embedding is an ordinary row of the table */
    int32_t has_qkv_bias;
    int32_t block_causal;  /* 0: full mutual attention inside the block (the method, Sec. 3.3); 1: the ablation of
                              Sec. 4.4 "Causal Attention": block row k sees the block rows up to itself only */
} sdlm_model_cfg;

typedef struct {
    int32_t max_batch;   /* sequences decoded together, >= 1 */
    int32_t max_seq_len; /* most known tokens a sequence may reach; a step needs n_b + D <= max_seq_len, so that
                            accepting all D tokens still fits */
    int32_t block_D;     /* D: block size, 1..16 */
    int32_t kv_layout;   /* 0: contiguous (each sequence owns a fixed run of 16-token tiles sized for
                            max_seq_len); 1: paged (tiles handed out from a shared pool on demand) */
    int32_t page_size;   /* tokens per page; must be 16 */
    int32_t n_pages;     /* paged only: pages in the pool (per layer) */
    float tau;           /* acceptance threshold of gamma_tau */
    int32_t conf_fn;     /* 0: logit-value confidence; 1: entropy-normalised confidence */
    int32_t accept_rule; /* 0: cumulative product >= tau (the paper's rule); 1: each leading confidence >= tau */
    int32_t prefill_rows; /* rows per prefill pass (0: library default) */
} sdlm_run_cfg;

/*
 * Source weights, every matrix [out_features, in_features] row-major with in_features contiguous, element
 * type given by sdlm_model_cfg.dtype.  Per-layer entries are arrays of n_layers pointers.  A NULL entry in a
 * per-layer array (or a NULL global) leaves that tensor's packed copy untouched, so weights may be streamed in
 * over several calls.
 */
typedef struct {
    const void *embed, *lm_head, *final_norm; /* [V,h] [V,h] [h] */
    const void *const *attn_norm;             /* [h] */
    const void *const *wq, *const *wk, *const *wv; /* [Hq*d,h] [Hkv*d,h] [Hkv*d,h] */
    const void *const *wo;                    /* [h,Hq*d] */
    const void *const *bq, *const *bk, *const *bv; /* [Hq*d] [Hkv*d] [Hkv*d]; ignored unless has_qkv_bias */
    const void *const *ffn_norm;              /* [h] */
    const void *const *w_gate, *const *w_up;  /* [F,h] */
    const void *const *w_down;                /* [h,F] */
} sdlm_weights;

/* Bytes of device workspace a context with these settings needs (0 on invalid settings). */
size_t sdlm_workspace_bytes(const sdlm_model_cfg *m, const sdlm_run_cfg *r);

/*
 * Create a context inside `workspace` [dev] (256-byte aligned, at least sdlm_workspace_bytes()).  `hip_stream`
 * is a hipStream_t (NULL: the default stream).  Synchronises the stream once (tables are uploaded).
 * Errors: SDLM_EINVAL (shape not supported: head_dim not a multiple of 32 or > 256, n_q_heads not a multiple
 * of n_kv_heads, block_D outside 1..16, page_size != 16, ...), SDLM_ECAPACITY (workspace too small).
 */
int sdlm_create(const sdlm_model_cfg *m, const sdlm_run_cfg *r, void *workspace, size_t workspace_bytes,
                void *hip_stream, sdlm_ctx **out);

/*
 * Copy and repack weights into the workspace (matrix-core tile order for bf16).  The sources may be freed once
 * the stream has been synchronised.  on_device != 0: the pointers inside `w` are [dev]; 0: they are [host]
 * (staged through pageable copies; this synchronises).  `w` itself and its pointer arrays are [host].
 */
int sdlm_init_weights(sdlm_ctx *ctx, const sdlm_weights *w, int32_t on_device);

/*
 * Start `batch` sequences (1..max_batch) from their prompts and fill the cache with a causal forward over
 * each prompt (no block rows, no LM head).  ids_packed [host]: all prompts back to back; offsets [host]:
 * batch+1 entries, prompt b is ids_packed[offsets[b] .. offsets[b+1]).  Every prompt needs >= 1 token and
 * len + D <= max_seq_len.  Discards all earlier sequences.  Afterwards n_b = c_b = len_b.
 */
int sdlm_prefill(sdlm_ctx *ctx, int32_t batch, const int32_t *ids_packed, const int32_t *offsets);

/*
 * One block-decode step for every sequence.  Outputs, all [dev]:
 *   ids    [batch, D]  int32  arg-max token of each block position (lowest index on exact ties); the first
 *                             count[b] entries of row b are the accepted tokens (Decode), the rest are the
 *                             predictions that were not accepted;
 *   count  [batch]     int32  gamma_tau, 1..D;
 *   conf   [batch, D]  float  confidence per block position (may be NULL);
 *   logits [batch*D,V] float  the logits Z (may be NULL; costs a batch*D*V write).
 * The step publishes nothing: K/V of the pending tokens are written into cache slots that stay invisible
 * until sdlm_kv_commit, and the block rows' K/V live in per-step staging.  It may therefore be repeated, with the same bits.
 * Sequences are independent, but which kernels a step takes depends on its rows (sdlm_debug_step_plan): a sequence's results in
 * another batch may differ by the order of fp32 sums and, in bf16, by what that changes in the roundings of operands.  On the generic
 * path they are the same bits while both batches' steps take the same form (the line is at most at batch x 2D = 32 rows, and again
 * where the products of many rows begin).
 * Errors: SDLM_ESTATE before prefill; SDLM_ECAPACITY if n_b + D > max_seq_len for some sequence, i.e. if accepting
 * all D tokens would not fit (the host tracks an upper bound of each length and refreshes it with a stream
 * synchronisation only when the bound trips; the same refresh reports a page pool that ran out at the last commit).
 */
int sdlm_decode_step(sdlm_ctx *ctx, int32_t *ids, int32_t *count, float *conf, float *logits);

/*
 * sdlm_decode_step for callers that cannot allocate device memory for the step's partial results: code under HIP
 * graph capture, tight serving loops, harnesses that forbid hipMalloc.  Same arguments, outputs and errors as
 * sdlm_decode_step; the partial-result scratch of the step's kernels (split-k slabs of the projections, split-KV
 * partial results of the attention, per-vocabulary-block partials of the LM head; in fp32 mode the logits when
 * `logits` is NULL) lives in a 32 MiB array that is part of the library's code object instead of the workspace:
 * 16 MiB of slabs, 12 MiB of attention partials (both only bound how far the work is split, so a large model runs
 * with fewer splits) and 4 MiB for the LM head, which must hold batch x D rows: otherwise SDLM_ECAPACITY.  Calls
 * no hipMalloc / hipFree and creates no events or graphs (phase timing and graph replay do not apply to it).
 * Every GPU the library runs on holds one copy of the array until the process ends, and every context on that GPU
 * shares it: calls that overlap on one GPU (other streams, other contexts) race; calls in stream order do not, and
 * nothing in the array needs to start at zero (every partial result is written before it is read).  The device
 * current at sdlm_create is the one whose copy is used.  SDLM_EHIP if the array's address could not be obtained.
 * A step (this or sdlm_decode_step) that the caller records into a graph of its own is launched for the capacity, not for the
 * present lengths, and may be replayed at any of them, also behind another sdlm_prefill of the same batch.
 */
int sdlm_decode_step_static(sdlm_ctx *ctx, int32_t *ids, int32_t *count, float *conf, float *logits);

/*
 * Replay the decode step as a HIP graph.  The launch sequence of sdlm_decode_step is fixed once the batch is known
 * (row counts, lengths and page tables live in device memory), except that the attention of short and of long contexts is
 * launched differently.  With enable != 0 the first sdlm_decode_step after a prefill, after its first commit, after the output
 * pointers change, or when the longest sequence passes such a line (at 256 keys and where the merge of the split cache
 * changes: a few times in a generation) captures its launches on the context's stream and later calls replay the captured graph: one submission instead of ~9 launches per layer, which is what bounds the step for small
 * batches.  Results are identical to the eager path.  The step runs eagerly regardless while any phase is being
 * timed (sdlm_profile) or a debug tap is set.  sdlm_verify_step and sdlm_kv_commit are always eager.
 * Errors: SDLM_ESTATE if the context was created on the null stream (which cannot be captured).
 */
int sdlm_graph(sdlm_ctx *ctx, int32_t enable);

/*
 * Second pass of a self-speculative step (Sec. 3.4, "Self-Speculative Decoding", Eq. 10); call it between
 * sdlm_decode_step, whose D arg-max tokens are the speculative tokens yhat^1..yhat^D, and sdlm_kv_commit.
 * Verification input j (j = 2..D) is the sequence extended by yhat^1..yhat^{j-1} followed by the mask tokens, i.e.
 * the input of an ordinary block step on that longer sequence; ytilde^j is the token that step would predict first
 * (input 1 is the first pass itself, so ytilde^1 = yhat^1).  All D-1 inputs of all sequences run as one batch of
 * rows through the same kernels as the step; they read the cache and write nothing to it.
 *   rule       0: gamma_verify = length of the longest prefix on which yhat and ytilde agree (at least 1);
 *              1: the equation as printed: the largest j with yhat^j == ytilde^j (at least 1).
 *   ids_tilde  [dev, batch x D] ytilde, or NULL.
 *   count      [dev, batch] gamma_verify, or NULL.  It also replaces the step's own count, so that a commit
 *              without overrides publishes yhat^1..yhat^{gamma_verify}.
 *   logits     [dev, batch x (D-1) x vocab] fp32 logits from which ytilde^2..ytilde^D were taken, or NULL.
 * Asynchronous on the context's stream.  Errors: SDLM_ESTATE without a preceding step, SDLM_EINVAL for an unknown
 * rule.  Every block size 1..16 is served; a sequence contributes (D-2) + (D-1) D rows to the pass (the causal rows
 * of the speculative tokens are shared by all inputs).
 */
int sdlm_verify_step(sdlm_ctx *ctx, int32_t rule, int32_t *ids_tilde, int32_t *count, float *logits);

/*
 * Publish the last step: the pending tokens' K/V become part of the cache (c_b = n_b) and the accepted tokens
 * become the next step's pending tokens (n_b += count_b); in the paged layout the page table grows to back
 * every position < n_b.  With both arguments NULL the step's own result is committed.  With ids_override
 * [dev, batch x D] and count_override [dev, batch] (1 <= count <= D; out-of-range counts are clamped and
 * reported through sdlm_get_lengths' return code, as are override ids outside the vocabulary, which are replaced by 0) the caller's tokens are committed instead: this is how a
 * verifier or a teacher-forced test drives the cache.  Errors: SDLM_ESTATE without a preceding step.
 */
int sdlm_kv_commit(sdlm_ctx *ctx, const int32_t *ids_override, const int32_t *count_override);

/*
 * Sampled tokens in the place of the arg-max ones: call it between sdlm_decode_step, which wrote `logits` [dev, batch x D x vocab], and sdlm_kv_commit.  Draws a token for every block position
 * (see sdlm_sample; the vectors are over the batch x D positions), and accepts with the drawn tokens' confidences: the logit confidence is a drawn token's softmax
 * probability (temperature 1, nothing filtered), the entropy confidence stays the position's.  A position without any token above -infinity keeps its arg-max token.
 *   ids, count, conf [dev]: as those of the step (conf may be NULL); they replace its result, which a commit without overrides then publishes.
 * May be repeated.  Asynchronous on the context's stream.  sdlm_verify_step behind it verifies the drawn tokens.  Errors: SDLM_ESTATE without a preceding step, SDLM_EINVAL (also for
 * vocabularies above 524288).
 */
typedef struct {
    const float *temperature, *top_p, *min_p; /* [dev, batch x D] or NULL: 1, off, off */
    const int32_t *top_k;                     /* [dev, batch x D] or NULL: off */
    const float *u;                           /* [dev, batch x D] uniform numbers in [0, 1) */
} sdlm_sampling;
int sdlm_sample_step(sdlm_ctx *ctx, const float *logits, const sdlm_sampling *how, int32_t *ids, int32_t *count, float *conf);

/*
 * Continue sequences as several, drop others: sequence b of the new batch becomes what sequence parents[b] is (`parents` [host], batch entries in 0 .. present batch - 1; batch up to
 * max_batch).  Several samples of one prompt are one prefill and one fork; a beam's step is a commit and a fork.  Sequences that are nobody's parent are gone, and their pages free.  In the
 * paged layout full pages are held in common (see sdlm_kv_fork); in the contiguous one a sequence that is no longer alone with its parent takes a free run and a copy of all pages.
 * The last step's result is discarded.  Synchronises the stream; not under graph capture.
 * Errors: SDLM_ESTATE before prefill or under capture, SDLM_EINVAL, SDLM_ECAPACITY (too few free pages: nothing was changed).
 */
int sdlm_fork(sdlm_ctx *ctx, int32_t batch, const int32_t *parents);

/*
 * Verify a tree of drafted tokens for every sequence in one pass; call it behind sdlm_decode_step.  Node i of sequence b is token tokens[b * n_nodes + i] behind node parents[b * n_nodes + i] (< i; -1: behind
 * the known tokens).  A node's prediction is the first token that a block step predicts for the sequence extended by the tokens on the node's branch, the inputs of sdlm_verify_step for every
 * node at once; the root's is the step's own first arg-max token.  Accepted is the branch that agrees with the predictions: from the root on, the child
 * whose token is the prediction (the lowest such node), until there is none.
 *   n_nodes        1 .. 16 D / (D + 1) (D = 1: 1 .. 16); the same for all sequences.  A negative token is no node: fill up with them.
 *   path           [dev, batch x n_nodes] accepted nodes, then -1; or NULL.
 *   count, next    [dev, batch] how many, and the prediction behind the last of them; or NULL.
 *   logits         [dev, batch x n_nodes x vocab] fp32 logits of the nodes' predictions, or NULL.
 * Reads the cache and writes nothing to it; may be repeated.  A token beyond the vocabulary or a parent that is not in front of its node takes the node out, and sdlm_get_lengths reports it.
 * Errors: SDLM_ESTATE without a preceding step, SDLM_EINVAL, SDLM_ECAPACITY if the nodes and a block do not fit behind the longest sequence (n + n_nodes + D > max_seq_len), or
 * batch x n_nodes x (D + 1) rows not into the workspace (sdlm_max_rows; more prefill_rows make room).
 */
int sdlm_verify_tree(sdlm_ctx *ctx, int32_t n_nodes, const int32_t *tokens, const int32_t *parents, int32_t *path, int32_t *count, int32_t *next, float *logits);

/*
 * Publish the accepted branch of the last sdlm_verify_tree, and the prediction behind it: the nodes' K/V are moved into the cache as they are (they were computed under causal attention),
 * so that only that last token is pending (n_b += count + 1, c_b = n_b - 1).  In the place of sdlm_kv_commit, which publishes the step's own tokens instead.
 * Errors: SDLM_ESTATE without a preceding sdlm_verify_tree, SDLM_ECAPACITY if the page pool might not hold n_nodes + 1 more tokens of every sequence.
 */
int sdlm_tree_commit(sdlm_ctx *ctx);

/*
 * Copy the per-sequence lengths to n [dev, batch] and c [dev, batch] (either may be NULL), then synchronise
 * and refresh the host's bounds.  Returns SDLM_ECAPACITY if a device-side guard (page pool exhausted) or
 * SDLM_EINVAL if a clamped override count was seen since the last call.
 */
int sdlm_get_lengths(sdlm_ctx *ctx, int32_t *n, int32_t *c);

/*
 * Debug taps.  The next sdlm_decode_step copies the named intermediate of layer `layer` into dst [dev]:
 *   0: residual stream entering the layer            float [R, hidden]
 *   1: attention output (before the O projection)    elem  [R, Hq*d]
 *   2: SwiGLU activation (input of the down proj.)   elem  [R, ffn]
 *   3: residual stream leaving the layer             float [R, hidden]
 *   4: normalised block rows entering the LM head    elem  [batch*D, hidden]   (layer ignored)
 *   5: rotated queries                               elem  [R, Hq*d]
 *   6: residual stream after the O projection        float [R, hidden]
 * The step's products, attention and results are those of an untapped step.  "elem" is float in fp32 mode and bf16 in bf16 mode.  R is the step's packed row count: per sequence its
 * pending rows then its D block rows.  `which` < 0 clears all taps.  dst must hold max_rows rows.
 */
int sdlm_debug_tap(sdlm_ctx *ctx, int32_t layer, int32_t which, void *dst);

/*
 * Copy the packed row description of the last step: tok, pos, seq, kind [dev, max_rows each] (kind: -1 for a
 * pending row, else the block index 0..D-1) and n_rows [dev, 1].  Any pointer may be NULL.
 */
int sdlm_debug_rows(sdlm_ctx *ctx, int32_t *tok, int32_t *pos, int32_t *seq, int32_t *kind, int32_t *n_rows);

/*
 * Read cached K and V vectors of one (layer, sequence, kv head) for positions [pos0, pos0+count) into
 * k_out, v_out [dev, count x head_dim] as float.  Positions must be < n_b.  pos0 = -1 reads instead the first
 * `count` (<= D) entries of the sequence's staging tile: the K/V of the last step's block rows at that layer.
 */
int sdlm_debug_read_kv(sdlm_ctx *ctx, int32_t layer, int32_t seq, int32_t kv_head, int32_t pos0, int32_t count,
                       float *k_out, float *v_out);

/*
 * Host logic only (no GPU work): the launch shape the bf16 matrix-core GEMM takes for `rows` launch rows of which
 * `min_rows` certainly exist (0: unknown), an [n, k] weight matrix (k a multiple of 64) and an epilogue (0: plain fp32
 * store, 1: residual add, 2: SiLU(gate)*up, 3: LM head).  Outputs: rows and columns of a workgroup's tile and the number
 * of splits along k between workgroups.  Columns count rows of the weight matrix, for epilogue 2 those of gate and up
 * together (n of each).  A tile of 16 rows, or for epilogue 2 of 32 x 64, is a kernel without LDS tiles; for epilogue 2, 64 or
 * 128 rows x 128 columns is a workgroup whose wavefronts take half of k each; 512 columns are eight wavefronts.  Not covered:
 * QKV projections that run together with RoPE and the K/V placement, and decode steps of at most 16 rows, whose kernels hold the norms too.  For tests of the
 * tile policy.  Errors: SDLM_EINVAL.
 */
int sdlm_debug_gemm_plan(int32_t epilogue, int32_t rows, int32_t min_rows, int32_t n, int32_t k, int32_t *tile_rows, int32_t *tile_cols,
                         int32_t *splits);

/*
 * Host logic only (no GPU work): the forms that a decode step of `batch` sequences takes, the longest of them with `longest` known tokens, before
 * (committed = 0) or after the first commit behind a prefill.  plan [host], SDLM_SP_N integers:
 *   CHAIN      the layers: 0 separate kernels; steps of few rows with the norms inside the products: 1 generic path, 2 matrix-core path, 3 the same with
 *              down by whole sums of k;
 *   EMBEDS     the embeddings: 0 a launch of their own, 1 gathered by the row assembly, 2 with the first operands of form 3;
 *   QKV_ROWS   matrix-core path, QKV with rotation and K/V placement in one launch: rows of a block that certainly holds some (0: separate launches);
 *   QKV_REST   ... and of one that may be empty;
 *   LM_HEAD    0 matrix-core kernel, 1 generic product behind a norm, 2 generic product with the norm inside;
 *   LM_ACCEPT  1: vocabulary reduction and acceptance are one launch;
 *   ATTN       matrix-core path: 0 one chunk, 1 chunks as teams of one workgroup, 2 to 5 chunks as workgroups and one of four merges behind them (-1: generic).
 * For tests of the dispatch.  Errors: SDLM_EINVAL.
 */
enum { SDLM_SP_CHAIN = 0, SDLM_SP_EMBEDS, SDLM_SP_QKV_ROWS, SDLM_SP_QKV_REST, SDLM_SP_LM_HEAD, SDLM_SP_LM_ACCEPT, SDLM_SP_ATTN, SDLM_SP_N };
int sdlm_debug_step_plan(const sdlm_model_cfg *m, const sdlm_run_cfg *r, int32_t batch, int32_t committed, int32_t longest, int32_t *plan);

/* Rows the activation buffers are sized for (decode: batch * 2D; prefill pass size). */
int32_t sdlm_max_rows(const sdlm_ctx *ctx);

/*
 * Per-phase GPU time.  sdlm_profile(ctx, mask) makes every later step bracket each phase p whose bit (1 << p) is
 * set in `mask` with HIP events on the context's stream (-1: all phases, 0: none); sdlm_profile_read
 * synchronises, adds up the events recorded since the last read and
 * returns, for phase p in 0..SDLM_N_PHASES-1, total milliseconds in ms[p] and launches in launches[p] ([host]).
 */
enum { SDLM_PH_ROWS = 0, SDLM_PH_NORM, SDLM_PH_QKV, SDLM_PH_ROPE, SDLM_PH_ATTN, SDLM_PH_OPROJ, SDLM_PH_GATEUP,
       SDLM_PH_DOWN, SDLM_PH_LMHEAD, SDLM_PH_ACCEPT, SDLM_PH_ATTN_MERGE /* merge of the split-KV partials */, SDLM_N_PHASES };
int sdlm_profile(sdlm_ctx *ctx, int32_t mask);
/*
 * Sampling: bracket only every n-th launch of a selected phase (n >= 1, default 1), counted per phase from this call
 * on.  An event record between two kernels keeps them from running back to back, so timing every launch of a phase
 * that runs once per layer slows the step it measures; with n coprime to the layer count the samples rotate through
 * the layers.  sdlm_profile_read then reports the sampled launches only.  Errors: SDLM_EINVAL.
 */
int sdlm_profile_every(sdlm_ctx *ctx, int32_t n);
int sdlm_profile_read(sdlm_ctx *ctx, float *ms, int32_t *launches);

/*
 * ---------------------------------------------------------------- Operators on the caller's tensors
 *
 * The same kernels that a context runs on its own state, for programs that keep logits or a cache of their own (or want to work on a
 * context's cache: sdlm_kv_describe).  They take the stream (a hipStream_t; NULL: the default stream) of the device that is current and
 * holds the tensors, allocate nothing, do not synchronise and keep nothing between calls; two calls may run at once if they share no workspace
 * and no output, and each may be captured into a graph.  Return value: 0 or a negative sdlm_status, whose text sdlm_op_error() gives.
 */

/* Text of the last operator call of this thread that failed ([host] string). */
const char *sdlm_op_error(void);

/*
 * Draw one token from each row of logits.
 *
 * The tokens of a row are ordered by logit, equal logits by index (lowest first); NaN counts as -infinity, and tokens at -infinity are never drawn.  With
 * w = exp((z - max z) / temperature) a token is kept while
 *   - it is among the first top_k (top_k <= 0: all), and
 *   - the weight of those before it, as a share of the first top_k together, is below top_p (top_p >= 1 or NaN: all), and
 *   - w >= min_p (min_p <= 0 or NaN: all; above 1: none);
 * the first is always kept.  Drawn is the first kept token, in that order, whose running weight exceeds u times the weight of all kept ones.  A temperature <= 0 (or NaN)
 * draws the first.  Where the largest logit is +infinity, only the tokens with it have weight.  A row without any token above -infinity gives id -1 and probability 0.
 * Weights are held to 2^-45 of the largest, where the whole row counts (no top_k) to 2^-44 of it and 2^-29 of themselves, in integers, equal ones for equal logits: a result does not depend on the launch or on the row's neighbours.  A token whose weight is below that is not drawn.
 */
typedef struct {
    const void *logits;        /* [dev] rows x vocab, element type `dtype` */
    int64_t row_stride;        /* elements between rows, >= vocab */
    int32_t dtype;             /* 0: fp32, 1: bf16 */
    int32_t rows, vocab;       /* rows 0 .. 1048576, vocab 1 .. 524288, rows * ceil((vocab + 7) / 16384) below 2^24 */
    const float *temperature;  /* [dev, rows] or NULL: 1 */
    const int32_t *top_k;      /* [dev, rows] or NULL: off */
    const float *top_p, *min_p;/* [dev, rows] or NULL: off */
    const float *u;            /* [dev, rows] uniform numbers in [0, 1); others are clamped */
    int32_t *ids;              /* [dev, rows] drawn tokens */
    float *prob;               /* [dev, rows] their share of the kept weight, or NULL */
} sdlm_sample_args;
size_t sdlm_sample_workspace_bytes(int32_t rows, int32_t vocab);   /* 0 for sizes outside the limits */
/* workspace [dev]: 256-byte aligned.  Errors: SDLM_EINVAL, SDLM_ECAPACITY (workspace too small), SDLM_EHIP. */
int sdlm_sample(const sdlm_sample_args *args, void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * A paged K/V cache.  `pool` holds tiles of 16 positions of one (layer, kv head): layer l, tile t, kv head h starts at element
 * l * layer_stride + (t * n_kv_heads + h) * 32 * head_dim.  Inside, first K, element i of slot s at (i / 8) * 128 + s * 8 + i % 8; then,
 * from 16 * head_dim on, V at ((i / 16) * 4 + s / 4) * 64 + (i % 16) * 4 + s % 4.  Position p of sequence b is slot p % 16 of tile
 * page_table[b * pages_per_seq + p / 16], in every layer and head.  Tiles 0 .. n_pages-1 are the pages that sequences can hold; a pool may have more tiles, for
 * other uses.  All pointers [dev]; a call reads and writes what its text names, and entries outside their range are never followed.
 */
typedef struct {
    void *pool;                /* 16-byte aligned */
    int64_t layer_stride;      /* elements between layers, a multiple of 8 (fp32: 4) */
    int32_t n_layers, n_tiles; /* n_tiles: tiles in a layer */
    int32_t n_kv_heads, head_dim;   /* head_dim 32, 64, 96 or 128; n_kv_heads up to 65535, with the layers 2^23 */
    int32_t dtype;             /* 0: fp32, 1: bf16 */
    int32_t n_pages;
    int32_t max_seqs, pages_per_seq;   /* up to 2^20, 2^26 */
    int32_t *page_table;       /* max_seqs x pages_per_seq; -1: no page */
    int32_t *lengths;          /* max_seqs: positions that hold K/V */
    int32_t *backed;           /* max_seqs: pages that the sequence holds */
    int32_t *page_refs;        /* n_pages: sequences that hold the page (0: free) */
    int32_t *free_pages;       /* n_pages: the free pages in ascending order, then -1 */
    int32_t *free_count;       /* 1 */
} sdlm_kv;

/* The cache of a context, to work on it with the operators below in the stream order of the context: lengths are its c.  The memory stays the context's; its
 * pages too, which its own calls hand out: n_pages is 0 and what sdlm_kv_fork needs is NULL, so that it refuses the cache (a context is forked by sdlm_fork). */
int sdlm_kv_describe(sdlm_ctx *ctx, sdlm_kv *kv);

/*
 * Attention of a tree of drafted tokens for each of n_seqs sequences over the cache.  Rows node_offsets[b] .. node_offsets[b+1]-1 of q and out are the nodes of sequence b
 * (at most max_nodes; further rows are left alone).  Node i of b sees the positions 0 .. lengths[b]-1 of the cache and those nodes j of b whose bit (word j / 64, bit j % 64) is set in row
 * node_offsets[b] + i of `mask`; a tree of drafts sets the node's own bit and its ancestors', but any mask will do.  K/V of node j are at position node_base[b] + j
 * of the table node_table (n_seqs x node_pages entries): the sequence's own table with node_base = lengths, where nodes are appended behind the cache, or pages of their own.
 *   out[r, h] = sum_j softmax_j(q[r, h] . K[j] / sqrt(head_dim)) V[j]; zeros for a node that sees nothing, or scores of -infinity only.
 * Query head h reads kv head h / (n_q_heads / n_kv_heads).  bf16: the softmax's weights keep 2^-16 of themselves in front of the product with V (two bf16 operands each),
 * sums, maxima and the division are fp32.  K/V that a node does not see may hold anything, NaN too, and changes nothing.  Reads pool, page_table and lengths of `kv`.
 */
typedef struct {
    const void *q;               /* [dev] n_rows x n_q_heads x head_dim, element type of the cache */
    void *out;                   /* [dev] as q; must not overlap it */
    int64_t q_stride, out_stride;/* elements between rows, >= n_q_heads * head_dim, multiples of 16 bytes; both base pointers 16-byte aligned */
    int32_t n_rows, n_seqs;      /* n_rows: rows of q and out in all; n_seqs <= kv->max_seqs */
    int32_t n_q_heads;           /* a multiple of n_kv_heads */
    int32_t max_nodes;           /* 1 .. 1024: most nodes of a sequence */
    int32_t max_len;             /* most positions of the cache a sequence has; 0: what the table can hold.  Steers the launch (fp32: and so the order of sums); longer ones are still read whole */
    const int32_t *node_offsets; /* [dev, n_seqs + 1] ascending, 0 .. n_rows */
    const int64_t *mask;         /* [dev] n_rows x mask_words */
    int32_t mask_words;          /* >= (max_nodes + 63) / 64 */
    int32_t node_pages;          /* entries of node_table a sequence */
    const int32_t *node_table;   /* [dev] */
    const int32_t *node_base;    /* [dev, n_seqs] or NULL: 0 */
} sdlm_tree_args;
size_t sdlm_tree_attention_workspace_bytes(const sdlm_kv *kv, int32_t n_q_heads, int32_t n_seqs, int32_t max_nodes, int32_t max_len);
int sdlm_tree_attention(const sdlm_kv *kv, int32_t layer, const sdlm_tree_args *args, void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * Make n_new sequences out of the cache's present ones: sequence b becomes what sequence parent[b] is now (-1: an empty one), and sequences from n_new on become empty.  A parent may be
 * named many times (samples of one prompt, a beam's survivors) or not at all, which frees it.
 *   share != 0: the first lengths / 16 pages, which are full, are held in common; the others (the one that is being written, and pages backed ahead) are each sequence's own.
 *   share == 0: all pages are.  (Pages that sequences hold in common since an earlier call stay with those that keep them.)
 * Own pages stay with a sequence that is its own parent, or else with the first that has it as its parent; the others take free pages, the lowest first, in the
 * order of sequences and positions, with the contents copied where a page has positions below lengths.  Pages that nobody holds any more are free at once, for this call too.
 * A sequence must not write to positions below the length that it was forked with, and its length must not fall below that while it shares pages.
 * Updates page_table, lengths, backed, page_refs (counted anew from the tables), free_pages, free_count and the copied tiles of `pool`.
 *   status [dev, 1]: 0, or nothing was changed: bit 0: there are not enough free pages; bit 1: a parent, or a page in the table, is out of range.
 */
size_t sdlm_kv_fork_workspace_bytes(const sdlm_kv *kv);
int sdlm_kv_fork(const sdlm_kv *kv, const int32_t *parent, int32_t n_new, int32_t share, int32_t *status, void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * Move the K/V of accepted tree nodes into the cache, in every layer: node path[b * path_stride + i] of sequence b to position lengths[b] + i, for i < path_len[b] (at most max_path).
 * Nodes are found as in sdlm_tree_attention.  A path has to ascend, without repetitions.  The destination's pages must be in the table, and not shared.  Nodes or positions without a page
 * are passed over.  lengths is left as it is: the caller adds path_len when it publishes the tokens, and until then the call may be repeated, unless the nodes stand
 * behind the sequence in its own pages, where it overwrites them.
 */
int sdlm_kv_compact(const sdlm_kv *kv, int32_t n_seqs, const int32_t *path, int32_t path_stride, const int32_t *path_len, int32_t max_path, const int32_t *node_table,
                    int32_t node_pages, const int32_t *node_base, void *hip_stream);

/* Which kernel family serves the GEMMs and the attention: "generic-fp32", "mfma-bf16", ... ([host] string). */
const char *sdlm_kernel_info(const sdlm_ctx *ctx);

const char *sdlm_last_error(const sdlm_ctx *ctx);
void sdlm_destroy(sdlm_ctx *ctx);

#ifdef __cplusplus
}
#endif
#endif /* SDLM_H */
