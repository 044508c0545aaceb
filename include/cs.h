/*
 * cs.h -- C ABI of the MI355X (gfx950) cached N-candidate DiT rollout.
 *
 * The library runs CachedSearch's exploration loop (Alg. 1 of the paper):
 * N candidate latents, one per seed, are integrated through T Euler steps of
 * the flow-matching ODE (Sec. Preliminaries, Eq. euler) with optional
 * classifier-free guidance (Eq. cfg).  At every step and for every candidate
 * and guidance branch, the transformation-vector cache (Sec. Adaptive
 * transformation-vector caching, Eqs. delta, skip, indicator) decides whether
 * the transformer is evaluated or its cached residual reused.  The final
 * latents are scored and ranked; the ranking is compared with the full
 * (uncached) rollouts of the same seeds by Spearman correlation (Sec.
 * Experiments, definitions and protocol).
 *
 * Conventions
 *  - Pointers documented "device" are HIP device pointers; "host" pointers
 *    are ordinary CPU memory.  The caller owns every pointer it passes.
 *  - cs_model_init copies the weights into memory the model owns; the
 *    caller's weight buffer may be freed after the call returns.  A rollout
 *    owns its state and workspace and frees them in cs_rollout_free.
 *  - All device work is enqueued on the HIP stream given at init (void* is a
 *    hipStream_t; NULL = the default stream).  Calls that write host outputs
 *    synchronise that stream before returning.
 *  - Every function returns a cs_status; no exception or abort crosses the
 *    ABI.  On failure, cs_last_error() returns a message (thread-local).
 *    Arguments are validated before any device work is enqueued, so a
 *    CS_E_INVAL/CS_E_STATE return leaves the device untouched.
 *  - Identical inputs give bitwise identical outputs, independent of N and
 *    of which other candidates are evaluated in the same step (no atomics,
 *    fixed reduction orders, the same in every tile shape).
 *  - Latents are float32 [C][F][H][W] per candidate, candidates contiguous.
 *    D = C*F*H*W.  Weights: see cs_model_weight_count.
 */
#ifndef CACHEDSEARCH_CS_H
#define CACHEDSEARCH_CS_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  CS_OK = 0,
  CS_E_INVAL = 1,        /* bad argument (null, out of range, NaN, shape)  */
  CS_E_NOMEM = 2,        /* device or host allocation failed               */
  CS_E_DEVICE = 3,       /* a HIP call failed (message names it)           */
  CS_E_STATE = 4,        /* call out of order (e.g. step k+2 after k)      */
  CS_E_UNSUPPORTED = 5   /* valid but not supported shape/config           */
} cs_status;

typedef enum { CS_BF16 = 0, CS_FP32 = 1 } cs_dtype;

/* Cache modes.  OFF computes every call (recovers the uncached rollout
 * G(c,s)); ADAPTIVE applies the accumulated drift rule with threshold tau;
 * STATIC computes every static_k-th step between warmup and cooldown (the
 * uniform-schedule baseline of Sec. Method, properties paragraph).
 * PAB is attention-output broadcasting, one of the published engines the
 * paper compares (Sec. Ranking preservation across published caching
 * methods, Table tab:baselines): every call runs the transformer, but each
 * block's self- and cross-attention output (after the output projection,
 * before the self-attention gate) is recomputed only every
 * pab_self_range / pab_cross_range steps and reused in between.  Steps
 * 1..k_warm and n_steps-k_cool+1..n_steps recompute both; a step s in
 * between recomputes a branch of range r iff (s - k_warm) % r == 0 or
 * nothing is stored yet.  PAB keeps two [n_blocks][N*B][tokens][hidden]
 * arrays of the compute type on the device. */
typedef enum {
  CS_CACHE_OFF = 0, CS_CACHE_ADAPTIVE = 1, CS_CACHE_STATIC = 2, CS_CACHE_PAB = 3
} cs_cache_mode;

/* Transformer shape.  The paper treats the velocity model v_theta(x, t, c)
 * as a black box (Sec. Preliminaries); the library implements a Wan-shaped
 * DiT: 1x2x2 patch embedding, n_blocks of [adaLN self-attention with
 * RMSNorm q/k and 3D RoPE, cross-attention to the text embedding,
 * adaLN tanh-GELU FFN], adaLN head.  Requirements: hidden = heads*head_dim,
 * head_dim in {32, 64, 128}, hidden % 64 == 0, ffn % 64 == 0,
 * text_dim % 64 == 0, in_ch % 16 == 0, freq_dim == 256, patch = (1,2,2),
 * lat_h and lat_w even.  dtype selects the transformer's matrix arithmetic (bf16 operands
 * with fp32 accumulation, or fp32 throughout); the cache state, latents,
 * residual stream and all reductions are fp32/fp64 in both modes. */
typedef struct {
  int32_t n_blocks, hidden, heads, head_dim, ffn;
  int32_t text_dim, text_len, freq_dim;
  int32_t in_ch, lat_f, lat_h, lat_w;
  int32_t patch_t, patch_h, patch_w;
  int32_t dtype;                 /* cs_dtype */
} cs_model_desc;

/* Rollout description (Alg. 1 inputs: seeds via x1, tau, mode).
 * n_branch: 1 = conditional only, 2 = CFG with guidance scale `guidance`
 * (branch 0 conditional, branch 1 unconditional).  Steps are 1-based; steps
 * 1..k_warm and n_steps-k_cool+1..n_steps always compute, as does any call
 * before the branch's first Delta exists.  tau >= 0, +INF allowed.
 * timesteps: host, n_steps+1 floats, timesteps[0] = 1 > ... >
 * timesteps[n_steps] = 0, strictly decreasing (copied at init). */
typedef struct {
  int32_t n_cand, n_steps, n_branch, k_warm, k_cool, static_k;
  int32_t mode;                  /* cs_cache_mode */
  float tau, guidance;
  const float* timesteps;
  int32_t pab_self_range;        /* >= 1, read in CS_CACHE_PAB mode only  */
  int32_t pab_cross_range;       /* >= 1, read in CS_CACHE_PAB mode only  */
} cs_rollout_desc;

typedef struct cs_model cs_model;
typedef struct cs_rollout cs_rollout;

/* Per-rollout counters, read by cs_rollout_stats. */
typedef struct {
  int32_t steps_done;            /* last completed step (0 after init)     */
  int64_t calls;                 /* transformer calls requested (N*B*steps)*/
  int64_t computed;              /* calls evaluated by the transformer     */
  int64_t self_reused;           /* PAB: calls that reused the stored      */
  int64_t cross_reused;          /*   self / cross attention outputs       */
  int32_t n_cand;                /* current candidate count (after retain) */
} cs_rollout_stats_t;

/* Kernel families timed by the optional profiler (cs_profile_*). */
typedef enum {
  CS_K_SELF_ATTN = 0, CS_K_CROSS_ATTN = 1, CS_K_GEMM = 2, CS_K_NORM = 3,
  CS_K_DECIDE = 4, CS_K_UPDATE = 5, CS_K_SCORE = 6, CS_K_OTHER = 7,
  CS_K_COUNT = 8
} cs_kernel_family;

/* ---------------------------------------------------------------- model */

/* Number of float32 values in the flat weight array for `desc`.  Order:
 * patch_w[d][p] patch_b[d] text1_w[d][text_dim] text1_b[d] text2_w[d][d]
 * text2_b[d] time1_w[d][256] time1_b[d] time2_w[d][d] time2_b[d]
 * mod_w[6d][d] mod_b[6d], then per block: mod[6][d] (shift1, scale1,
 * gate1, shift2, scale2, gate2) qkv_w[3d][d] qkv_b[3d] q_gain[d] k_gain[d]
 * o_w[d][d] o_b[d] ca_ln_g[d] ca_ln_b[d] caq_w caq_b cak_w cak_b cav_w
 * cav_b ([d][d], [d]) caq_gain[d] cak_gain[d] cao_w[d][d] cao_b[d]
 * ffn1_w[ffn][d] ffn1_b[ffn] ffn2_w[d][ffn] ffn2_b[d], then head_mod[2][d]
 * (shift, scale) head_w[p][d] head_b[p], with d = hidden and
 * p = in_ch*patch_t*patch_h*patch_w.  Matrices are [out][in] row-major. */
cs_status cs_model_weight_count(const cs_model_desc* desc, size_t* count);

/* Build a model.  weights: device, float32, cs_model_weight_count values
 * (copied; matrices rounded to bf16 round-to-nearest-even in CS_BF16 mode,
 * vectors kept fp32).  stream: hipStream_t or NULL.  On success *out owns
 * device memory until cs_model_free. */
cs_status cs_model_init(const cs_model_desc* desc, const float* weights, size_t n_weights,
                        void* stream, cs_model** out);
void cs_model_free(cs_model* model);

/* RMS norm of q and k inside the transformer: over the whole hidden width
 * (cs_model_init), or over each head's own channels (cs_qk_norm_rope).  The
 * gains are the same [d] vectors either way. */
typedef enum { CS_QK_NORM_FULL = 0, CS_QK_NORM_HEAD = 1 } cs_qk_norm;
/* cs_model_init with the choice of the norm (cs_qk_norm).  Everything else,
 * rollouts included, is as with cs_model_init. */
cs_status cs_model_init_norm(const cs_model_desc* desc, int32_t qk_norm, const float* weights,
                             size_t n_weights, void* stream, cs_model** out);

/* One transformer evaluation v_theta(x, t, c) (Sec. Preliminaries) for n
 * latents sharing the timestep t and one text context.  x: device
 * [n][D] float32; ctx: device [text_len][text_dim] float32; v: device
 * [n][D] float32 (may not alias x).  Enqueued on the model's stream. */
cs_status cs_velocity(cs_model* model, const float* x, int32_t n, float t, const float* ctx,
                      float* v);

/* Contexts: the text of n_prompts prompts of their own lengths, projected to
 * the keys and values of every block once and kept, in the model's compute type
 * or in 4 bits (cs_kv4_cache: about a quarter of the memory, and its rounding).
 * ctx: device [n_prompts][text_len][text_dim] float32, lens: host [n_prompts],
 * the rows of each prompt (0..text_len; a prompt of none adds no attention), or
 * NULL for text_len each; rows past a prompt's length may hold anything.
 * Synchronises the model's stream.  The context belongs to its model and is freed
 * before it. */
typedef enum { CS_KV_NATIVE = 0, CS_KV_4BIT = 1 } cs_kv_format;
typedef struct cs_context cs_context;
cs_status cs_context_init(cs_model* model, const float* ctx, const int32_t* lens,
                          int32_t n_prompts, int32_t kv_format, cs_context** out);
void cs_context_free(cs_context* context);

/* cs_velocity for n latents that attend to prompts of a context, each over its
 * prompt's length: prompt: host [n], the prompt of each latent; NULL: latent i
 * attends to prompt i (n <= n_prompts). */
cs_status cs_velocity_context(cs_model* model, cs_context* context, const float* x,
                              const int32_t* prompt, int32_t n, float t, float* v);

/* -------------------------------------------------------------- rollout */

/* Start a generation (Alg. 1: reset cache state, then G_tau(c, s_i) for
 * every seed).  x1: device [n_cand][D] float32 initial noise (copied).
 * ctx_cond / ctx_uncond: device [text_len][text_dim] float32; ctx_uncond
 * must be non-NULL iff n_branch == 2 (copied into per-branch cross-attention
 * keys/values here, once per rollout).  All cache state is zeroed.  In
 * CS_CACHE_PAB mode both ranges must be >= 1 (else CS_E_INVAL) and the two
 * attention-output arrays are allocated here (CS_E_NOMEM if they do not
 * fit). */
cs_status cs_rollout_init(cs_model* model, const cs_rollout_desc* desc, const float* x1,
                          const float* ctx_cond, const float* ctx_uncond, cs_rollout** out);
void cs_rollout_free(cs_rollout* r);

/* Cache decision for step `step` (must be the next step, 1..n_steps) for
 * every candidate i and branch b (Eq. indicator and its rule): forced
 * calls compute; otherwise a_ib += ||x_i - xref_ib||_F / ||xref_ib||_F and
 * the call is skipped iff a_ib <= tau (a call with ||xref|| = 0 computes).
 * override_mask: NULL, or host [n_cand][n_branch] bytes (1 = compute) that
 * replace the rule's decisions (replay); the indicator is still accumulated
 * and reported.  An override that skips a call with no cached residual (in
 * CS_CACHE_OFF mode, or before that branch's first computed call) is
 * rejected with CS_E_INVAL before any device work.  mask_out: NULL or host [n_cand][n_branch] (1 = compute).
 * a_out: NULL or host [n_cand][n_branch], the indicator value compared with
 * tau at this step, NaN where the call was forced.  Calling it twice for
 * the same step returns CS_E_STATE.  In CS_CACHE_PAB mode every call
 * computes (mask all 1, a NaN) unless overridden. */
cs_status cs_cache_decide(cs_rollout* r, int32_t step, const uint8_t* override_mask,
                          uint8_t* mask_out, double* a_out);

/* Execute step `step`: evaluate the transformer for the computed calls,
 * refresh Delta = v - x and x_ref = x on them (Eq. delta), form x + Delta on
 * the skipped ones (Eq. skip), combine branches (Eq. cfg) and take the
 * Euler step (Eq. euler).  Runs cs_cache_decide(step, NULL, NULL, NULL)
 * first if it was not called for this step.  In CS_CACHE_PAB mode the
 * attention outputs follow the broadcast schedule described with
 * cs_cache_mode; a replay override is then not allowed (CS_E_UNSUPPORTED
 * from cs_cache_decide). */
cs_status cs_denoise_step(cs_rollout* r, int32_t step);

/* Scores s_i = <w, x_i> / sqrt(D) of the current latents, summed in fp64 in
 * a fixed order (the stand-in verifier of Alg. 1).  w: device [D] float32;
 * scores: host [n_cand] double.  Synchronises. */
cs_status cs_score(cs_rollout* r, const float* w, double* scores);

/* Allocation-free scoring, for callers that cannot allocate device memory
 * (code under HIP graph capture, serving loops or harnesses that forbid
 * hipMalloc): the scores of cs_score, s_i = <w, x_i> / sqrt(D) summed in
 * fp64 in the same fixed order (bitwise equal to cs_score on the same
 * latents), for n latents the caller holds, without a rollout handle.
 * x: device [n][D] float32, w: device [D] float32, both 16-byte aligned;
 * D % 4 == 0; scores: device [n] double (written); stream: hipStream_t or
 * NULL.  Only enqueues work (no synchronisation, no allocation, no memset).
 * The per-chunk partial sums go to a static device array owned by the
 * library, CS_SCORE_NOALLOC_MAX_PARTIALS doubles (4 MiB) per GPU, held until
 * the process ends; n * ceil(D / 8192) above that capacity returns
 * CS_E_INVAL before any device work.  Every call on one GPU shares that
 * array and it keeps the last call's contents: calls that overlap on one
 * GPU (different streams, or host threads) race and must be serialised by
 * the caller. */
#define CS_SCORE_NOALLOC_MAX_PARTIALS (512 * 1024)
cs_status cs_score_noalloc(const float* x, const float* w, int32_t n, int64_t D, double* scores,
                           void* stream);

/* Pruned composition (Sec. Composition with pruned search).
 * cs_rollout_enable_preview(r, 1) makes every following cs_denoise_step also
 * keep the guided velocity v~ of that step (one extra [n_cand][D] fp32
 * buffer, allocated here; 0 frees it).  cs_preview_score then scores the
 * sampler's x0 estimate after the last completed step k,
 * x0_hat = x_{t_{k+1}} - t_{k+1} v~_k, as <w, x0_hat>/sqrt(D) (fp64, fixed
 * order); it returns CS_E_STATE unless the preview was enabled before step
 * k.  w: device [D]; scores: host [n_cand].  Synchronises.
 * cs_rollout_retain keeps only the candidates keep[0..n_keep-1] (host,
 * strictly increasing indices in the current numbering) with their complete
 * cache state; they are renumbered 0..n_keep-1 and n_cand becomes n_keep.
 * Not allowed between cs_cache_decide and cs_denoise_step (CS_E_STATE),
 * nor in CS_CACHE_PAB mode (CS_E_UNSUPPORTED).  Synchronises. */
cs_status cs_rollout_enable_preview(cs_rollout* r, int32_t on);
cs_status cs_preview_score(cs_rollout* r, const float* w, double* scores);
cs_status cs_rollout_retain(cs_rollout* r, const int32_t* keep, int32_t n_keep);

/* Copy the current latents to dst: device [n_cand][D] float32. */
cs_status cs_rollout_latents(cs_rollout* r, float* dst);

cs_status cs_rollout_stats(cs_rollout* r, cs_rollout_stats_t* out);

/* Checkpoint: the complete rollout state {step, x, x_ref, Delta, a,
 * has_ref}.  cs_rollout_export with buf == NULL stores the required size in
 * *bytes; otherwise buf (host) must hold *bytes bytes.  cs_rollout_import
 * restores a state exported from a rollout with the same model and
 * description.  Both synchronise.  Not available in CS_CACHE_PAB mode,
 * whose state includes the attention-output arrays (CS_E_UNSUPPORTED). */
cs_status cs_rollout_export(cs_rollout* r, void* buf, size_t* bytes);
cs_status cs_rollout_import(cs_rollout* r, const void* buf, size_t bytes);

/* -------------------------------------------------------------- operators
 *
 * Operators of the transformer by themselves, on tensors the caller holds.
 * They take and keep no handle.  Rules common to all of them:
 *  - All tensors are device memory of the current device; dtype (cs_dtype)
 *    is the type of the floating tensors.  Strides are counted in elements;
 *    the channels of a head are contiguous.  Rows are moved 16 bytes at a
 *    time: tensor pointers are 16-byte aligned and strides multiples of 16
 *    bytes (CS_E_INVAL otherwise).  Strides are not negative; an output's
 *    are not zero either, where its axis has several entries.  Beyond that
 *    it is up to the caller that an output's rows and heads do not overlap.
 *  - The work is enqueued on `stream` (hipStream_t or NULL); nothing is
 *    allocated, copied or waited for, so calls can be captured into a HIP
 *    graph.  Descriptors are read before the call returns.  Tensors must
 *    stay valid until the enqueued work is done.
 *  - Calls with nothing to do (no tokens, no queries) return CS_OK.
 *  - A workspace (16-byte aligned, at least the size the _workspace function
 *    gives) carries nothing from one call to the next, but calls that may
 *    overlap (two streams, two graphs) need one each.
 *  - Results do not depend on the batch: a token, or a query set with its
 *    context, gives bitwise the same output alone and among others, and a
 *    query's output does not depend on the values of its set's other queries.
 *    Calls of another lq, lk or number of heads may take other kernels or
 *    cut the keys elsewhere: the same query then agrees to rounding. */

/* Pairs a rotation turns: adjacent channels (2p, 2p + 1), or the first and
 * the second half of the rotated channels (p, p + rot_dim / 2). */
typedef enum { CS_ROPE_PAIRS = 0, CS_ROPE_HALVES = 1 } cs_rope_style;

/* Tokens of cs_qk_norm_rope.  q is [tokens][heads_q][head_dim] with strides
 * q_row and q_head, its output has qo_row and qo_head; k likewise (k_*, ko_*).
 * head_dim: a multiple of 16 up to 256.  rot_dim: channels that turn, the first
 * ones of a head, a multiple of 16 up to head_dim, 0 for none.  rope_rows: rows
 * of the table.  q_gain_head, k_gain_head: stride of the gains from head to
 * head, 0 if all heads share one. */
typedef struct {
  int32_t dtype;                 /* cs_dtype */
  int32_t tokens, heads_q, heads_k, head_dim;
  int32_t rot_dim, rope_rows, rope_style;
  float eps;                     /* >= 0 */
  int64_t q_row, q_head, k_row, k_head;
  int64_t qo_row, qo_head, ko_row, ko_head;
  int64_t q_gain_head, k_gain_head;
} cs_qk_norm_desc;

/* RMS norm of every head of q and k over its own channels, then the rotation:
 *   y_c = x_c / sqrt(mean_c(x_c^2) + eps) * gain_c,
 *   (a, b) -> (a cos - b sin, a sin + b cos) for the pairs of the first rot_dim
 * channels, in fp32 and rounded once (the sum of squares too: a head of length 1.8e19 or
 * more gives zeros, and with eps 0 one shorter than 1e-19 is not resolved).  rope: device float
 * [rope_rows][rot_dim / 2][2] (cos, sin); token t takes row pos[t] (device
 * int32), or row t % rope_rows if pos is NULL.  A token whose position is
 * negative is skipped: its outputs are left as they were (padding).  One whose
 * position is not below rope_rows gets NaN.  Gains are fp32.  heads_q or heads_k
 * may be 0: those pointers are then not read.  An output may be its input (same
 * pointer and strides); other overlaps are not allowed. */
cs_status cs_qk_norm_rope(const cs_qk_norm_desc* desc, const void* q, const void* k, void* q_out,
                          void* k_out, const float* q_gain, const float* k_gain,
                          const float* rope, const int32_t* pos, void* stream);

/* Attention of queries to contexts: n_q query sets of lq queries each, n_kv
 * contexts of up to lk keys and values.  heads_q is a multiple of heads_kv: query
 * head h reads key head h / (heads_q / heads_kv).  head_dim 32, 64 or 128.
 * Strides: set or context (_b), row (_r) and head (_h); mask_b is the stride of
 * the mask from context to context (bytes, any alignment).  scale, in (0, 1e38),
 * multiplies the products q.k; scores of 10^9 and more in magnitude are not
 * supported (the softmax subtracts rounded maxima). */
typedef struct {
  int32_t dtype;                 /* cs_dtype of q, o (and k, v) */
  int32_t n_q, n_kv, lq, lk;
  int32_t heads_q, heads_kv, head_dim;
  float scale;
  int64_t q_b, q_r, q_h, k_b, k_r, k_h, v_b, v_r, v_h, o_b, o_r, o_h;
  int64_t mask_b;
} cs_attn_desc;

/* o = softmax(scale q k^T) v over the keys that are left of each set's context.
 * kv_of: device int32 [n_q], the context of each query set; NULL: set i reads
 * context i (n_kv >= n_q then).  kv_len: device int32 [n_kv], keys of each
 * context (clamped to 0..lk); NULL: lk.  kv_mask: device bytes, row j at kv_mask +
 * j * mask_b, key i of context j is left out where byte i is 0; NULL: none.  Keys
 * that are left out are never met: their rows may hold anything, NaN included.  A
 * query with no key left, or whose kv_of is not in 0..n_kv-1, gets zeros.  Scores
 * and sums are fp32; in CS_BF16 mode the softmax weights are rounded to bf16 for
 * the product with v and summed as rounded.  In CS_FP32 mode a product may be taken
 * as six products of bf16 terms (off by at most 2^-22 of its magnitude; it is where
 * lq * heads_q is at least 8,192 and lq * heads_q / heads_kv above 64).  An element
 * of 3.39e38 or more, infinities included, in a query or in a key or value that is
 * not left out then makes NaN of the outputs it enters, and one below 2^-103 (1e-31) is
 * held to 2^-134 instead of its 24 bits.  o must not overlap the
 * inputs.
 * cs_cross_attention_workspace gives the bytes of `work` (0: work may be NULL). */
cs_status cs_cross_attention_workspace(const cs_attn_desc* desc, size_t* bytes);
cs_status cs_cross_attention(const cs_attn_desc* desc, const void* q, const void* k, const void* v,
                             const int32_t* kv_of, const int32_t* kv_len, const uint8_t* kv_mask,
                             void* o, void* work, size_t work_bytes, void* stream);

/* A key/value cache in 4 bits: n_kv contexts of cap rows, `heads` heads of
 * head_dim (32, 64 or 128) channels.  A row of a head is held as e2m1 codes
 * (magnitudes 0, 0.5, 1, 1.5, 2, 3, 4, 6; sign in bit 3), two to a byte with the
 * even channel in the low half, and one scale byte b = 2^(b - 127) per 32
 * channels:
 *   codes  [n_kv][heads][cap][head_dim / 2], scales [n_kv][heads][cap][head_dim / 32]
 * for the keys and for the values, contiguous, 16-byte aligned: 4.25 bits a
 * channel.  The caller owns the four arrays; rows never stored hold what the
 * caller left there. */
typedef struct {
  uint8_t *k_codes, *k_scales, *v_codes, *v_scales;
  int32_t n_kv, heads, cap, head_dim;
} cs_kv4_cache;

/* Rows of keys and values, [n_rows][heads][head_dim] with the given strides, for
 * cs_kv4_store and cs_kv4_load. */
typedef struct {
  int32_t dtype, n_rows;
  int64_t k_row, k_head, v_row, v_head;
} cs_kv4_rows;

/* Store rows into the cache, or load the values that stored rows stand for.
 * slots: device int32 [n_rows], row i belongs to slot (context * cap + row); a
 * negative slot, or one not below n_kv * cap, skips the row (a loaded row is then
 * left as it was).  NULL: row i belongs to slot i (n_rows <= n_kv * cap).  Slots
 * named twice in one store end with an unspecified mix of the rows.
 * Rounding: a group's scale is the power of two that puts its largest magnitude
 * into [3.5, 7) (at least 2^-126), its codes are the nearest magnitudes, halfway
 * values to the even code, values over 6 to 6.  A group that holds an infinity or
 * a NaN gets scale byte 255 and stands for NaNs (bf16 magnitudes from 1.75 x 2^127 on
 * load as infinities).  k and v, or their rows' pointers,
 * may not be NULL unless n_rows is 0.  n_kv * cap is below 2^31. */
cs_status cs_kv4_store(const cs_kv4_cache* cache, const cs_kv4_rows* rows, const void* k,
                       const void* v, const int32_t* slots, void* stream);
cs_status cs_kv4_load(const cs_kv4_cache* cache, const cs_kv4_rows* rows, void* k, void* v,
                      const int32_t* slots, void* stream);

/* cs_cross_attention over a 4-bit cache: context j is the cache's context j, and
 * desc's n_kv, lk, heads_kv and head_dim are the cache's (its k_ and v_ strides are
 * not read).  In CS_FP32 mode queries are taken in bf16 terms, with their limits.  Rows
 * that are left out may hold any bytes.  In CS_BF16 mode with more than
 * 192 queries to a key head (lq * heads_q / heads_kv) the workspace holds the keys and
 * values of min(n_q, n_kv) contexts in bf16: 4 * lk * heads_kv * head_dim bytes each. */
cs_status cs_kv4_attention_workspace(const cs_attn_desc* desc, size_t* bytes);
cs_status cs_kv4_attention(const cs_attn_desc* desc, const void* q, const cs_kv4_cache* cache,
                           const int32_t* kv_of, const int32_t* kv_len, const uint8_t* kv_mask,
                           void* o, void* work, size_t work_bytes, void* stream);

/* ---------------------------------------------------------------- ranking */

/* Host only, thread-safe.  Orders candidates by decreasing score (equal
 * scores: lower index first) for both score vectors, and computes the
 * Spearman correlation of average ranks (NaN if a vector is constant) and
 * top-1 agreement (Sec. Experiments, definitions and protocol; Alg. 1's
 * argmax).  s_cached, s_full: host [n] doubles; order_cached, order_full:
 * host [n] int32 (position 0 = best).  n >= 2 else CS_E_INVAL; scores must
 * not be NaN.  Any output pointer may be NULL.
 * Order only: with s_full == NULL only order_cached is written (n >= 1);
 * order_full, rho and top1_agree must then be NULL (else CS_E_INVAL).  This
 * is the ranking step of a search without a reference: keep mode's argmax
 * (order_cached[0]) and the top-k of pruned search. */
cs_status cs_rank(const double* s_cached, const double* s_full, int32_t n, int32_t* order_cached,
                  int32_t* order_full, double* rho, int32_t* top1_agree);

/* ---------------------------------------------------------------- profiler */

/* Enable (1) or disable (0) HIP-event timing of every kernel launch the
 * rollout (and its model's cs_velocity) enqueues, per cs_kernel_family.
 * cs_profile_read synchronises, then reports the summed device time in ms
 * and the number of launches since the last reset. */
cs_status cs_profile_enable(cs_model* model, int32_t on);
cs_status cs_profile_reset(cs_model* model);
cs_status cs_profile_read(cs_model* model, int32_t family, double* total_ms, int64_t* launches);

/* Thread-local description of the last failure in this thread. */
const char* cs_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* CACHEDSEARCH_CS_H */
