/*
 * sara.h - C ABI of libsara: the rollout-generation hot path of SARA
 * (Sequential Adaptive Rollout Allocation) on one MI355X (gfx950).
 *
 * One allocation step (Algorithm 1, section 3.3) is driven by the host as
 *
 *     sara_begin_step(...)                      prompt pool in, prefill, first draws
 *     repeat: sara_decode_step -> sara_posterior_decide -> sara_refill
 *             (or sara_run, which replays that triple from a HIP graph)
 *     until the step is done (sara_query / sara_run report it)
 *     sara_finish_step(...)                     GRPO advantages of committed groups
 *
 * All calls enqueue work on the context's stream and return at once unless
 * stated otherwise.  Pointers prefixed d_ are device (HIP) memory, h_ host
 * memory.  Sizes are element counts.  The context is not thread safe: use one
 * context per host thread and stream.
 *
 * Errors: every int-returning call returns SARA_OK or a negative code and
 * sets a thread-local message readable with sara_last_error().  Argument
 * errors are detected synchronously (SARA_EINVAL) and enqueue nothing.
 * Budget or prompt-pool exhaustion is not an error: the step ends with fewer
 * than B committed groups.
 */
#ifndef SARA_H
#define SARA_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct sara_ctx sara_ctx;

enum {
  SARA_OK = 0,
  SARA_EINVAL = -1,   /* invalid argument or unsupported configuration         */
  SARA_ENOMEM = -2,   /* device allocation failed                              */
  SARA_EHIP = -3,     /* a HIP runtime call failed                             */
  SARA_ESTATE = -4,   /* call out of order (e.g. decode before begin_step)     */
  SARA_EDEVICE = -5   /* a device-side check failed (see sara_step_stats.error) */
};
enum { SARA_F32 = 0, SARA_BF16 = 1 };
/* SARA_MODE_SARA_THOMPSON: SARA with the posterior-sampling priority of the
 * index-policy proposition (Thompson sampling as the alternative index to
 * p_eff): when a prompt's rollouts are queued (at its draw, or at a CONTINUE
 * decision after n outcomes with s successes) it draws g ~ Beta(a, b), its
 * current posterior (a = alpha0 + s, b = beta0 + n - s), as the a-th
 * smallest of a + b - 1 uniforms (w + 1/2) 2^-32, w the words of
 * Philox4x32-10 under the sampler's key at counters (uid, n, c, 2), and its
 * pending rollouts are ordered by P(group of k ends mixed | g) (Eq. peff at
 * the draw: 1 - g^k - (1-g)^k, 1 - (1-g)^r after s = 0, 1 - g^r after
 * s = n, r = k - n; powers by repeated fp64 multiplication) instead of
 * p_eff.  Decisions are unchanged.  A prompt whose posterior parameters are
 * not integers, or with a + b - 1 > 4096, keeps the p_eff index. */
enum { SARA_MODE_SARA = 0, SARA_MODE_FIXED_K = 1, SARA_MODE_SARA_THOMPSON = 2 };
/* decision codes in the decision log */
enum { SARA_COMMIT = 1, SARA_ABANDON = 2, SARA_CONTINUE = 3 };
/* per-prompt status */
enum { SARA_UNDRAWN = 0, SARA_ACTIVE = 1, SARA_COMMITTED = 2, SARA_ABANDONED = 3 };
/* bits of the device error word (sara_step_stats.error) */
enum { SARA_DEVERR_WARM_ID = 1 };   /* a warm-start prompt id outside [0, n_store) */

/* Decoder shape.  Pre-norm GQA decoder: RMSNorm, rotate-half RoPE, SwiGLU,
 * untied LM head, no biases.  head_dim in {64, 128}; n_heads a multiple of
 * n_kv_heads with at most 8 query heads per KV head; d_model, d_ffn and
 * n_heads*head_dim multiples of 64; vocab a multiple of 16.  dtype SARA_BF16 stores weights, KV cache
 * and GEMM inputs in bf16 (fp32 accumulation); SARA_F32 computes in fp32.
 * eos_id = -1 disables the EOS token. */
typedef struct {
  int32_t n_layers, d_model, n_heads, n_kv_heads, head_dim, d_ffn, vocab;
  float rope_theta, rms_eps;
  int32_t dtype;
  int32_t eos_id;
} sara_model_desc;

/* Allocation problem of one step (Algorithm 1 inputs; implementation-details
 * appendix for commit_min, the prior and the budget cap):
 *   mode        SARA_MODE_SARA, SARA_MODE_FIXED_K or SARA_MODE_SARA_THOMPSON
 *   B           effective groups wanted (ignored in SARA_MODE_FIXED_K)
 *   k           group size;  n0 probe rollouts per fresh prompt (1..k)
 *   commit_min  commit floor (2..k); tau_low abandon threshold in [0, 1]
 *   alpha0/beta0  Beta prior (> 0);  budget_N  rollout budget of the step
 *   pool_U      prompts in the step's pool;  n_slots concurrent rollout slots
 *   kv_block    KV page size in tokens (must be 16)
 *   max_prompt  longest prompt;  max_new  generated-token cap per rollout
 *   temperature sampling temperature (> 0);  top_p in (0, 1]: 1 samples the
 *               full softmax, < 1 the top-p nucleus (smallest set of most
 *               likely ids whose probability mass reaches top_p, with every
 *               id tied at the cut; mass counted in integer weights
 *               floor(exp(z - z_max) * 2^44) of z = fp32(logit / T)).  The
 *               nucleus path writes fp32 logits [n_slots][vocab] (library
 *               memory for bf16 models) and runs separate sampler kernels
 *   forced_eos_u32  per-token probability x / 2^32 of a forced EOS (0 = off)
 *   prio_quant_bits  quantisation of the p_eff priority key (1..21)
 *   seed        key material of the counter-based sampler and reward hash
 * Limits: min(budget_N, pool_U * k) <= 4096 queued rollouts; pool_U < 2^26;
 * n_slots <= 4096. */
typedef struct {
  int32_t B, k, n0, commit_min;
  double tau_low, alpha0, beta0;
  int64_t budget_N;
  int32_t pool_U, n_slots, kv_block, max_prompt, max_new, mode;
  float temperature, top_p;
  uint32_t forced_eos_u32;
  int32_t prio_quant_bits;
  uint64_t seed;
} sara_alloc_desc;

typedef struct {
  int32_t done;          /* 1 once no prompt is active                      */
  int32_t error;         /* device error word, 0 = none                      */
  int32_t decode_steps;  /* decode steps executed in this allocation step    */
  int32_t drawn;         /* prompts drawn from the pool                      */
  int32_t committed;     /* |C|: effective groups collected                  */
  int32_t abandoned;
  int32_t active;        /* |A|                                             */
  int32_t queued;        /* rollouts waiting for a slot                      */
  int32_t running;       /* occupied slots                                   */
  int32_t pad_;
  int64_t budget_left;   /* N - rollouts issued (k reserved per active prompt) */
  int64_t rollouts;      /* rollouts issued                                  */
  int64_t tokens;        /* tokens generated                                 */
  int64_t n_decisions, n_draws, n_assigns, n_finishes;  /* log lengths       */
} sara_step_stats;

/* Create a context on the current HIP device for one allocation problem:
 * the inputs of Algorithm 1 (its Require line: pool, target B, group size k,
 * probe n0, threshold tau_low, prior (alpha0, beta0), budget cap) plus the
 * defaults of the implementation-details appendix ("Defaults and history
 * warm-start": commit_min, the 6Bk safety cap) and the decoder that
 * generates the rollouts.
 * d_weights: n_weights device pointers in this order, each row-major
 * [out][in] in the model dtype (bf16 as raw 16-bit patterns):
 *   embed[V][d]; per layer l: attn_norm[d], wq[Hq*hd][d], wk[Hkv*hd][d],
 *   wv[Hkv*hd][d], wo[d][Hq*hd], ffn_norm[d], wg[ffn][d], wu[ffn][d],
 *   wd[d][ffn]; then final_norm[d], lm_head[V][d].
 * n_weights must be 3 + 9 * n_layers.  The weights are copied (repacked)
 * into library-owned memory; the caller may free its copies once the stream
 * has passed this call.  stream: a hipStream_t, or NULL for the null stream.
 * All KV, slot, controller and workspace memory is allocated here. */
int sara_init(const sara_model_desc* model, const sara_alloc_desc* alloc,
              const void* const* d_weights, int32_t n_weights, void* stream,
              sara_ctx** out);

/* Start an allocation step over a pool of pool_U prompts (Algorithm 1, first
 * state: the collected set empty, B fresh prompts probed with n0 rollouts
 * each; the pool is the prompt pool D of its Require line).
 * d_tokens: concatenated prompt token ids (device, int32);
 * h_offsets: pool_U + 1 host offsets into d_tokens (prompt u is
 *   [h_offsets[u], h_offsets[u+1]), length 1..max_prompt);
 * d_p: per-prompt success probability of the synthetic verifier (device, fp64);
 * d_forced_len: NULL or [pool_U * k] forced rollout lengths in 1..max_new
 *   (the token at that index becomes EOS and the rollout ends);
 * step_index: enters the sampler key and the reward hash.
 * The inputs are copied; the caller may reuse them once the stream has
 * passed this call.  Enqueues: state reset, prefill of every prompt of the
 * pool into its shared paged KV blocks, the first draws and slot
 * assignments. */
int sara_begin_step(sara_ctx* ctx, const int32_t* d_tokens, const int32_t* h_offsets,
                    const double* d_p, const int32_t* d_forced_len, int32_t step_index);

/* One decode step over every occupied slot, one token for each running
 * rollout: the batched generation call of Algorithm 1 ("one batched call"),
 * and of the implementation-details appendix ("Round-synchronous batched
 * scheduling": one generation call over all active prompts), taken here one
 * token at a time so that decisions can follow every token.  Embedding, n_layers decoder
 * layers over the paged KV cache, LM head, Gumbel-max sampling keyed by
 * (seed, step_index, rollout id uid*k + j, generated index), forced EOS,
 * reward hash, termination.
 * d_forced_tok: NULL or [pool_U * k][max_new] teacher-forcing table (device);
 * the forced token is appended and rewarded, the sampled one is recorded.
 * d_logits: NULL or [n_slots][vocab] fp32 (device); receives the logits of
 * each occupied slot's row.  model_free != 0 skips the decoder: the forced
 * table (required) supplies every token. */
int sara_decode_step(sara_ctx* ctx, const int32_t* d_forced_tok, float* d_logits,
                     int32_t model_free);

/* Section 3.2-3.3 (Beta posterior, Proposition 1, Eq. decide; the loop body
 * of Algorithm 1).  Apply the finished rollouts of the last decode step to
 * their prompts' (n, s) and decide every quiescent active prompt with Eq. decide:
 * Beta(alpha0 + s, beta0 + n - s), p_eff by Proposition 1 (fp64 lgamma),
 * commit / abandon (refund k - n) / continue (queue more rollouts). */
int sara_posterior_decide(sara_ctx* ctx);

/* The reallocation of Algorithm 1 (draw fresh prompts, probe n0, toward the
 * remaining need; advance continuing prompts prioritised by p_eff, section
 * 3.3).  Draw fresh prompts while |A| < B - |C|, budget_left >= k and the pool is
 * not exhausted; order the pending rollouts by (quantised p_eff desc, uid,
 * j) and assign them to free slots in ascending slot order. */
int sara_refill(sara_ctx* ctx);

/* The while loop of Algorithm 1 on the device (implementation-details
 * appendix, "Round-synchronous batched scheduling": rounds of one batched
 * generation call followed by the decisions and the reallocation; here the
 * decisions follow every decode step and no round barrier reaches the
 * host).  Drives the step to completion: replays [decode, decide, refill]
 * from a HIP graph of graph_iters iterations, polling the done flag
 * asynchronously.  (bf16 models: from one of two graphs, by the live rows;
 * same results.)
 * Synchronises before returning.  d_forced_tok as in sara_decode_step.
 * *iters_out receives the number of loop iterations enqueued. */
int sara_run(sara_ctx* ctx, const int32_t* d_forced_tok, int32_t graph_iters,
             int64_t max_iters, int64_t* iters_out);

/* Synchronise the stream and report the step's counters: the loop state of
 * Algorithm 1 (|C|, |A|, budget left) and its cost in rollouts and tokens
 * (experimental setup appendix, "Metrics").  Returns SARA_EDEVICE when the
 * device error word is set. */
int sara_query(sara_ctx* ctx, sara_step_stats* out);

/* Last line of Algorithm 1: the GRPO update (Eq. grpo, section 2) receives
 * the effective groups of C.  Build the CSR of committed groups (ascending
 * uid, rollouts in j order) and compute their advantages with
 * grpo_group_advantages.  Enqueued. */
int sara_finish_step(sara_ctx* ctx, float eps);

/* History warm start (implementation details, "defaults and history
 * warm-start": each prompt carries its posterior across steps with an
 * exponential decay lambda).  For a finite prompt set revisited across
 * allocation steps, set prompt p keeps pseudo-counts (a_p, b_p) >= 0.
 *
 * sara_set_warm_start: from the next sara_begin_step on, pool prompt u is
 * set prompt d_ids[u] and starts from the prior Beta(alpha0 + a_{ids[u]},
 * beta0 + b_{ids[u]}) in place of Beta(alpha0, beta0): its p_eff, its
 * decisions (Eq. decide on the posterior Beta(alpha0 + a + s,
 * beta0 + b + n - s)) and the priority of its probes use that prior.
 *   d_ids  [pool_U] int32, distinct values in [0, n_store)
 *   d_a, d_b [n_store] fp64 pseudo-counts
 * All three stay owned by the caller and must stay valid while warm start is
 * on: every sara_begin_step reads d_ids, d_a and d_b (update the ids between
 * steps to move the pool over the set), sara_warm_start_update writes d_a
 * and d_b.  d_ids == NULL turns warm start off (back to Beta(alpha0, beta0)).
 * Errors: SARA_EINVAL for a null context, or non-null d_ids with null d_a /
 * d_b or n_store < 1.  An id outside [0, n_store) is found on the device:
 * that prompt falls back to Beta(alpha0, beta0) and the step's device error
 * word gets SARA_DEVERR_WARM_ID (sara_query then returns SARA_EDEVICE).
 * Duplicate ids are not detected; their count updates race. */
int sara_set_warm_start(sara_ctx* ctx, const int32_t* d_ids, double* d_a, double* d_b, int32_t n_store);

/* After a step's decode loop has ended (the step is done): for every set
 * prompt p, a_p <- lambda (a_p + s_p) and b_p <- lambda (b_p + n_p - s_p),
 * where n_p and s_p are the rollouts and successes the step gave the pool
 * prompt with id p (0 and 0 if the step did not draw it).  lambda in [0, 1]:
 * 0 forgets (every step starts cold), 1 keeps every outcome.  Enqueued.
 * Errors: SARA_EINVAL for a null context or lambda outside [0, 1];
 * SARA_ESTATE when no warm start is set or no step has begun. */
int sara_warm_start_update(sara_ctx* ctx, double lambda);

/* Asynchronous poll of the loop condition of Algorithm 1: enqueues on the
 * context's stream a small kernel that writes the device error word to
 * h_pinned[1] and then, after a system-scope fence, the done flag (1 once no
 * prompt is active) to h_pinned[0], and returns at once.  h_pinned: 2 int32
 * of pinned host memory (hipHostMalloc, or a pinned torch tensor) owned by
 * the caller.  Set h_pinned[0] = -1 before the call and spin on it (volatile
 * read) until it changes, or synchronise the stream: h_pinned[1] is valid
 * once h_pinned[0] has changed, which lets the host overlap its own work with
 * the decode loop.  Errors: SARA_EINVAL for a null argument or memory that
 * is not pinned host memory; SARA_ESTATE before sara_begin_step. */
int sara_poll(sara_ctx* ctx, int32_t* h_pinned);

/* Copy results to host (synchronises).  Any pointer may be NULL.
 *   h_tokens  [pool_U*k][max_new] int32 appended tokens (-1 past the end)
 *   h_sampled [pool_U*k][max_new] int32 sampler choices
 *   h_len     [pool_U*k] int32 rollout lengths (0 = never issued)
 *   h_reward  [pool_U*k] int32 rewards
 *   h_status, h_n, h_s [pool_U] int32; h_peff [pool_U] fp64 (last p_eff) */
int sara_read_rollouts(sara_ctx* ctx, int32_t* h_tokens, int32_t* h_sampled, int32_t* h_len,
                       int32_t* h_reward, int32_t* h_status, int32_t* h_n, int32_t* h_s,
                       double* h_peff);

/* Copy logs to host (synchronises).  Row formats (int64 each):
 *   decisions: (t, uid, code, n, s, p_eff bits as int64)   [n_decisions][6]
 *   draws:     (t_start, uid)                               [n_draws][2]
 *   assigns:   (t_start, slot, uid, j)                      [n_assigns][4]
 *   finishes:  (t, slot, uid, j, length, reward)            [n_finishes][6]
 * cap_* are row capacities of the buffers; rows beyond a capacity are dropped. */
int sara_read_logs(sara_ctx* ctx, int64_t* h_dec, int64_t cap_dec, int64_t* h_draw,
                   int64_t cap_draw, int64_t* h_asg, int64_t cap_asg, int64_t* h_fin,
                   int64_t cap_fin);

/* GRPO data of the last sara_finish_step (synchronises).
 * h_offsets [committed + 1], h_rewards / h_adv [offsets[committed]]. */
int sara_read_advantages(sara_ctx* ctx, int32_t* h_offsets, float* h_rewards, float* h_adv,
                         int32_t cap);

/* Closed-form predictor of Proposition 1 (Eq. peff) for count prompts, each
 * under its own prior (section 3.2; per-prompt priors are what the history
 * warm start of the implementation-details appendix produces):
 *   d_out[i] = P(group of size k is mixed | d_n[i] observed, d_s[i]
 *              successes) under the prior Beta(d_alpha[i], d_beta[i])
 * in fp64 via lgamma (the posterior is Beta(alpha + s, beta + n - s)).
 * All five arrays are device memory of count elements, owned by the caller.
 * Entries with a non-positive or non-finite prior parameter, or outside
 * 0 <= s <= n <= k, give NaN.  Argument errors (count < 0, k < 1, a null
 * array with count > 0) return SARA_EINVAL and enqueue nothing.  Pure;
 * enqueued on stream. */
int sara_peff_batch(const double* d_alpha, const double* d_beta, const int32_t* d_n,
                    const int32_t* d_s, int32_t k, int32_t count, double* d_out, void* stream);

/* Group-relative advantages of Eq. grpo: for group g with rewards
 * d_r[d_group_off[g] .. d_group_off[g+1]), A_i = (r_i - mean) / (std + eps),
 * std unbiased (m - 1); groups of size < 2 get 0.  d_group_off has
 * n_groups + 1 entries (device).  Enqueued on stream. */
int grpo_group_advantages(const float* d_r, const int32_t* d_group_off, int32_t n_groups,
                          float eps, float* d_adv, void* stream);

/* Sampler alone, for parity on given logits: rows r < n_rows, logits
 * d_logits[r][vocab] fp32, rollout ids d_rid[r], generated indices d_pos[r]
 * -> d_tok[r] (Gumbel-max at temperature over the top-p nucleus, the whole
 * vocabulary when top_p = 1; forced EOS if eos_id >= 0 and forced_eos_u32 >
 * 0).  top_p in (0, 1], else SARA_EINVAL.  -inf logits are masked ids.  At
 * top_p = 1 a +inf logit wins over all finite ones (the lowest id of several)
 * and a NaN never wins; a row of NaN only gives INT32_MAX.  With top_p < 1 a
 * row's largest logit must be finite.  Synchronises the stream. */
int sara_sample_logits(const float* d_logits, int32_t n_rows, int32_t vocab,
                       const int32_t* d_rid, const int32_t* d_pos, uint64_t seed,
                       int32_t step_index, float temperature, float top_p, int32_t eos_id,
                       uint32_t forced_eos_u32, int32_t* d_tok, void* stream);

/* For callers that cannot allocate device memory (code under HIP graph
 * capture, tight serving loops, harnesses that forbid hipMalloc): the
 * sampler of sara_sample_logits with the same arguments and results, whose
 * buffers (per-row chunk winners, top-p histograms and state)
 * live in one static device array per GPU of SARA_NOALLOC_SCRATCH_BYTES
 * bytes, held from the first call on a device until the process ends.  It
 * calls no allocating routine and does not synchronise: the work is
 * enqueued on stream (which must belong to the current device) and d_tok is
 * valid once the stream has passed it.
 * Limits: n_rows <= SARA_NOALLOC_MAX_ROWS, and n_rows <=
 * SARA_NOALLOC_MAX_TOPP_ROWS when top_p < 1; larger inputs, like the
 * argument errors of sara_sample_logits, return SARA_EINVAL and enqueue
 * nothing.  Every call on one GPU shares that GPU's array: calls whose work
 * overlaps on the device (other streams, other threads) race and give
 * undefined tokens; calls ordered on one stream are safe. */
#define SARA_NOALLOC_MAX_ROWS 4096
#define SARA_NOALLOC_MAX_TOPP_ROWS 64
#define SARA_NOALLOC_SCRATCH_BYTES 17307136
int sara_sample_logits_noalloc(const float* d_logits, int32_t n_rows, int32_t vocab,
                               const int32_t* d_rid, const int32_t* d_pos, uint64_t seed,
                               int32_t step_index, float temperature, float top_p, int32_t eos_id,
                               uint32_t forced_eos_u32, int32_t* d_tok, void* stream);

/* Self-check of the fused LM-head sampler (bf16 models).  That sampler
 * bounds the score of every vocabulary id from the bits of its noise word,
 * scores the best bounds with an fp32 estimate of the Gumbel noise, and
 * re-scores exactly (fp64 noise rounded to fp32, the definition of the noise
 * above) only the ids whose bound reaches the best such score less a fixed
 * margin; its output equals the exact Gumbel-max provided the estimate is
 * within 2e-5 of the exact noise for every input.  This call evaluates both for all
 * 2^24 noise inputs on the device and writes the largest absolute distance
 * to *h_out (host).  Synchronous on stream; returns SARA_EHIP on HIP
 * failure. */
int sara_gumbel_fast_max_error(double* h_out, void* stream);

/* ---------------------------------------------------------------------------
 * KV cache in 8 bits
 *
 * A paged cache of one layer that holds K and V in one byte an element, for
 * decoders that keep their own layers (scoring rollouts, long contexts): half
 * the memory and half the attention traffic of bf16 pages.
 *
 * A page holds 16 tokens of a sequence.  For each page and KV head one scale,
 * a power of two, serves its 16 x head_dim elements:
 *     value = code * 2^(b - 127),   b the exponent byte;  b = 255: NaN
 * with codes int8 (-127..127) or fp8 e4m3 (the OCP format, up to 448).  Every
 * value is exact in fp32 and in bf16, but for the two ends of the range: e4m3
 * pages of b = 1 or 2 hold values below bf16's smallest step, 2^-133 (rounded
 * to nearest there), and rounding up to a code may pass the largest finite
 * number (inf).  The caller owns all memory: pages are
 * handed out by page tables d_pages [n_seqs][max_pages] (int32): position p
 * of sequence i lies in page d_pages[i][p / 16], token p % 16.  Sequences may
 * share pages that no call writes.  A page id outside [0, n_pages), -1 for
 * example, is no page: writes to it are dropped, reads give 0, attention does
 * not see its positions.
 *
 * Rows of the ragged calls: sequence i owns rows [d_off[i], d_off[i + 1]) of
 * the caller's tensors (d_off [n_seqs + 1], not decreasing, inside
 * [0, n_rows]); d_off == NULL: one row a sequence (n_rows == n_seqs).  dtype is
 * that of the caller's tensors (SARA_BF16 or SARA_F32): row r, head h begins at
 * r * row_stride + h * head_stride elements, head_dim elements are contiguous.
 * Those pointers and strides must be multiples of 16 bytes, as the codes'
 * pointers.  Rows and heads that a call writes must not overlap: the larger of
 * their strides spans the other axis.  All calls are enqueued on stream and allocate nothing.  head_dim is
 * 64 or 128.  Argument errors return SARA_EINVAL and enqueue nothing. */
enum { SARA_KV8_INT8 = 0, SARA_KV8_E4M3 = 1 };
typedef struct {
  void *k, *v;               /* codes [n_pages][n_kv_heads][16][head_dim]        */
  uint8_t *k_exp, *v_exp;    /* exponent bytes [n_pages][n_kv_heads]             */
  int32_t n_pages, n_kv_heads, head_dim, format;
} sara_kv8_cache;

/* Quantise new K and V rows into the cache: row t of sequence i goes to
 * position d_start[i] + t.  For each page and head that gets a row, with a the
 * largest magnitude of its new elements:
 *     b = the smallest byte >= 1 with a <= M * 2^(b - 127), M = 127 or 448,
 * or, where the page keeps tokens from before d_start[i], the larger of that
 * and the page's old byte; kept codes are rounded to the new scale if it grew.
 * What a page held past its new rows is not kept.  Codes are rounded to
 * nearest, ties to even.  A NaN or infinite element makes
 * the page's byte 255 until a write covers the page's first token again.
 * Positions past the page table are dropped, and so are the rows of a sequence
 * with d_start[i] < 0.  No two sequences of a call may write the same page. */
int sara_kv8_write(const sara_kv8_cache* cache, const void* d_k, int64_t k_row_stride, int64_t k_head_stride,
                   const void* d_v, int64_t v_row_stride, int64_t v_head_stride, int32_t dtype, int32_t n_rows,
                   const int32_t* d_pages, int32_t max_pages, const int32_t* d_start, const int32_t* d_off,
                   int32_t n_seqs, void* stream);

/* Read positions d_start[i] + t of the cache back into rows t of sequence i
 * (0 where there is no page, positions below 0 among them). */
int sara_kv8_read(const sara_kv8_cache* cache, void* d_k, int64_t k_row_stride, int64_t k_head_stride, void* d_v,
                  int64_t v_row_stride, int64_t v_head_stride, int32_t dtype, int32_t n_rows, const int32_t* d_pages,
                  int32_t max_pages, const int32_t* d_start, const int32_t* d_off, int32_t n_seqs, void* stream);

/* Causal grouped-query attention over the cache.  Sequence i holds d_ctx[i]
 * tokens, the queries' own among them (write them first): its n_i query rows
 * are its last n_i positions, row t sees positions 0 .. d_ctx[i] - n_i + t.
 * n_heads is a multiple of the cache's KV heads; head h reads KV head
 * h / (n_heads / n_kv_heads).
 *     out = sum_j softmax_j(scale * q . k_j) v_j    over the visible positions
 * (|scale| at most 2e38)
 * accumulated in fp32, rounded once to dtype; a row that sees nothing is 0.
 * A value whose code rounded past the largest finite number may count as the
 * largest multiple of its page's scale that is finite; a weight times V's scale
 * below 2^-126 may count as 0.
 * max_ctx <= 16 * max_pages and 2^30: no d_ctx[i] is larger (the rows of one
 * that is are NaN); it sizes the launch, so keep it near the longest.
 * d_ws: workspace of at least the bytes that sara_kv8_attention_workspace
 * gives for the same sizes (16-byte aligned; NULL if 0), free for reuse once
 * the stream has passed the call. */
int sara_kv8_attention_workspace(int32_t n_kv_heads, int32_t head_dim, int32_t n_rows, int32_t n_heads, int32_t n_seqs,
                                 int32_t ragged, int32_t max_ctx, int64_t* bytes);
int sara_kv8_attention(const sara_kv8_cache* cache, const void* d_q, int64_t q_row_stride, int64_t q_head_stride,
                       void* d_out, int64_t out_row_stride, int64_t out_head_stride, int32_t dtype, int32_t n_rows,
                       int32_t n_heads, const int32_t* d_pages, int32_t max_pages, const int32_t* d_ctx,
                       const int32_t* d_off, int32_t n_seqs, int32_t max_ctx, float scale, void* d_ws, int64_t ws_bytes,
                       void* stream);

/* The same attention where sequences come in groups that share pages, as the
 * rollouts of a prompt do.  Group j holds the sequences [d_groups[j],
 * d_groups[j + 1]) (d_groups [n_groups + 1], not decreasing, inside [0, n_seqs];
 * a sequence of no group shares nothing); they have d_shared[j] tokens in
 * common, of which the whole pages among the first max_shared are shared.
 * Positions in those pages are read through the page table of the group's FIRST
 * sequence, whatever its d_ctx and the other tables hold there, later positions
 * through each sequence's own.  Every sequence may have any d_ctx, less than
 * d_shared among them; all else is as above.  Where the sizes of the call say
 * that it pays, a group's pages are read once for all of its rows; sizes alone
 * decide, so a captured call keeps its way.  max_shared <= 16 * max_pages and
 * 2^30: keep it near the longest. */
int sara_kv8_group_attention_workspace(int32_t n_kv_heads, int32_t head_dim, int32_t n_rows, int32_t n_heads, int32_t n_seqs,
                                       int32_t n_groups, int32_t ragged, int32_t max_ctx, int32_t max_shared, int32_t dtype,
                                       int64_t* bytes);
int sara_kv8_group_attention(const sara_kv8_cache* cache, const void* d_q, int64_t q_row_stride, int64_t q_head_stride,
                             void* d_out, int64_t out_row_stride, int64_t out_head_stride, int32_t dtype, int32_t n_rows,
                             int32_t n_heads, const int32_t* d_pages, int32_t max_pages, const int32_t* d_ctx,
                             const int32_t* d_off, int32_t n_seqs, const int32_t* d_groups, const int32_t* d_shared,
                             int32_t n_groups, int32_t max_ctx, int32_t max_shared, float scale, void* d_ws, int64_t ws_bytes,
                             void* stream);

/* ---------------------------------------------------------------------------
 * Token log probabilities
 *
 * What the policy-gradient objective needs of a rollout (section 2: the
 * log probabilities of its tokens under a policy) and its gradient.  For rows
 * r < n_rows of logits d_logits[r * row_stride + id], id < vocab (both at most
 * 2^30), in dtype (SARA_BF16 or SARA_F32; any alignment), with
 * z = logit / temperature
 * (1e-37 to 1e37),
 * p = softmax(z) and s = sum exp(z - max z):
 *   d_logp[r]     = log p(d_tok[r]); 0 where d_tok[r] is outside [0, vocab)
 *                   (rows without a token, such as padding)
 *   d_entropy[r]  = -sum p log p
 *   d_stats[r]    = {largest logit, s}: what the gradient needs of the row;
 *                   log sum exp z = stats[0] / temperature + log(stats[1])
 *   d_top_id, d_top_logp [n_rows][n_top]  the n_top (0..32) ids with the
 *                   largest logits, the lower id first among equals, and their
 *                   log p; (-1, -inf) past the ids with a logit above -inf
 * Any of d_logp, d_entropy, d_stats may be NULL, d_top_* if n_top is 0.  -inf
 * logits are masked ids; a row of nothing else gives log p -inf, entropy 0,
 * stats {-inf, 0}.  A NaN or +inf logit makes the row's outputs NaN (NaN is
 * never among the top ids).  Sums are fp32, exponentials below 2^-126 count as
 * 0; one pass over the logits.
 * d_ws: workspace of the bytes that sara_token_logprobs_workspace gives.
 * Enqueued on stream, allocates nothing. */
int sara_token_logprobs_workspace(int32_t n_rows, int32_t vocab, int32_t n_top, int64_t* bytes);
int sara_token_logprobs(const void* d_logits, int32_t dtype, int64_t row_stride, int32_t n_rows, int32_t vocab,
                        const int32_t* d_tok, float temperature, int32_t n_top, float* d_logp, float* d_entropy,
                        float* d_stats, int32_t* d_top_id, float* d_top_logp, void* d_ws, int64_t ws_bytes, void* stream);

/* Gradient of sum_r (d_g_logp[r] * logp[r] + d_g_entropy[r] * entropy[r]) with
 * respect to the logits, in the logits' dtype:
 *   d_grad[r][j] = (g ([j = tok] - p_j) - h p_j (log p_j + entropy)) / temperature
 * d_stats and d_entropy are those of sara_token_logprobs on the same logits
 * and temperature.  d_g_logp or d_g_entropy may be NULL (0); d_entropy may be
 * NULL if d_g_entropy is.  Rows whose g and h are 0, or that have no id left,
 * get 0.  d_grad may be d_logits (same stride): each element is read
 * before it is written, by the same thread.  Enqueued on stream. */
int sara_token_logprobs_grad(const void* d_logits, int32_t dtype, int64_t row_stride, int32_t n_rows, int32_t vocab,
                             const int32_t* d_tok, float temperature, const float* d_stats, const float* d_entropy,
                             const float* d_g_logp, const float* d_g_entropy, void* d_grad, int64_t grad_row_stride,
                             void* stream);

/* ---------------------------------------------------------------------------
 * Token log probabilities from hidden states
 *
 * The same of rows whose logits are products with the LM head,
 *     logit[r][id] = sum_k hidden[r][k] weight[id][k],
 * summed in fp32 and never stored, so that a policy update keeps neither
 * [n_rows][vocab] logits nor their gradient.  d_hidden[r * hidden_stride + k]
 * and d_weight[id * weight_stride + k], k < d_model, are of one dtype (SARA_BF16
 * or SARA_F32: products at fp32 accuracy either way, but for low bits of numbers
 * below 2^-110, which bf16 parts may not hold); 16-byte aligned, rows,
 * strides (at least d_model) and d_model multiples of 16 bytes.  d_logp,
 * d_entropy, d_stats, d_tok and temperature are those of sara_token_logprobs;
 * each of the three outputs may be NULL.  A logit that is not finite (an element
 * that is not, or a sum past fp32) makes its row's outputs NaN.
 * d_ws: workspace of at least the bytes that sara_head_logprobs_workspace gives
 * for the same sizes (grad 0 or 1 for the call below; 16-byte aligned), free for
 * reuse once the stream has passed the call.  Enqueued on stream, allocates
 * nothing; results do not depend on what else runs. */
int sara_head_logprobs_workspace(int32_t dtype, int32_t n_rows, int32_t d_model, int32_t vocab, int32_t grad,
                                 int32_t weight_grad_dtype, int64_t* bytes);
int sara_head_logprobs(const void* d_hidden, int64_t hidden_stride, const void* d_weight, int64_t weight_stride,
                       int32_t dtype, int32_t n_rows, int32_t d_model, int32_t vocab, const int32_t* d_tok, float temperature,
                       float* d_logp, float* d_entropy, float* d_stats, void* d_ws, int64_t ws_bytes, void* stream);

/* Gradients of sum_r (d_g_logp[r] * logp[r] + d_g_entropy[r] * entropy[r]): with
 *   D[r][j] = g ([j = tok] - p_j) - h p_j (log p_j + entropy)
 * formed by pieces of the vocabulary,
 *   d_grad_hidden = D weight / temperature     [n_rows][d_model], in dtype
 *   d_grad_weight = D^T hidden / temperature   [vocab][d_model], in
 *                   weight_grad_dtype: dtype or SARA_F32 (for sums over
 *                   micro-batches); accumulate != 0 adds to what it holds
 * summed in fp32 and rounded once.  D enters the products of a bf16 call rounded
 * to bf16 (2^-8 of an element), for an fp32 weight gradient in two bf16 parts
 * (2^-17), with one part more where a row's largest elements are: a gradient that
 * a few elements make is off by its own rounding, in norm.  That is no bound for
 * each output: one whose terms are all small, or cancel, is off by up to 2^-8
 * (2^-17) of those terms more.  The products of an fp32 call take three parts.
 * Small problems keep D in fp32.  n_rows <= 131,072: more come in several calls,
 * with accumulate.  Either gradient may be NULL, not both; they must not
 * overlap the inputs.  d_stats and d_entropy are those of sara_head_logprobs on
 * the same inputs.  d_g_logp or d_g_entropy may be NULL (0); d_entropy may be
 * NULL if d_g_entropy is.  g counts as 0 where d_tok[r] is outside [0, vocab);
 * rows whose g and h are 0 take no part and get 0, whatever they hold.  Without
 * rows d_grad_weight is 0 (or stays as it is). */
int sara_head_logprobs_grad(const void* d_hidden, int64_t hidden_stride, const void* d_weight, int64_t weight_stride,
                            int32_t dtype, int32_t n_rows, int32_t d_model, int32_t vocab, const int32_t* d_tok,
                            float temperature, const float* d_stats, const float* d_entropy, const float* d_g_logp,
                            const float* d_g_entropy, void* d_grad_hidden, int64_t grad_hidden_stride, void* d_grad_weight,
                            int64_t grad_weight_stride, int32_t weight_grad_dtype, int32_t accumulate, void* d_ws,
                            int64_t ws_bytes, void* stream);

/* Per-kernel timing of eager decode steps.  While enabled, every
 * sara_decode_step call (not the graph replays of sara_run) records a HIP
 * event pair around each kernel it launches on the context's stream, waits
 * for them before returning, and adds to that kernel's class the elapsed
 * time and the algorithmic HBM bytes and flops of the launch (weights,
 * activations and the K/V pages the kernel must touch; workspace traffic
 * of split-K partials is not algorithmic and is not counted). */
typedef struct {
  char name[40];
  int64_t launches;
  double ms;      /* summed event-timed kernel time */
  double bytes;   /* algorithmic bytes of those launches */
  double flops;   /* algorithmic flops of those launches */
} sara_kernel_profile;

int sara_set_profiling(sara_ctx* ctx, int32_t enable);   /* totals are kept */
int sara_reset_profile(sara_ctx* ctx);                   /* zero the totals */
/* Copy up to cap classes (in a fixed order) and their totals; *n_out receives
 * the number of classes. */
int sara_read_profile(sara_ctx* ctx, sara_kernel_profile* out, int32_t cap, int32_t* n_out);

void sara_destroy(sara_ctx* ctx);
const char* sara_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* SARA_H */
