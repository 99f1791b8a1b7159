/* espo.h -- C ABI of the ESPO early-stopping hot path for NVIDIA B200 (sm_100a).
 *
 * ESPO (Early-Stopping Proximal Policy Optimization) ends a rollout during decoding
 * once a smoothed, normalised regret signal computed from the policy's own logits
 * exceeds a threshold gated by the critic's value estimate, and trains on the
 * truncated prefix as an absorbing failure transition.  This library implements the
 * two data-parallel pieces of that method:
 *
 *   espo_step        one pass of the rollout loop body (Algorithm 1) over a batch of
 *                    logit rows: log-softmax statistics, Philox Gumbel-max sampling,
 *                    surrogate regret (Eq. 6), normalisation (Eq. 9), smoothing (Eq. 10),
 *                    value-gated stop test (Eq. 11), per-trajectory bookkeeping;
 *   espo_advantages  TD errors and GAE (Eq. 4-5) over ragged truncated trajectories with
 *                    the failure transition of Eq. 13.
 *
 * and, on the same trajectory slots, the operators of the decode step around espo_step: the paged key/value cache
 * (espo_kv_append, espo_kv_append_rows, espo_kv_gather), attention over shared prompts (espo_attention) and sampling with
 * per-row parameters (espo_sample).
 *
 * Conventions for every entry point
 *   - "device" pointers are CUDA device memory owned by the caller, on the device that
 *     was current when the state was created; "host" pointers are ordinary memory.
 *   - `stream` is a cudaStream_t passed as void* (NULL = the default stream).  Work is
 *     only enqueued; no entry point synchronises the host unless it says so.
 *   - Every function returns an int: ESPO_OK (0) or a negative ESPO_ERR_* code.
 *     Argument errors are found on the host before anything is launched.  Conditions
 *     found on the device (unusable logit rows, bad slot ids, a wait that ran out) are
 *     recorded in a sticky device status word, never trapped.
 *   - There is no CPU fallback: without a CUDA device the calls return ESPO_ERR_CUDA.
 */
#ifndef ESPO_H_
#define ESPO_H_

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* ---- return codes ------------------------------------------------------------------ */
#define ESPO_OK              0
#define ESPO_ERR_NULL       -1   /* a required pointer was NULL                          */
#define ESPO_ERR_BAD_DTYPE  -2   /* dtype code is not ESPO_F32 / ESPO_BF16 (a cache: ESPO_BF16 / ESPO_E4M3) */
#define ESPO_ERR_BAD_SHAPE  -3   /* a size is non-positive, or a stride is shorter than V */
#define ESPO_ERR_ALIGN      -4   /* a pointer is not aligned to its element type          */
#define ESPO_ERR_CAPACITY   -5   /* more rows / tokens than the state or workspace holds  */
#define ESPO_ERR_CUDA       -6   /* a CUDA runtime call failed (see espo_last_cuda_error) */
#define ESPO_ERR_BAD_PARAM  -7   /* a parameter is outside its documented range           */

/* ---- element types of caller buffers ----------------------------------------------- */
#define ESPO_F32   0
#define ESPO_BF16  1
#define ESPO_E4M3  2   /* key/value caches only: 8 bits with a power-of-two scale per (token, head) */

/* ---- sampler ------------------------------------------------------------------------ */
/* Both draw a_t ~ softmax(logits / temperature) exactly, by Gumbel-max with Philox4x32-10
 * noise keyed by (seed; batch_id, trajectory slot, step, index).  They differ in how many
 * draws they need and therefore return different (equally valid) tokens.
 *   FLAT  one draw per vocabulary id: a_t = argmax_a (x_a + G_a).
 *   HIER  the same argmax taken level by level -- first over blocks of 1024 ids scored by
 *         their log-sum-exp, then over sub-blocks of 32 ids inside the winner, then over
 *         the 32 ids -- which needs ~V/1024 + 64 draws per row instead of V.            */
#define ESPO_SAMPLER_FLAT  0
#define ESPO_SAMPLER_HIER  1

/* ---- stop rule (espo_params.stop_mode): the method's own rule and the ablation's replacements (Sec. 6) ---- */
#define ESPO_STOP_ESPO         0   /* z_t > beta * max(V_phi(s_t), eps)            (Eq. 11)          */
#define ESPO_STOP_VALUE_ONLY   1   /* V_phi(s_t) < tau                             (variant D)       */
#define ESPO_STOP_REGRET_ONLY  2   /* z_t > tau                                    (variant E)       */
#define ESPO_STOP_RANDOM       3   /* with probability p_random on every step      (variant F)       */

/* ---- per-trajectory status (espo_state_view: status[]) ------------------------------ */
#define ESPO_ROW_ACTIVE   0
#define ESPO_ROW_STOPPED  1   /* ESPO's rule fired (Eq. 11): failure transition            */
#define ESPO_ROW_EOS      2   /* sampled the end-of-sequence token                          */
#define ESPO_ROW_TMAX     3   /* reached the horizon t_max                                  */
#define ESPO_ROW_BAD      4   /* the logit row held NaN / +inf, or no finite entry          */

/* ---- bits of the sticky device status word (espo_state_status) ---------------------- */
#define ESPO_DEV_BAD_ROW     1u   /* some row was marked ESPO_ROW_BAD                       */
#define ESPO_DEV_BAD_SLOT    2u   /* a row_ids entry was outside [0, capacity)              */
#define ESPO_DEV_TIMEOUT     4u   /* a bounded in-kernel wait ran out; results incomplete   */
                                  /* (the launch's row tickets are left stale: call        */
                                  /* espo_reset_state before the state is used again)      */
#define ESPO_DEV_NAN_VALUE   8u   /* a value estimate was NaN (that row did not stop)       */
#define ESPO_DEV_BAD_LENGTHS 16u  /* espo_advantages: sum(lengths) != total_tokens or L < 0 */
                                  /* espo_attention: a length outside [0, max_pages *        */
                                  /* page_size], clamped; espo_kv_append_rows: not written   */
#define ESPO_DEV_BAD_PAGE    32u  /* a page, cache slot or group outside the cache or tables; its tokens are left out */
#define ESPO_DEV_CACHE_FULL  64u  /* espo_kv_append_rows: a row's pages are full, its token was not written          */

/* Parameters that stay frozen for a whole rollout batch (Sec. 4.2: the statistics are
 * only updated at batch boundaries).  Plain data, passed by host pointer, copied at call. */
typedef struct espo_params {
  float   temperature;      /* > 0 samples from softmax(logits/temperature); 0 = greedy    */
  float   mu_g;             /* running mean of the regret, Eq. 7                            */
  float   sigma2_g;         /* running variance of the regret, Eq. 8 (>= 0)                 */
  float   delta;            /* stabiliser under the square root in Eq. 9 (sigma2_g+delta>0) */
  float   clip_c;           /* clipping bound c of Eq. 9 (> 0)                              */
  float   alpha_s;          /* smoothing factor of Eq. 10, in [0, 1)                         */
  float   beta;             /* threshold multiplier of Eq. 11                               */
  float   eps;              /* value floor epsilon of Eq. 11                                */
  int32_t warmup_complete;  /* 0: the stop test is disabled (critic warm-up); z still runs  */
  int32_t t_max;            /* horizon T_max (> 0)                                          */
  int32_t eos_token;        /* end-of-sequence id, or -1 for none                           */
  int32_t sampler;          /* ESPO_SAMPLER_FLAT or ESPO_SAMPLER_HIER                       */
  int32_t stop_mode;        /* ESPO_STOP_*; every rule is gated by warmup_complete          */
  int32_t shadow;           /* != 0: the first step at which the rule holds is recorded in   */
                            /* t_stop, but the trajectory is not ended and stop_out stays 0  */
                            /* (the "Original" curves of the analysis section)               */
  float   tau;              /* threshold of ESPO_STOP_VALUE_ONLY / ESPO_STOP_REGRET_ONLY     */
  float   p_random;         /* per-step stop probability of ESPO_STOP_RANDOM, in [0, 1]; the */
                            /* draw is Philox level 3, index 0 of the step's stream          */
  int32_t want_entropy;     /* != 0: also compute the policy entropy H(pi(.|s_t)) in the same */
                            /* pass (the quantity tracked in the analysis section); needs    */
                            /* ESPO_SAMPLER_HIER                                              */
  /* Filtered sampling (the paper's evaluation decodes with top-p 0.7, Sec. 5; it gives no rule for ties): a token
   * stays in the support iff the tokens strictly more probable than it weigh less than top_p and number fewer than
   * top_k, so equally probable tokens stay or go together; the token is drawn from the renormalised support and
   * log pi(a_t) refers to it, the regret of Eq. 6 is unchanged.  Needs ESPO_SAMPLER_FLAT; ignored when greedy.
   * A filtered step runs its own kernel (one CTA per row, the row re-read from L2 once per 8 bits of the logit
   * type), not the single-sweep one. */
  float   top_p;            /* in (0, 1): nucleus mass; <= 0 or >= 1: no filter                */
  int32_t top_k;            /* > 0: at most the k most probable (more if tied); 0: no filter  */
} espo_params;

/* Opaque per-rollout-batch state: for each of `capacity` trajectory slots the smoothed
 * regret z, the step counter t, the status, and running sums of g; plus the library's
 * scratch.  Created and destroyed by the library; lives on the device current at creation. */
typedef struct espo_state espo_state;

/* Create the state for up to `capacity` trajectories over a vocabulary of V ids
 * (the initialisation of Algorithm 1: z = 0, t = 0, not done -- for every slot).
 *   out       host pointer that receives the handle
 *   seed      64-bit Philox key;  batch_id  rollout-batch number (< 2^30), part of the counter
 * Allocates device memory (this call and espo_free_state are the only ones that do for the
 * step path) and enqueues the initialisation on `stream`.
 * Errors: NULL, BAD_SHAPE (capacity or V < 1), BAD_PARAM (batch_id >= 2^30), CAPACITY, CUDA. */
int espo_init_state(espo_state** out, int32_t capacity, int32_t V, uint64_t seed, uint64_t batch_id,
                    void* stream);

/* Start a new rollout batch in an existing state: every slot back to z = 0, t = 0, active,
 * sums cleared, sticky status cleared; new batch_id.  Enqueued on `stream`. */
int espo_reset_state(espo_state* st, uint64_t batch_id, void* stream);

/* Release the state and its device memory (synchronises the device). NULL is ignored. */
void espo_free_state(espo_state* st);

/* One decode step for n_rows trajectories (Algorithm 1, loop body; Eq. 6, 9, 10, 11).
 *   logits      device, [n_rows, V] row-major, element type logits_dtype, rows row_stride
 *               ELEMENTS apart (row_stride >= V).  Read exactly once from DRAM.  Entries may
 *               be -inf (masked ids).  The fast path needs a 16-byte aligned base and
 *               row_stride*sizeof(elem) and V*sizeof(elem) multiples of 16; anything else
 *               takes a slower element-wise loader with identical results.
 *   values      device, [n_rows] critic estimates V_phi(s_t) for the same positions, values_dtype
 *   row_ids     device, [n_rows] trajectory slot of each row, or NULL for row i = slot i.
 *               Slots must be distinct within a call.
 *   n_rows      0 <= n_rows <= capacity (0 is a no-op)
 *   params      host pointer; copied before the call returns
 *   tokens_out  device int32 [n_rows]: the sampled token a_t; -1 for a row whose slot is not
 *               active (such rows are otherwise left untouched); 0 for an unusable row
 *   stop_out    device uint8 [n_rows]: 1 iff ESPO's rule fired for the row on this step.
 *               EOS and T_max endings are reported through status[], not here; a sampled
 *               EOS takes precedence over a stop on the same step.
 * For an active row with step counter t the call draws a_t (Philox counter uses t), forms
 * g_t = (max logit - logit[a_t]) / temperature, g~_t, z <- alpha_s z + (1-alpha_s) g~_t,
 * adds g_t and g_t^2 to the slot's running sums, sets t <- t+1, and updates status/t_stop.
 * mu_g, sigma2_g and beta are never modified.  Enqueued on `stream`; calls on the same
 * state must not overlap on the device.
 * Errors: NULL, BAD_DTYPE, BAD_SHAPE, ALIGN, CAPACITY, BAD_PARAM, CUDA. */
int espo_step(const void* logits, int32_t logits_dtype, int64_t row_stride,
              const void* values, int32_t values_dtype,
              const int32_t* row_ids, int32_t n_rows,
              espo_state* st, const espo_params* params,
              int32_t* tokens_out, uint8_t* stop_out, void* stream);

/* Read-only device pointers to the per-slot arrays (each of length capacity); any output
 * pointer may be NULL.  g, g_tilde and logp hold the values of each slot's latest step
 * (logp = log pi(a_t | s_t) under the temperature-scaled distribution).  t is the number
 * of tokens generated; t_stop is the index of the stop step or -1; sum_g, sum_g2 are the
 * double-precision sums over the slot's tokens that the batch statistics of Eq. 7-8 need;
 * entropy is the policy entropy of the slot's latest step and sum_h its running sum (both only
 * maintained by steps with want_entropy set). */
int espo_state_view(espo_state* st, const float** z, const float** g, const float** g_tilde,
                    const float** logp, const int32_t** t, const uint8_t** status,
                    const int32_t** t_stop, const double** sum_g, const double** sum_g2,
                    const float** entropy, const double** sum_h);

/* Expert knob: override the step kernel's launch shape for this state.  consumer_warps =
 * streaming warps per CTA (1..31), stages = blocks of 1024 ids each warp keeps in flight,
 * ctas_per_sm = resident CTAs per SM; 0 keeps the library default for any of them, and the
 * library shrinks what does not fit in shared memory.  Results never depend on it.
 * Errors: NULL, BAD_PARAM. */
int espo_set_launch_config(espo_state* st, int32_t consumer_warps, int32_t stages, int32_t ctas_per_sm);

/* Programmatic dependent launch for the step kernel of ESPO_SAMPLER_HIER (the paper has no counterpart; it is how a
 * decode loop hides launch latency on this hardware).  With enable != 0, espo_step launches its kernel so that the
 * GPU may set it up -- place its thread blocks, run the part that touches no global memory -- while the kernel
 * that precedes it in the stream is still finishing; the step kernel waits for that kernel's completion before it
 * reads or writes any global memory, so what it computes does not change.  The step kernel in turn lets a
 * kernel launched after it in the same way start early; espo_compact_active is launched the same way.  Off by
 * default.  Errors: NULL. */
int espo_set_dependent_launch(espo_state* st, int32_t enable);

/* Stable compaction of the active set: writes the slots whose status is ESPO_ROW_ACTIVE, in
 * increasing order, to row_ids_out (device int32 [capacity]) and their number to
 * n_active_out (device int32 [1]).  Enqueued on `stream`. */
int espo_compact_active(espo_state* st, int32_t* row_ids_out, int32_t* n_active_out, void* stream);

/* Batch boundary (Sec. 4.2, Eq. 7-8 and Sec. 4.3, Eq. 12), to be called after the last step of a
 * rollout batch and before espo_reset_state.  Over the slots that took part (t > 0) it forms, on
 * the device, the mean and the population variance of every regret value g generated in the
 * batch (stop-step tokens included) and the empirical stop rate rho = stopped / took part, then
 *   mu_g     <- alpha_ema mu_g     + (1 - alpha_ema) mean      (set to mean if first_update)
 *   sigma2_g <- alpha_ema sigma2_g + (1 - alpha_ema) variance  (set to variance if first_update)
 *   beta     <- clip(beta + eta_beta (rho - tau), beta_min, beta_max)
 * reading the old values from *params_inout (host) and writing the new ones back to it; the
 * other fields are left alone.  The paper's values: alpha_ema 0.99, eta_beta 0.1, tau 0.25,
 * beta_min 0; it names beta_max without a value.  A batch without tokens changes nothing.
 *   stats_out  host double [6] or NULL: mean, variance, rho, tokens, trajectories, stopped
 * Synchronises `stream`.  Errors: NULL, BAD_PARAM (alpha_ema outside [0,1], NaN, beta_min >
 * beta_max), CUDA. */
int espo_end_batch(espo_state* st, float alpha_ema, float eta_beta, float tau, float beta_min,
                   float beta_max, int32_t first_update, espo_params* params_inout,
                   double* stats_out, void* stream);

/* The batch boundary when the rollout batch's trajectories are spread over several states (one per GPU): every
 * part calls espo_end_batch on a scratch copy of the parameters to obtain its stats_out, the parts exchange those six
 * numbers (one all-gather), and every part calls this with all of them and with the real parameters.  The pooled mean,
 * population variance and stop rate are what espo_end_batch would have found over all trajectories at once, and the
 * same updates (Eq. 7, 8, 12) are applied to *params_inout, so all parts end with identical parameters.  Host only.
 *   stats      host double [n_parts][6], each row as written by espo_end_batch
 *   stats_out  host double [6] or NULL: the pooled mean, variance, rho, tokens, trajectories, stopped
 * Errors: NULL, BAD_SHAPE, BAD_PARAM (as espo_end_batch; also negative counts or NaN in stats). */
int espo_end_batch_merge(const double* stats, int32_t n_parts, float alpha_ema, float eta_beta, float tau,
                         float beta_min, float beta_max, int32_t first_update, espo_params* params_inout,
                         double* stats_out);

/* ---- vocabulary shards (a tensor-parallel LM head leaves every GPU with V/N of each logit row) ----
 * The paper samples from whole rows (Algorithm 1); this pair of calls computes the same step when a row's logits
 * are spread over several buffers.  Every shard reduces its part of the rows to one espo_partial per row
 * (espo_step_partial), the partials of all shards are brought together (one all-gather of 32 bytes per row and
 * shard when the shards live on different GPUs; the library does not communicate) and espo_step_merge finishes the
 * step on the trajectory state: regret, normalisation, smoothing, stop rule, bookkeeping (Eq. 6, 9-11), exactly as
 * espo_step does.  With the flat sampler the Gumbel draws belong to token ids, so the perturbed maximum over the
 * shards is the perturbed maximum over the row and the token does not depend on how the row is cut.  With the
 * hierarchical sampler the block-level draws belong to blocks of 1024 ids of the whole vocabulary: shards that start
 * on such a block give exactly the token of espo_step (each shard resolves the token inside its own best block and
 * reports that block's perturbed score; the merge takes the best of them).  Greedy decoding (temperature 0) and the
 * entropy are offered with the flat sampler only. */
typedef struct espo_partial {
  float m;             /* largest logit of the shard's part of the row (-inf if it has no finite entry)           */
  float s;             /* sum over the part of exp((x - m) / temperature)                                          */
  float best;          /* largest perturbed score x/T + G of the part (greedy: the largest logit; hierarchical       */
                       /* sampler: the best block's score m_b/T + ln s_b + G_b)                                     */
  int32_t best_id;     /* global token id that attains it, lowest id on ties (hierarchical: the token drawn inside  */
                       /* that block); -1: none                                                                     */
  float x_best;        /* that token's logit                                                                        */
  uint32_t flags;      /* bit 0: the part held NaN or +inf; bit 1: nothing computed (bad slot or ended trajectory) */
  uint32_t reserved[2];
} espo_partial;        /* 32 bytes */

/* One shard's share of a decode step.  Reads the state (step counter and slot choose the random stream) and writes
 * partial_out; changes nothing else, so the shards of a step may run in any order or on different GPUs with
 * replicas of the state.
 *   logits_shard   device [n_rows, v_shard] with row_stride elements between rows, dtype as for espo_step
 *   vocab_offset   global id of the shard's first logit; a multiple of 4 (ESPO_SAMPLER_HIER: of 1024);
 *                  vocab_offset + v_shard <= V
 *   partial_out    device espo_partial [n_rows], 16-byte aligned
 *   params         either sampler; ESPO_SAMPLER_HIER needs temperature > 0 and want_entropy = 0 (else
 *                  ESPO_ERR_BAD_PARAM); with ESPO_SAMPLER_FLAT temperature 0 = greedy
 * Calls that use the same state must not overlap on the device (they share its scratch).
 * Errors: NULL, BAD_SHAPE, BAD_DTYPE, BAD_PARAM, ALIGN, CAPACITY, CUDA. */
int espo_step_partial(const void* logits_shard, int32_t logits_dtype, int64_t row_stride, int32_t v_shard,
                      int32_t vocab_offset, const int32_t* row_ids, int32_t n_rows, espo_state* st,
                      const espo_params* params, espo_partial* partial_out, void* stream);

/* Merges the shards' partials and commits the step, with the outputs and state changes of espo_step.
 *   partials      device espo_partial: shard k's result for row r at partials[k * shard_stride + r]
 *   n_shards >= 1, shard_stride >= n_rows (elements)
 *   values, row_ids, tokens_out, stop_out, params: as for espo_step, with the same params as the partial calls
 * A row is marked ESPO_ROW_BAD if any shard flagged NaN / +inf or no shard held a finite logit.
 * Errors: NULL, BAD_SHAPE, BAD_DTYPE, BAD_PARAM, ALIGN, CAPACITY, CUDA. */
int espo_step_merge(const espo_partial* partials, int32_t n_shards, int64_t shard_stride, const void* values,
                    int32_t values_dtype, const int32_t* row_ids, int32_t n_rows, espo_state* st,
                    const espo_params* params, int32_t* tokens_out, uint8_t* stop_out, void* stream);

/* Copy the sticky device status word (ESPO_DEV_* bits) to *host_out.  Synchronises `stream`. */
int espo_state_status(espo_state* st, uint32_t* host_out, void* stream);

/* TD errors and GAE over B ragged trajectories (Eq. 4-5) with ESPO's failure transition
 * (Eq. 13).  Trajectory i owns tokens [off_i, off_i + lengths[i]) of the packed arrays,
 * off = exclusive prefix sum of lengths.
 *   rewards, values  device float32 [total_tokens]
 *   lengths          device int32 [B] (>= 0; the stop-step token of a stopped trajectory is
 *                    its last token)
 *   stopped          device uint8 [B]: 1 = ended by ESPO's rule; its last reward is REPLACED
 *                    by r_fail
 *   total_tokens     host value of sum(lengths); a mismatch sets ESPO_DEV_BAD_LENGTHS
 *   adv_out          device float32 [total_tokens]
 * With r'_t the (possibly replaced) rewards and V_L := 0 for every trajectory (nothing is
 * bootstrapped past the last token): delta_t = r'_t + gamma V_{t+1} - V_t and
 * A_t = delta_t + gamma*lambda*A_{t+1}, A_L := 0.
 * Trajectories do not interact: a NaN or infinity among one trajectory's rewards or values
 * spoils that trajectory's advantages only.
 * Uses a per-device workspace that grows on demand: a call that needs more than any
 * earlier call (or espo_advantages_reserve) allocates device memory after synchronising
 * the device; otherwise nothing is allocated.  Calls on one device must not overlap.
 * Errors: NULL, BAD_SHAPE, ALIGN (arrays must be 16-byte aligned), CUDA. */
int espo_advantages(const float* rewards, const float* values, const int32_t* lengths,
                    const uint8_t* stopped, int32_t B, int64_t total_tokens,
                    float gamma, float lambda, float r_fail, float* adv_out, void* stream);

/* espo_advantages that also writes the value targets of the critic, returns_t = A_t + V(s_t) (the
 * lambda-return that goes with the GAE of Eq. 5), in the same pass.
 *   returns_out  device float32 [total_tokens], 16-byte aligned, or NULL (then exactly espo_advantages)
 * Everything else as for espo_advantages. */
int espo_advantages_returns(const float* rewards, const float* values, const int32_t* lengths,
                            const uint8_t* stopped, int32_t B, int64_t total_tokens,
                            float gamma, float lambda, float r_fail, float* adv_out,
                            float* returns_out, void* stream);

/* espo_advantages_returns that also leaves the two sums a trainer normalises ("whitens") a batch of advantages
 * with.  The paper does not normalise advantages (Sec. 3 uses the GAE of Eq. 5 as it is); this is the usual
 * PPO companion step, offered because the sums fall out of the same pass.
 *   stats_out    device float64 [2], 8-byte aligned, or NULL (then exactly espo_advantages_returns):
 *                stats_out[0] = sum_t A_t, stats_out[1] = sum_t A_t^2 over all total_tokens tokens, taken in
 *                double precision before the advantages are rounded to float32; mean = stats_out[0] / total_tokens,
 *                variance = stats_out[1] / total_tokens - mean^2.  With B == 0 or total_tokens == 0 both are set to 0.
 * Every CTA adds up its own tokens and the CTA that finishes last adds up the CTAs' sums in a fixed order, so
 * repeated calls on the same input give bit-identical sums.  Everything else as for espo_advantages. */
int espo_advantages_stats(const float* rewards, const float* values, const int32_t* lengths,
                          const uint8_t* stopped, int32_t B, int64_t total_tokens,
                          float gamma, float lambda, float r_fail, float* adv_out,
                          float* returns_out, double* stats_out, void* stream);

/* Pre-size the advantage workspace of the current device so that later calls with
 * B <= max_B and total_tokens <= max_tokens allocate nothing. */
int espo_advantages_reserve(int32_t max_B, int64_t max_tokens);

/* Copy the advantage workspace's sticky status word (ESPO_DEV_TIMEOUT, ESPO_DEV_BAD_LENGTHS)
 * of the current device to *host_out and clear it.  Synchronises `stream`. */
int espo_advantages_status(uint32_t* host_out, void* stream);

/* espo_advantages_returns for the padded layout: rewards, values and the outputs are [B, t_max] row-major and
 * trajectory i owns the first lengths[i] entries of row i (Eq. 4-5 and 13 as for espo_advantages; the layout is this
 * library's, the paper does not fix one).
 *   rewards, values  device float32 [B * t_max], 16-byte aligned; what the padding holds is never used (it may be
 *                    NaN)
 *   lengths          device int32 [B], 0 <= lengths[i] <= t_max; a value outside sets ESPO_DEV_BAD_LENGTHS and is
 *                    clamped
 *   adv_out          device float32 [B * t_max]; padding entries are written as 0
 *   returns_out      device float32 [B * t_max] or NULL; padding entries are written as 0
 * The pass writes all B * t_max entries and reads all but the 3072-entry chunks that lie wholly inside one row's
 * padding; a batch that is mostly padding is cheaper packed.  Workspace and errors as for espo_advantages. */
int espo_advantages_padded(const float* rewards, const float* values, const int32_t* lengths,
                           const uint8_t* stopped, int32_t B, int32_t t_max,
                           float gamma, float lambda, float r_fail, float* adv_out,
                           float* returns_out, void* stream);

/* Limits of espo_advantages_noalloc. */
#define ESPO_NOALLOC_MAX_B       4096          /* trajectories per call                          */
#define ESPO_NOALLOC_MAX_TOKENS  16777216      /* sum(lengths) per call (2^24)                   */

/* espo_advantages for callers that must not allocate device memory.  (The paper has no
 * counterpart of this entry point; it computes exactly what espo_advantages computes.)
 *
 * Who needs it: a rollout worker whose serving engine claimed all free device memory for its
 * own pools at start-up, so that a cudaMalloc issued by a library fails; and a training loop
 * that cannot afford the device-wide synchronisation that cudaMalloc/cudaFree imply.  This call
 * never calls cudaMalloc, cudaFree or any other allocating routine: its scratch is a fixed
 * array of about 55 KB that is part of the library image, so every device that loads the
 * library holds that array until the process exits.
 *
 * Arguments are those of espo_advantages, plus
 *   status_out   device uint32 [1] or NULL: ESPO_DEV_TIMEOUT / ESPO_DEV_BAD_LENGTHS bits are
 *                OR-ed into it (the caller clears it); with NULL they go to a word inside the
 *                scratch that cannot be read back.
 * Limits: B <= ESPO_NOALLOC_MAX_B and total_tokens <= ESPO_NOALLOC_MAX_TOKENS, otherwise
 * ESPO_ERR_CAPACITY and nothing is launched.
 * The first call on each device looks up the scratch array's device address (with that device
 * current) and remembers it; make that first call outside any stream capture.
 * All calls on a device share the one array and it keeps the previous call's contents; no
 * part of it has to start at zero, because each call rewrites every entry it later reads.
 * Two calls that overlap on the device (different streams, no dependency) race on it:
 * serialise them.
 * Errors: BAD_SHAPE, CAPACITY, NULL, ALIGN (16-byte arrays), BAD_PARAM, CUDA. */
int espo_advantages_noalloc(const float* rewards, const float* values, const int32_t* lengths,
                            const uint8_t* stopped, int32_t B, int64_t total_tokens,
                            float gamma, float lambda, float r_fail, float* adv_out,
                            uint32_t* status_out, void* stream);

/* ---- around the step: the key/value cache, attention over shared prompts, sampling from given numbers ----
 * A decode loop surrounds espo_step with the same three operations on the same trajectory slots: write the new token's
 * keys and values, attend over the prompt and the tokens generated so far, and (where the request rather than the
 * rollout batch chooses the sampling) draw the token.  The paper has none of them (its rollouts run inside a serving
 * engine, Sec. 5); its batch gives them their shape: 64 prompts x 8 rollouts, so eight rows share each prompt, and rows
 * leave one by one as the stop rule ends them -- every call takes the state's status array and leaves ended rows out. */

/* A paged key/value cache in caller-owned device memory.  Plain data, passed by host pointer, copied at call.
 *   k, v           device [n_pages, n_kv_heads, page_size, head_dim], element type dtype, 16-byte aligned
 *   k_exp, v_exp   ESPO_E4M3: device uint8 [n_pages, n_kv_heads, page_size], 16-byte aligned; ESPO_BF16: NULL
 *   page_size 16, 32, 64 or 128; head_dim 64 or 128; n_pages * n_kv_heads * page_size < 2^31
 *   dtype          ESPO_BF16, or ESPO_E4M3: the number stored is code * 2^(exp - 127), where the 8-bit code has 4
 *                  exponent and 3 mantissa bits (largest 448) and exp, 63 to 190, belongs to the (token, head) vector.  A
 *                  power of two loses nothing against a finer scale: the code's own relative step does not depend on it.
 * A "cache slot" is page * page_size + offset. */
typedef struct espo_kv_cache {
  void*    k;
  void*    v;
  uint8_t* k_exp;
  uint8_t* v_exp;
  int32_t  n_pages;
  int32_t  page_size;
  int32_t  n_kv_heads;
  int32_t  head_dim;
  int32_t  dtype;
  int32_t  reserved;
} espo_kv_cache;

/* Rotary position embedding.  For position p, pair i of the first rot_dim dims of a head turns by p * inv_freq[i]:
 *   (a, b) -> (a cos - b sin, b cos + a sin) * mscale;  the dims from rot_dim on are left alone.
 *   inv_freq     device float64 [rot_dim / 2], 8-byte aligned (espo_rope_frequencies computes them)
 *   rot_dim      a multiple of 8, 0 < rot_dim <= head_dim
 *   interleaved  0: pair i is dims (i, i + rot_dim/2); 1: dims (2i, 2i + 1) */
typedef struct espo_rope {
  const double* inv_freq;
  int32_t       rot_dim;
  int32_t       interleaved;
  float         mscale;
  int32_t       reserved;
} espo_rope;

/* The sequences of a rollout batch by trajectory slot: the tokens of the slot's group's prefix (the shared prompt),
 * followed by the slot's own.  Plain data, passed by host pointer, copied at call; the arrays are read on the device, so
 * a captured graph sees the lengths and tables of the moment it runs.
 *   pages, max_pages   device int32 [capacity, max_pages]: own token j of slot s lies in page pages[s][j / page_size]
 *   length             device int32 [capacity]: own tokens of the slot (>= 0)
 *   status             device uint8 [capacity] or NULL: slots whose status is not ESPO_ROW_ACTIVE are left out
 *                      (espo_state_view's array)
 *   group              device int32 [capacity] or NULL: the slot's group; < 0: none
 *   prefix_pages, max_prefix_pages, prefix_length, n_groups   device int32 [n_groups, max_prefix_pages], [n_groups];
 *                      needed with group */
typedef struct espo_sequences {
  const int32_t* pages;
  int32_t*       length;
  const uint8_t* status;
  const int32_t* group;
  const int32_t* prefix_pages;
  const int32_t* prefix_length;
  int32_t        max_pages;
  int32_t        capacity;
  int32_t        max_prefix_pages;
  int32_t        n_groups;
} espo_sequences;

#define ESPO_ROPE_PLAIN    0   /* theta^(-2i/rot_dim)                                                          */
#define ESPO_ROPE_LINEAR   1   /* the same divided by factor                                                   */
#define ESPO_ROPE_BY_PARTS 2   /* slow pairs divided by factor, fast ones kept, a ramp between                  */

/* Rotary frequencies, on the host, in 64 bits.  ESPO_ROPE_BY_PARTS stretches a context of original_length tokens by
 * factor: with dim(t) = rot_dim ln(original_length / (2 pi t)) / (2 ln theta), pairs up to floor(dim(fast_turns)) keep
 * their frequency, pairs from ceil(dim(slow_turns)) on are divided by factor, linear in between; its mscale is
 * 0.1 ln(factor) + 1 (1 otherwise).
 *   inv_freq_out  host double [rot_dim / 2];  mscale_out  host float or NULL
 * Errors: NULL, BAD_PARAM (kind, theta <= 1, rot_dim not a positive multiple of 8, factor < 1, original_length < 1,
 * slow_turns <= 0, fast_turns <= slow_turns; the last three for ESPO_ROPE_BY_PARTS only). */
int espo_rope_frequencies(int32_t kind, double theta, int32_t rot_dim, double factor, double original_length,
                          double fast_turns, double slow_turns, double* inv_freq_out, float* mscale_out);

/* Writes the keys and values of n_tokens tokens into the cache, rotating keys (and queries) on the way.
 *   key, value     device [n_tokens, n_kv_heads, head_dim], dtype ESPO_F32 or ESPO_BF16, tokens key_stride /
 *                  value_stride ELEMENTS apart (slices of a fused projection)
 *   cache_slots    device int32 [n_tokens]: where each token goes; a negative entry skips the token's cache write
 *                  (its query is still rotated); the others must be distinct: what a slot that is named twice
 *                  holds afterwards is unspecified, and may be parts of both tokens
 *   positions      device int32 [n_tokens]; needed with rope
 *   rope           host pointer or NULL (no rotation; positions unused)
 *   q, q_out       device [n_tokens, n_q_heads, head_dim] of the same dtype, or both NULL with n_q_heads 0; q_out may
 *                  be q
 *   status_out     device uint32 or NULL: ESPO_DEV_BAD_PAGE is OR-ed into it for a slot outside the cache (not written)
 * All base pointers 16-byte aligned, strides multiples of 8 elements and >= n_heads * head_dim.  The arithmetic is
 * 32-bit (angles: 64-bit), rounded once: to bf16, or to e4m3 with the smallest exponent in [-64, 63] that keeps the
 * vector's largest magnitude <= 448 * 2^e.  Infinite entries become the largest code, NaN stays NaN.
 * Enqueued on `stream`.  Errors: NULL, BAD_DTYPE, BAD_SHAPE, BAD_PARAM, ALIGN, CAPACITY, CUDA. */
int espo_kv_append(const espo_kv_cache* cache, const espo_rope* rope, const void* key, int64_t key_stride,
                   const void* value, int64_t value_stride, int32_t dtype, const int32_t* cache_slots,
                   const int32_t* positions, int32_t n_tokens, const void* q, int64_t q_stride, int32_t n_q_heads,
                   void* q_out, int64_t q_out_stride, uint32_t* status_out, void* stream);

/* The decode form of espo_kv_append: row i is the next token of slot row_ids[i] (NULL: slot i; slots distinct within a
 * call).  It goes to the slot's own position length[s] (position prefix_length[group] + length[s] for the rotation), and
 * length[s] is incremented on the device.  Rows whose slot is not active are left alone, q_out included; a row whose
 * pages are full sets ESPO_DEV_CACHE_FULL, and a slot id, group, page or length outside its range ESPO_DEV_BAD_SLOT /
 * ESPO_DEV_BAD_PAGE / ESPO_DEV_BAD_LENGTHS: its cache and length stay as they were (its q_out is unspecified). */
int espo_kv_append_rows(const espo_kv_cache* cache, const espo_rope* rope, const void* key, int64_t key_stride,
                        const void* value, int64_t value_stride, int32_t dtype, const espo_sequences* seqs,
                        const int32_t* row_ids, int32_t n_rows, const void* q, int64_t q_stride, int32_t n_q_heads,
                        void* q_out, int64_t q_out_stride, uint32_t* status_out, void* stream);

/* Reads cache entries back as the numbers they stand for.
 *   cache_slots    device int32 [n_tokens]; a negative entry gives zeros, one outside the cache zeros and
 *                  ESPO_DEV_BAD_PAGE
 *   k_out, v_out   device [n_tokens, n_kv_heads, head_dim] contiguous, dtype ESPO_F32 or ESPO_BF16 (both hold every
 *                  stored number exactly, subnormal bf16 numbers included), 16-byte aligned; either may be NULL
 * Errors: NULL, BAD_DTYPE, BAD_SHAPE, ALIGN, CUDA. */
int espo_kv_gather(const espo_kv_cache* cache, const int32_t* cache_slots, int32_t n_tokens, void* k_out, void* v_out,
                   int32_t dtype, uint32_t* status_out, void* stream);

/* Attention of one query token per row over prefix and own tokens, queries grouped over the key/value heads (query head
 * h reads key/value head h / (n_q_heads / n_kv_heads)):
 *   out[i, h] = sum_j softmax_j(scale * q[i, h] . k_j) v_j  over the group's prefix_length tokens and the slot's length.
 * The prefix is read once per run of consecutive rows of the same group, not once per row; rows of a group in any other
 * order are computed correctly, with the prefix read once per run.
 *   q, out         device bf16 [n_rows, n_q_heads, head_dim], rows q_stride / out_stride elements apart (multiples of 8,
 *                  >= n_q_heads * head_dim), 16-byte aligned; out must not overlap q
 *   n_q_heads      a multiple of n_kv_heads, at most 64 per key/value head
 *   row_ids        device int32 [n_rows] or NULL (row i = slot i)
 *   scale          at most 2^127 in magnitude; q . k itself, before the scale, has to be finite as a 32-bit float
 *   workspace      device, 256-byte aligned, at least espo_attention_workspace bytes; calls that share one must not
 *                  overlap on the device
 *   status_out     device uint32 or NULL: ESPO_DEV_BAD_SLOT, BAD_PAGE (page or group; the page's tokens, or the row's
 *                  prefix, are left out), BAD_LENGTHS (clamped to 0 .. the table's tokens), TIMEOUT are OR-ed into it
 * Rows that are not active (or whose slot id is out of range) keep what out held.  A row without tokens gives zeros.
 * What the cache holds beyond a sequence's tokens is never used (it may be NaN).  Scores, the running maximum, the sums
 * and the output's accumulation are 32-bit; the weights are rounded to 16 bits for the product with v (bf16; fp16 for the
 * own tokens of an e4m3 cache), the output once to bf16.
 * Enqueued on `stream`.  Errors: NULL, BAD_DTYPE, BAD_SHAPE, BAD_PARAM, ALIGN, CAPACITY (workspace_bytes; n_rows above the
 * sequences' capacity), CUDA. */
int espo_attention(const espo_kv_cache* cache, const espo_sequences* seqs, const void* q, int64_t q_stride,
                   int32_t n_q_heads, const int32_t* row_ids, int32_t n_rows, float scale, void* out, int64_t out_stride,
                   void* workspace, int64_t workspace_bytes, uint32_t* status_out, void* stream);

/* Bytes of workspace that espo_attention needs for up to n_rows rows, written to *bytes_out (host).
 * Errors: NULL, BAD_SHAPE, BAD_DTYPE, BAD_PARAM, ALIGN, CUDA. */
int espo_attention_workspace(const espo_kv_cache* cache, int32_t n_rows, int32_t n_q_heads, int64_t* bytes_out);

/* One token per row from given random numbers, every row with its own sampling parameters (the request's, where
 * espo_step has one set per rollout batch and draws its own noise).  It stands in place of espo_step's draw, not before it:
 * the step scores the token that it draws itself, so a rollout that early stopping watches takes its tokens from the step, and
 * this call serves rows without it (evaluation, requests with parameters of their own).  With w_a = exp((x_a - max x) / T),
 * Z their sum, and A(a), n(a) the mass and the number of ids strictly more probable than a, the support is
 *   { a : x_a > -inf,  A(a) < top_p Z,  n(a) < top_k,  w_a >= min_p }
 * (the rule of espo_params.top_p / top_k, so equally probable ids stay or go together), and the token is the lowest
 * supported id whose running sum of supported weights, in id order, exceeds u times their total.
 *   logits         device [n_rows, V], element type logits_dtype, rows row_stride elements apart (>= V); entries may be
 *                  -inf
 *   u              device float32 [n_rows] in [0, 1)
 *   temperature    device float32 [n_rows] or NULL (1); 0 = the lowest id of the largest logit, log-probability 0
 *   top_k          device int32 [n_rows] or NULL; <= 0: no filter
 *   top_p, min_p   device float32 [n_rows] or NULL; outside (0, 1): no filter (min_p: outside (0, 1]; NaN: no filter)
 *   row_ids        device int32 [n_rows] or NULL;  status  device uint8 [capacity] or NULL: row i belongs to slot
 *                  row_ids[i] (i), and gets token -1, logp untouched, if its status is not ESPO_ROW_ACTIVE
 *   tokens_out     device int32 [n_rows]
 *   logp_out       device float32 [n_rows] or NULL: ln(w_token / sum of supported weights)
 *   workspace      device, 256-byte aligned, at least espo_sample_workspace bytes; calls that share one must not overlap
 *                  on the device
 *   status_out     device uint32 or NULL: ESPO_DEV_BAD_ROW is OR-ed into it for an unusable row (NaN or +inf logit,
 *                  nothing finite, the largest within 140 T of the lowest float, u outside [0, 1) or NaN,
 *                  temperature negative, above 1e30 or NaN): token 0, logp NaN;
 *                  ESPO_DEV_BAD_SLOT for a slot outside [0, capacity): token -1; ESPO_DEV_TIMEOUT if a bounded wait
 *                  ran out (that row: token 0, logp NaN)
 * Weights and their sums are 64-bit (exponential: relative error below 2^-38; min_p compares x_a - max x with T ln min_p
 * instead); inside a support found by a filter they are
 * rounded to multiples of 2^-42 of the largest one and added up as integers, so that the token does not depend on the order
 * of the additions; an id whose weight is below 2^-43 of the largest is not drawn there.
 * V at most 2^19.  Enqueued on `stream`.  Errors: NULL, BAD_DTYPE, BAD_SHAPE, ALIGN, CAPACITY (V,
 * workspace_bytes), CUDA. */
int espo_sample(const void* logits, int32_t logits_dtype, int64_t row_stride, int32_t n_rows, int32_t V, const float* u,
                const float* temperature, const int32_t* top_k, const float* top_p, const float* min_p,
                const int32_t* row_ids, const uint8_t* status, int32_t capacity, int32_t* tokens_out, float* logp_out,
                void* workspace, int64_t workspace_bytes, uint32_t* status_out, void* stream);

/* Bytes of workspace that espo_sample needs for up to n_rows rows of V ids, written to *bytes_out (host).
 * Errors: NULL, BAD_SHAPE, CAPACITY (V). */
int espo_sample_workspace(int32_t n_rows, int32_t V, int64_t* bytes_out);

/* Text for a return code; never NULL. */
const char* espo_strerror(int code);

/* The last cudaError_t (as int) seen by this library on the calling thread, 0 if none. */
int espo_last_cuda_error(void);

#ifdef __cplusplus
}
#endif
#endif /* ESPO_H_ */
