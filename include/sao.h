/*
 * sao.h -- C ABI of the SAO per-token RL loss head on one GB300 (sm_103a).
 *
 * The operations follow "Single-Rollout Asynchronous Optimization for Agentic
 * Reinforcement Learning" (arxiv 2607.07508):
 *   - sao_token_logprobs_fwd/bwd : log pi_theta(a_t|s_t) of Eq. 1-2 from the
 *     LM head (logits H W^T, log-softmax, gather), vocabulary-chunked so the
 *     [N, V] logits are never stored, and its gradient;
 *   - sao_policy_loss_fwd/bwd    : the DIS ratio of Eq. 2 against the rollout
 *     log-probs, the strict double-sided calibration f of Eq. 3 and the token
 *     objective of Eq. 1 (§3.1), with the clip-ratio counts of §4.4;
 *   - sao_advantages             : token-level GAE (Preliminaries) with the
 *     skip-observation link of Eq. 4-5 (§3.2) and the length-adaptive lambda
 *     of §4.1, as a reverse scan over packed trajectories;
 *   - sao_value_loss             : the value error (V - R)^2 (Preliminaries)
 *     and the explained-variance sums of §4.4.
 * Beside them, auxiliary losses of the same training step:
 *   - sao_distill_loss_fwd/bwd   : distillation from a teacher's top logits
 *     over the LM head;
 *   - sao_balance_loss_fwd/bwd   : load balance of a mixture of experts.
 * And what stands directly around the losses in that step:
 *   - sao_route_fwd/bwd          : a router's choice of experts and their weights;
 *   - sao_rms_norm_fwd/bwd       : the root-mean-square norm in front of the LM
 *     head, of the residual stream's sum, in 8 bits too;
 *   - sao_grad_sumsq, sao_grad_clip : the global norm of all gradients, clipping.
 *
 * Conventions shared by every entry point:
 *   - Every array argument is a DEVICE pointer owned by the caller; the
 *     library never allocates, frees or keeps a pointer past the call.
 *   - Scratch space comes from the caller's workspace `ws` of `ws_bytes`
 *     bytes, 256-byte aligned, of at least sao_workspace_bytes(...) bytes.
 *     Its contents on entry do not matter; one workspace must not be used by
 *     two calls that overlap on the GPU.
 *   - Each call only enqueues kernels on `stream` (a cudaStream_t; NULL is
 *     the legacy default stream) and returns without waiting, unless checked
 *     mode is on (sao_set_checked), in which case it synchronises the stream
 *     and reports device-side validation failures as SAO_ERR_DEVICE_CHECK.
 *   - Errors are returned as sao_status; no exception crosses the ABI; the
 *     last error message is available from sao_last_error_string().
 *   - N is the number of packed tokens; row t of H predicts token y[t] (the
 *     caller does the shift). Per-token floating point arrays are fp32;
 *     token ids and cu_seqlens are int32; counts are int64.
 *   - Arrays are contiguous (row-major for matrices). Vectorised paths need
 *     16-byte aligned pointers; other alignments take a scalar path.
 */
#ifndef SAO_H_
#define SAO_H_

#include <stddef.h>
#include <stdint.h>

#if defined(__GNUC__)
#define SAO_API __attribute__((visibility("default")))
#else
#define SAO_API
#endif

#ifdef __cplusplus
extern "C" {
#endif

typedef struct CUstream_st *sao_stream_t; /* a cudaStream_t */

typedef enum sao_status {
  SAO_OK = 0,
  SAO_ERR_INVALID_ARG = 1,  /* null pointer, bad scalar, misaligned workspace */
  SAO_ERR_SHAPE = 2,        /* inconsistent or unsupported sizes */
  SAO_ERR_WORKSPACE = 3,    /* ws_bytes smaller than required */
  SAO_ERR_UNSUPPORTED = 4,  /* dtype, or a device that is not sm_103 */
  SAO_ERR_CUDA = 5,         /* a CUDA runtime or driver call failed */
  SAO_ERR_DEVICE_CHECK = 6  /* checked mode: the device flagged bad input */
} sao_status;

typedef enum sao_dtype {
  SAO_F32 = 0,   /* fp32 H, W, dH: tensor cores on three bf16 pieces per operand, fp32 sums (pieces exact for
                    2^-110 <= |a| < 2^100; |a| off by up to 2^-134 below, fp32 FMA products above) */
  SAO_BF16 = 1   /* bf16 H, W, dH (tcgen05 tensor-core path, fp32 accumulate) */
} sao_dtype;

/* Per-token flag values written by sao_policy_loss_fwd (Eq. 3). */
#define SAO_FLAG_IN 0        /* 1 - eps_low < r < 1 + eps_high: kept, f(r) = r */
#define SAO_FLAG_LOW 1       /* r <= 1 - eps_low: masked, f(r) = 0 */
#define SAO_FLAG_HIGH 2      /* r >= 1 + eps_high: masked, f(r) = 0 */
#define SAO_FLAG_NONFINITE 3 /* log-ratio or advantage not finite: masked */
#define SAO_FLAG_NOT_ACTION 4/* loss_mask == 0 (prompt / observation token) */

/* Device-side error bits (checked mode), OR-ed into one word. */
#define SAO_DEVERR_TOKEN_ID 0x1u     /* some y[t] outside [0, V) */
#define SAO_DEVERR_CU_SEQLENS 0x2u   /* cu_seqlens not 0..N non-decreasing */
#define SAO_DEVERR_SCAN_TIMEOUT 0x4u /* advantage scan gave up waiting for a carry */
#define SAO_DEVERR_PIPE_TIMEOUT 0x8u /* a GEMM pipeline wait gave up */
#define SAO_DEVERR_CACHE_ROW 0x10u   /* cached backward: a row with grad != 0 the forward skipped */
#define SAO_DEVERR_TOP_ID 0x20u      /* a teacher's entry with an id >= V, or one id twice in a row */
#define SAO_DEVERR_EXPERT_ID 0x40u   /* some expert id >= E */
#define SAO_DEVERR_LOGITS 0x80u      /* a row of router logits without scores (NaN, +inf under softmax) */

/* Library version, major * 10000 + minor * 100 + patch. */
SAO_API int sao_version(void);

/* Message for the most recent non-OK status on the calling host thread. */
SAO_API const char *sao_last_error_string(void);

/* Checked mode (off by default): every call synchronises its stream, reads
 * and clears the device error word, and returns SAO_ERR_DEVICE_CHECK if it is
 * non-zero. Process-wide setting. */
SAO_API void sao_set_checked(int on);
SAO_API int sao_get_checked(void);

/* Upper bound on the dZ buffer of sao_token_logprobs_bwd (default 4 GiB, at
 * least 1 MiB; fp32 heads: on the three bf16 pieces of dZ and, beside them, on
 * those of the chunk of W that a call splits at a time, never less than 256
 * columns). The backward never holds dZ for all N x V logits: it works on blocks
 * of rows times chunks of the vocabulary whose bf16 dZ fits the budget (one
 * block and one chunk when N x V does), choosing the split with the least extra
 * traffic (an fp32 dH accumulator read and written once
 * per extra vocabulary chunk; dW added to once per extra row block). The parts
 * that a product of few tiles is cut into (fp32: up to 16 copies of the chunk of
 * dW or of dH; one of dW too where h is not a multiple of 8) take workspace beside
 * it. Affects sao_workspace_bytes. Process-wide. */
SAO_API void sao_set_dz_budget_bytes(size_t bytes);
/* The current bound (bytes) set by sao_set_dz_budget_bytes or the default. */
SAO_API size_t sao_get_dz_budget_bytes(void);

/* Tiling of the bf16 tensor-core GEMMs (process-wide; default 0). on = 1:
 * CTA pairs, clusters of 2 CTAs sharing each tcgen05.mma.cta_group::2 of
 * M = 256 (each CTA loads its own 128 rows of A and half of the B tile); on =
 * 0: single CTAs with M = 128 MMAs. Results agree to within the fp32
 * accumulation order. On one GB300 under its power cap the pairs do about 3 %
 * more work per SM clock but run at a lower clock, and the moe step takes
 * 2.5 % longer, hence the default. Affects later calls only. */
SAO_API void sao_set_cta_pairs(int on);
SAO_API int sao_get_cta_pairs(void);

/*
 * Test hooks of the advantage scan (process-wide; defaults restored by
 * (0, 0)): every look-back wait gives up after wait_ns nanoseconds (0: the
 * default 2 s; longer values are capped at it), and the scan's top
 * skip_chunks chunks (of 1024, 2048 or 4096 tokens, chosen from N) are never
 * processed, so the chunks below them
 * wait for a carry that never comes. Failure-detection tests use them to make
 * the bounded wait run out: the call still completes, the context stays
 * usable, and checked mode reports SAO_DEVERR_SCAN_TIMEOUT. Not for
 * production use (the skipped chunks' outputs are left unwritten).
 */
SAO_API void sao_debug_set_scan_hooks(uint64_t wait_ns, int32_t skip_chunks);

/* Workspace bytes that every entry point needs for N tokens, hidden size h,
 * vocabulary V and dtype dt (pass h = V = 0 when only the O(N) calls are
 * used). Returns 0 for invalid sizes. */
SAO_API size_t sao_workspace_bytes(int64_t N, int32_t h, int32_t V, sao_dtype dt);

/*
 * Eq. 1-2: logp[t] = z[t, y[t]] - lse[t], z = H W^T, lse[t] = log sum_v e^z[t,v].
 *   H        [N, h] dt, row-major          W  [V, h] dt, row-major
 *   y        [N] int32 in [0, V)           row_mask [N] uint8 or NULL: rows
 *            with row_mask[t] == 0 are not computed and get logp = lse = 0
 *   logp,lse [N] fp32 outputs (lse is kept for the backward)
 * Sizes: N >= 0; 1 <= V; h >= 1; for bf16, h % 8 == 0 (TMA row pitch).
 * A token id outside [0, V) yields logp = NaN (and SAO_DEVERR_TOKEN_ID).
 */
SAO_API sao_status sao_token_logprobs_fwd(const void *H, const void *W, sao_dtype dt, const int32_t *y,
                                  const uint8_t *row_mask, int64_t N, int32_t h, int32_t V,
                                  float *logp, float *lse, void *ws, size_t ws_bytes,
                                  sao_stream_t stream);

/*
 * Gradient of sum_t G[t] * logp[t] (G = grad_logp): with p = e^(z - lse),
 * dZ[t, v] = G[t] * (1[v == y[t]] - p[t, v]); dH = dZ W; dW = dZ^T H.
 *   lse       [N] fp32 from sao_token_logprobs_fwd on the same H, W, y
 *   grad_logp [N] fp32; rows with grad_logp == 0 contribute nothing
 *   dH        [N, h] dt output (overwritten)
 *   dW        [V, h] fp32 output; overwritten if accumulate_dW == 0, else
 *             the gradient is added to its contents
 */
SAO_API sao_status sao_token_logprobs_bwd(const void *H, const void *W, sao_dtype dt, const int32_t *y,
                                  const float *lse, const float *grad_logp, int64_t N, int32_t h,
                                  int32_t V, void *dH, float *dW, int accumulate_dW, void *ws,
                                  size_t ws_bytes, sao_stream_t stream);

/*
 * The same two calls with the forward's probabilities kept for the backward
 * (bf16 only), so the backward needs neither the logits nor dZ in memory.
 * For every row it computes, the forward takes a shift kappa = z[t, y] + 20
 * (the sampled token's logit, from a pre-pass) and stores e[t, v] = exp(z[t,
 * v] - kappa) in bf16; once lse is known, the entry at v = y becomes e[t, y] -
 * exp(lse - kappa). Then dZ[t, .] = -G[t] exp(kappa - lse[t]) e[t, .], and the
 * backward is two GEMMs on e: dH = (e W) scaled per row, dW = e^T (s H). A row
 * with some z[t, v] more than 60 above z[t, y] (p_y below e^-60) would
 * overflow that range: the forward flags it (its lse and log-prob are still
 * exact) and the backward recomputes that row's logits. The results match
 * sao_token_logprobs_fwd / _bwd within the bf16 rounding of e and of s H.
 *   cache        caller-owned device buffer of sao_logprob_cache_bytes(N, V)
 *                bytes (about 2 N V bytes), 256-byte aligned; written by the
 *                forward, read (not modified) by the backward, which must get
 *                the same H, W, y, N, V and the forward's lse
 * A backward row with grad_logp != 0 that the forward skipped (row_mask 0)
 * has no stored probabilities: it contributes nothing and raises
 * SAO_DEVERR_CACHE_ROW. Other arguments as the uncached calls; SAO_F32 gives
 * SAO_ERR_UNSUPPORTED.
 */
SAO_API size_t sao_logprob_cache_bytes(int64_t N, int32_t V);
SAO_API sao_status sao_token_logprobs_fwd_cached(const void *H, const void *W, sao_dtype dt, const int32_t *y,
                                                 const uint8_t *row_mask, int64_t N, int32_t h, int32_t V,
                                                 float *logp, float *lse, void *cache, size_t cache_bytes, void *ws,
                                                 size_t ws_bytes, sao_stream_t stream);
SAO_API sao_status sao_token_logprobs_bwd_cached(const void *H, const void *W, sao_dtype dt, const int32_t *y,
                                                 const float *lse, const float *grad_logp, int64_t N, int32_t h,
                                                 int32_t V, void *dH, float *dW, int accumulate_dW,
                                                 const void *cache, size_t cache_bytes, void *ws, size_t ws_bytes,
                                                 sao_stream_t stream);

/*
 * Skip-observation GAE (Preliminaries; §3.2 Eq. 4-5; §4.1). For trajectory b
 * (tokens cu_seqlens[b] .. cu_seqlens[b+1]-1) only action tokens
 * (loss_mask == 1) take part; the Bellman successor of an action token is the
 * next action token of the same trajectory, skipping observation tokens; the
 * value after the last action token is 0 and rewards[b] is the reward of the
 * last action token. delta_j = r_j + gamma V_next - V_j,
 * A_j = delta_j + gamma lambda_b A_next, ret_j = GAE(lambda_critic)_j + V_j.
 * lambda_b = lambda_policy, or 1 - 1/(alpha * L_b) clamped to [0,1] when
 * len_adaptive_alpha = alpha > 0 (L_b = number of action tokens of b).
 * Non-action tokens get adv = ret = 0. Computed in double-float (about 48
 * significant bits) and rounded to fp32.
 *   values [N] fp32, rewards [B] fp32, loss_mask [N] uint8,
 *   cu_seqlens [B+1] int32 with 0 = cu[0] <= ... <= cu[B] = N
 *   adv, ret [N] fp32 outputs
 * Scalars: 0 <= gamma, lambda_policy, lambda_critic <= 1.
 * Arrays that start 16-byte aligned move by TMA tensor copies; other
 * alignments are staged element by element (same results, slower).
 * The scan keeps each chunk's values in TMEM between its two passes: while it
 * runs, each SM's 512 TMEM columns are held by its CTAs, so a kernel on
 * another stream that allocates TMEM on the same SM waits for them (and the
 * scan waits for such a kernel's columns); neither depends on the other's
 * progress, so the wait always ends.
 */
SAO_API sao_status sao_advantages(const float *values, const float *rewards, const uint8_t *loss_mask,
                          const int32_t *cu_seqlens, int32_t B, int64_t N, float gamma,
                          float lambda_policy, float lambda_critic, float len_adaptive_alpha,
                          float *adv, float *ret, void *ws, size_t ws_bytes, sao_stream_t stream);

/* Step value definitions of sao_step_advantages (App. A.1). */
#define SAO_STEP_AVERAGE 0 /* V(S) = mean of the step's token values; every step token is a value-loss token */
#define SAO_STEP_LAST 1    /* V(S) = value of the step's last token; only that token is a value-loss token */

/*
 * Step-level GAE (App. A.1, "RL with Agentic Step as Action"). A step is one
 * conversation turn: a maximal run of action tokens (loss_mask == 1) inside a
 * trajectory. With V(S_i) per `mode`, the terminal reward on the last step and
 * the step value after the last step 0: delta_i = r_i + gamma V(S_{i+1}) -
 * V(S_i), A_i = delta_i + gamma lambda A_{i+1} where lambda = lambda_policy,
 * or 1 - 1/(alpha * number of steps) clamped to [0,1] when
 * len_adaptive_alpha = alpha > 0 (the length-adaptive rule counted in steps).
 * Every token of step i receives adv = A_i and ret = GAE(lambda_critic)_i +
 * V(S_i); other tokens get 0. value_mask (nullable, [N] uint8) marks the
 * tokens the value loss keeps: all step tokens (SAO_STEP_AVERAGE) or the last
 * token of each step (SAO_STEP_LAST). Per-step sums are compensated fp32
 * pairs and the step recursion runs in double-float (about 48 bits each; the
 * fp64 pipe is not used), then each result is rounded once to fp32.
 * Arguments otherwise as sao_advantages; workspace from sao_workspace_bytes.
 */
SAO_API sao_status sao_step_advantages(const float *values, const float *rewards, const uint8_t *loss_mask,
                                       const int32_t *cu_seqlens, int32_t B, int64_t N, float gamma,
                                       float lambda_policy, float lambda_critic, float len_adaptive_alpha, int mode,
                                       float *adv, float *ret, uint8_t *value_mask, void *ws, size_t ws_bytes,
                                       sao_stream_t stream);

/* Normalisation of sao_clip_loss_fwd/bwd (Preliminaries, unified objective). */
#define SAO_NORM_TOKEN 0    /* mean over all action tokens of the batch */
#define SAO_NORM_SEQUENCE 1 /* 1/|y| mean inside each trajectory, then the mean over trajectories */

/*
 * Clipped surrogate of the Preliminaries' unified objective with asymmetric
 * ("clip-higher") bounds: the loss of the paper's PPO/GRPO comparison arms
 * (§4.2; "GRPO w/ DIS" passes rollout log-probs as old_logp). With
 * r_t = exp(logp_t - old_logp_t):
 *   loss = -sum_t w_t min(r_t adv_t, clip(r_t, 1 - eps_low, 1 + eps_high) adv_t)
 * over action tokens, w_t = 1/(action tokens) for SAO_NORM_TOKEN, or
 * 1/(|y_b| * trajectories with an action token) for SAO_NORM_SEQUENCE. A token
 * is clipped when the min takes the clipped term strictly (adv > 0 and
 * r > 1 + eps_high: flag 2; adv < 0 and r < 1 - eps_low: flag 1), decided in
 * fp32; clipped tokens have coef = 0, others coef = d loss / d logp =
 * -w_t r_t adv_t. Non-finite tokens: flag 3, masked. counts = {n_action,
 * n_clip_low, n_clip_high, n_nonfinite}. coef and flags may be NULL.
 * cu_seqlens [B+1] as for sao_advantages (used by both normalisations).
 */
SAO_API sao_status sao_clip_loss_fwd(const float *logp, const float *old_logp, const float *adv,
                                     const uint8_t *loss_mask, const int32_t *cu_seqlens, int32_t B, int64_t N,
                                     float eps_low, float eps_high, int norm, float *loss, float *coef,
                                     uint8_t *flags, int64_t *counts, void *ws, size_t ws_bytes, sao_stream_t stream);

/* grad_logp[t] = grad_loss[0] * coef[t] of sao_clip_loss_fwd, recomputed. */
SAO_API sao_status sao_clip_loss_bwd(const float *logp, const float *old_logp, const float *adv,
                                     const uint8_t *loss_mask, const int32_t *cu_seqlens, int32_t B, int64_t N,
                                     float eps_low, float eps_high, int norm, const float *grad_loss,
                                     float *grad_logp, void *ws, size_t ws_bytes, sao_stream_t stream);

/*
 * GRPO's group-normalised advantage (Preliminaries): for trajectory b in
 * group g = group_ids[b], A_b = (R_b - mean_g R) / sqrt(var_g R + eps_stab)
 * (population variance over the group's trajectories: sums in compensated
 * fp32, about 48 bits, the final moments in fp64), broadcast to b's
 * action tokens; every other token gets 0. Cost O(B^2 / SMs) for the group
 * statistics (deterministic), then O(N).
 */
SAO_API sao_status sao_group_advantages(const float *rewards, const int32_t *group_ids, int32_t B,
                                        const uint8_t *loss_mask, const int32_t *cu_seqlens, int64_t N,
                                        float eps_stab, float *adv, void *ws, size_t ws_bytes, sao_stream_t stream);

/*
 * Running-mean reward baseline, the single-rollout alternative to a value
 * model in the ablations (§4.3: window of the 8 most recent rewards of each
 * prompt; §4.5: one window of the 128 most recent rewards, i.e. one prompt
 * id for all). Trajectories are taken in batch order: the baseline of b is
 * the mean of the at most `window` most recent rewards recorded for prompt
 * prompt_ids[b] before b (0 if none), A_b = R_b - baseline is written to b's
 * action tokens (0 elsewhere), then R_b enters that prompt's window.
 *   history [num_prompts, window] fp32 and seen [num_prompts] int64: the
 *   windows (ring buffers indexed by seen % window) and the number of rewards
 *   recorded per prompt; caller-owned device state, updated in place (zero
 *   both before the first batch). prompt_ids in [0, num_prompts); a
 *   trajectory with an id outside that range gets advantage 0 and is not
 *   recorded.
 */
SAO_API sao_status sao_running_mean_advantages(const float *rewards, const int32_t *prompt_ids, int32_t B,
                                               int32_t num_prompts, float *history, int64_t *seen, int32_t window,
                                               const uint8_t *loss_mask, const int32_t *cu_seqlens, int64_t N,
                                               float *adv, void *ws, size_t ws_bytes, sao_stream_t stream);

/* Extra per-token flag values written by sao_decoupled_loss_fwd. */
#define SAO_FLAG_MISMATCH_LOW 5  /* w = pi_old / pi_rollout <= w_low: masked */
#define SAO_FLAG_MISMATCH_HIGH 6 /* w >= w_high: masked */

/*
 * Decoupled three-policy objective, the mechanism that DIS simplifies (§3.1:
 * pi_theta / pi_old corrects staleness, pi_old / pi_rollout the training /
 * rollout mismatch, and tokens whose mismatch leaves a band are masked). With
 *   r_t = exp(logp_t - prox_logp_t)          (pi_theta / pi_old)
 *   w_t = exp(prox_logp_t - rollout_logp_t)  (pi_old / pi_rollout)
 * a token is kept when it is an action token, both log-ratios and adv_t are
 * finite and w_low < w_t < w_high (strict); then
 *   loss = -(1/n) sum_t w_t min(r_t adv_t, clip(r_t, 1 - eps_low, 1 + eps_high) adv_t)
 * with n = n_norm if n_norm > 0, else the number of action tokens. w is a
 * detached coefficient: coef_t = d loss / d logp_t = -w_t r_t adv_t / n when
 * the min keeps r_t adv_t (flag 0), and 0 when it is clipped (flag 1: adv < 0
 * and r < 1 - eps_low; flag 2: adv > 0 and r > 1 + eps_high) or the token is
 * masked (flags 3-6). Decisions are taken in fp32, the band before the clip.
 *   logp, prox_logp, rollout_logp, adv [N] fp32; loss_mask [N] uint8
 *   loss [1] fp32, coef [N] fp32 (nullable), flags [N] uint8 (nullable)
 *   counts [6] int64 = {n_action, n_clip_low, n_clip_high, n_nonfinite,
 *                       n_mismatch_low, n_mismatch_high}
 * Scalars: eps_low, eps_high >= 0; 0 <= w_low < w_high (w_high may be +inf).
 * Workspace from sao_workspace_bytes. Deterministic (fixed-order reductions).
 */
SAO_API sao_status sao_decoupled_loss_fwd(const float *logp, const float *prox_logp, const float *rollout_logp,
                                          const float *adv, const uint8_t *loss_mask, int64_t N, float eps_low,
                                          float eps_high, float w_low, float w_high, int64_t n_norm, float *loss,
                                          float *coef, uint8_t *flags, int64_t *counts, void *ws, size_t ws_bytes,
                                          sao_stream_t stream);

/* grad_logp[t] = grad_loss[0] * coef[t] of sao_decoupled_loss_fwd, recomputed
 * from the inputs (stateless); grad_loss is a device scalar. */
SAO_API sao_status sao_decoupled_loss_bwd(const float *logp, const float *prox_logp, const float *rollout_logp,
                                          const float *adv, const uint8_t *loss_mask, int64_t N, float eps_low,
                                          float eps_high, float w_low, float w_high, int64_t n_norm,
                                          const float *grad_loss, float *grad_logp, void *ws, size_t ws_bytes,
                                          sao_stream_t stream);

/*
 * sao_advantages without a workspace argument, for callers that cannot
 * allocate device memory: a host library that is handed only data pointers
 * and a stream by another framework and has no allocator of its own, or a
 * process that reserves all device memory at start-up and forbids later
 * allocations (cudaMalloc also synchronises the whole device, which a
 * latency-critical caller cannot afford). The paper has no counterpart to
 * this entry point; it computes exactly what sao_advantages computes.
 *
 * Scratch: a fixed 16 MiB array inside this library's device image, present on
 * every GPU that loads the library until the process exits. It bounds the
 * sizes: about 200 bytes per 1024 tokens plus 36 bytes per trajectory must
 * fit (for example 2^25 tokens with up to 65,536 trajectories); larger
 * inputs return SAO_ERR_SHAPE with the bytes needed. Nothing is allocated
 * and nothing is freed.
 * Each call made outside stream capture looks up the array's device address
 * (with the calling thread's current device) and remembers it for that
 * device, so a device reset or a new primary context is picked up; a call
 * under stream capture uses the remembered address and returns
 * SAO_ERR_INVALID_ARG if no call on that device came before the capture.
 * Every call on a device shares the one array, so calls that overlap
 * on the GPU (two streams, or two threads) race and corrupt each other's
 * results; serialise them. Each call clears the parts of the array that must
 * start at zero, so stale contents from a previous call do no harm.
 */
SAO_API sao_status sao_advantages_noalloc(const float *values, const float *rewards, const uint8_t *loss_mask,
                                          const int32_t *cu_seqlens, int32_t B, int64_t N, float gamma,
                                          float lambda_policy, float lambda_critic, float len_adaptive_alpha,
                                          float *adv, float *ret, sao_stream_t stream);

/*
 * Eq. 1-3 (§3.1). r_t = exp(logp_t - old_logp_t); a token is kept iff it is an
 * action token, its log-ratio and advantage are finite and
 * 1 - eps_low < r_t < 1 + eps_high (strict; decided in fp32). With n = n_norm
 * if n_norm > 0, else the number of action tokens:
 *   loss    = -(1/n) sum_{kept t} r_t adv_t            [1] fp32 output
 *   coef[t] = d loss / d logp_t = -r_t adv_t / n (kept), 0 otherwise (f(r) is
 *             a detached coefficient)                   [N] fp32 output
 *   flags[t]  SAO_FLAG_* value                          [N] uint8 output
 *   counts  = {n_action, n_low, n_high, n_nonfinite}    [4] int64 output
 * coef and flags may be NULL. The reductions are deterministic.
 * Scalars: eps_low >= 0 (eps_low >= 1 disables the lower bound), eps_high >= 0.
 */
SAO_API sao_status sao_policy_loss_fwd(const float *logp, const float *old_logp, const float *adv,
                               const uint8_t *loss_mask, int64_t N, float eps_low, float eps_high,
                               int64_t n_norm, float *loss, float *coef, uint8_t *flags,
                               int64_t *counts, void *ws, size_t ws_bytes, sao_stream_t stream);

/*
 * grad_logp[t] = grad_loss[0] * coef[t], with coef recomputed from the same
 * inputs as sao_policy_loss_fwd (stateless). grad_loss is a device scalar.
 */
SAO_API sao_status sao_policy_loss_bwd(const float *logp, const float *old_logp, const float *adv,
                               const uint8_t *loss_mask, int64_t N, float eps_low, float eps_high,
                               int64_t n_norm, const float *grad_loss, float *grad_logp, void *ws,
                               size_t ws_bytes, sao_stream_t stream);

/*
 * Value loss (Preliminaries, PPO): over the action tokens, with n = n_norm if
 * n_norm > 0, else the number of action tokens,
 *   loss = (1/n) sum_t (V_t - ret_t)^2           [1] fp32 output
 *   grad_values[t] = 2 (V_t - ret_t) / n, 0 on non-action tokens   [N] fp32
 *   ev_sums = {sum (R-V), sum (R-V)^2, sum R, sum R^2} over action tokens
 *             ([4] fp64, may be NULL), from which explained variance
 *             EV = 1 - Var(R - V) / Var(R) (§4.4) follows.
 * n_norm is the normaliser shared by data-parallel ranks (the action tokens
 * of the whole batch), as for the policy loss: the ranks' losses and
 * gradients then add up to those of the unsplit batch. With n_norm > 0 the
 * call makes one pass over the tokens; otherwise it counts them first.
 */
SAO_API sao_status sao_value_loss(const float *values, const float *ret, const uint8_t *loss_mask,
                          int64_t N, int64_t n_norm, float *loss, float *grad_values, double *ev_sums,
                          void *ws, size_t ws_bytes, sao_stream_t stream);

/* Most entries a row that sao_distill_loss_fwd/bwd take. */
#define SAO_DISTILL_MAX_K 1024

/*
 * Distillation from a teacher's top logits over the LM head (an auxiliary loss
 * beside the RL objective; the paper has no counterpart). Row t of the student
 * has logits z_v = H_t . W_v / T over the vocabulary; the teacher gives K
 * entries a row, ids with logits, of which those with a negative id are none
 * (a row that the teacher answered with fewer). With a_k = top_logits / T:
 *   la   = log sum_k e^a_k (teacher_lse NULL: the entries are renormalised), or
 *          teacher_lse[t] = the teacher's log sum e^(logit / T) over its whole
 *          vocabulary, whose mass outside the entries is then one more outcome:
 *   p_k  = e^(a_k - la),  rho = max(0, 1 - sum_k p_k)  (renormalised: 0)
 *   loss[t] = sum_k p_k (a_k - la - z_k + lse) + rho (log rho - (lse_rest - lse))
 * the Kullback-Leibler divergence from the teacher's distribution to the
 * student's, with lse over all columns and lse_rest over those without an entry
 * (-inf, and rho = 0, where the entries are the whole vocabulary). The p_k are taken
 * as they are: where they add up to more than 1 (entries rounded to bf16 against the
 * log-sum-exp of the exact logits), or are the whole vocabulary's and do not add up to
 * 1, the loss is least, though not 0, at q_k in proportion to p_k. Not scaled by
 * T^2. The [N, V] logits are never stored.
 *   H [N, h], W [V, h] dt      top_ids [N, K] int32 in any order, each below V and
 *                              at most once a row
 *   top_logits [N, K] top_dt   teacher_lse [N] fp32 or NULL
 *   row_mask [N] uint8 or NULL: rows with 0 are not computed, loss = lse = 0
 *   loss, lse, lse_rest [N] fp32, z_top [N, K] fp32 (the entries' z_k, 0 where
 *   there is none): outputs; the last three go to the backward
 * Sizes as sao_token_logprobs_fwd, and 1 <= K <= SAO_DISTILL_MAX_K; T > 0.
 * A row without an entry, or renormalised without one of a logit above -inf, has
 * loss 0 and no gradient. A row with an id out of range or there twice has loss
 * NaN (and SAO_DEVERR_TOP_ID). lse_rest is NaN on the rows that take no gradient:
 * masked ones, and those whose loss is not finite or has nothing to learn from.
 * bf16 H and W are 16-byte aligned. Their logits' sums leave the tensor cores,
 * which truncate as they add, every 512 elements of h and go on in fp32: lse is
 * within 5e-7 of itself up to h = 6,144.
 * The workspace of both calls: sao_distill_workspace_bytes, which never falls as N or K
 * grows: one buffer, sized for the most rows, serves every call of fewer (with the same
 * h, V, dtype and dZ budget), although some of those need more than a call of N does.
 */
SAO_API size_t sao_distill_workspace_bytes(int64_t N, int32_t h, int32_t V, int32_t K, sao_dtype dt);
SAO_API sao_status sao_distill_loss_fwd(const void *H, const void *W, sao_dtype dt, const int32_t *top_ids,
                                        const void *top_logits, sao_dtype top_dt, const float *teacher_lse,
                                        const uint8_t *row_mask, int64_t N, int32_t h, int32_t V, int32_t K,
                                        float temperature, float *loss, float *lse, float *lse_rest, float *z_top,
                                        void *ws, size_t ws_bytes, sao_stream_t stream);

/*
 * Gradient of sum_t grad_loss[t] * loss[t]: with q = e^(z - lse) and the teacher's mass
 * m = sum_k p_k + rho (1 mostly; renormalised: 1),
 *   dz_k = m q_k - p_k at the entries, dz_v = e^(z_v - lse_rest) (m e^(lse_rest - lse)
 *   - rho) elsewhere, dZ = grad_loss dz / T, dH = dZ W, dW = dZ^T H.
 *   lse, lse_rest, z_top  from the forward on the same inputs
 *   grad_loss [N] fp32    rows with 0 contribute nothing
 *   dH [N, h] dt          overwritten (zeros on rows without a gradient)
 *   dW [V, h] dw_dt       SAO_F32, overwritten or (accumulate_dW != 0) added to,
 *                         so that it adds to another loss's dW; or for a bf16 head
 *                         SAO_BF16, overwritten only (a sum over calls needs fp32)
 * A bf16 head's dH and dW are 16-byte aligned. Its dZ is rounded to bf16 once
 * before the two products (as in sao_token_logprobs_bwd): 2^-8 of each of its
 * elements, 2^-16 up to 64 rows and, up to 8,192, for the entries of the 32 rows
 * that would lose most; not at all for one row of
 * h <= 6,144 or two of h <= 2,048. Beside that rounding, dZ outside the entries has the error
 * of logits formed again without the forward's care: the tensor cores truncate h / 16 times
 * as they add, by up to 2^-23 of a partial sum, so an element is off by up to h / 16 *
 * 2^-24 sum_k |H_tk W_vk| / T of itself. Measured with logits of 12 and 24: 2.5e-5 and 5e-5
 * of dW (in fp32, outside the entries) at h = 2,048, 8e-5 and 1.6e-4 at 6,144, 2^-16 being 1.5e-5.
 * Few rows (those, and of an fp32 head up to
 * eight of h <= 1,024, four of h <= 2,048, one of h <= 4,096) read W once in each
 * direction.
 */
SAO_API sao_status sao_distill_loss_bwd(const void *H, const void *W, sao_dtype dt, const int32_t *top_ids,
                                        const void *top_logits, sao_dtype top_dt, const float *teacher_lse,
                                        const float *lse, const float *lse_rest, const float *z_top,
                                        const float *grad_loss, int64_t N, int32_t h, int32_t V, int32_t K,
                                        float temperature, void *dH, void *dW, sao_dtype dw_dt, int accumulate_dW,
                                        void *ws, size_t ws_bytes, sao_stream_t stream);

/* How sao_balance_loss_fwd/bwd turn a token's E router logits into probabilities. */
#define SAO_SCORE_SOFTMAX 0 /* s_e = softmax(x)_e */
#define SAO_SCORE_SIGMOID 1 /* s_e = sigmoid(x_e) / sum_j sigmoid(x_j) */

/* Most experts that sao_balance_loss_fwd/bwd take. */
#define SAO_BALANCE_MAX_EXPERTS 1024

/*
 * Load-balance loss of a mixture-of-experts router, with per-expert counts (an
 * auxiliary loss beside the RL objective; the paper has no counterpart). Over the
 * n counted rows of a segment, with the k experts that each token was sent to:
 *   counts_e = how often expert e was chosen, prob_sums_e = sum_t s_te,
 *   loss = E / (k n^2) sum_e counts_e prob_sums_e        (1 when both are even)
 * cu_seqlens NULL: one segment, the batch (B is taken as 1). Otherwise each of
 * the B packed trajectories is balanced by itself and the loss is the mean over
 * those with a counted row (0 without any).
 *   logits [N, E] dt           expert_ids [N, k] int32; negative: no expert (a
 *                              dropped choice), E or more: none either (and
 *                              SAO_DEVERR_EXPERT_ID)
 *   row_mask [N] uint8 or NULL: rows with 0 are not counted
 *   cu_seqlens [B + 1] int32 or NULL, as for sao_advantages
 *   loss [1] fp32, counts [B, E] int64, prob_sums [B, E] fp32, rows [B] int64
 *   (the counted rows): outputs. The loss is a function of the last three, so
 *   data-parallel ranks that balance their joint batch (cu_seqlens NULL) add
 *   those up before the backward and form the loss from the sums.
 * A row of logits that are all -inf has no probabilities and no gradient.
 * Deterministic. 1 <= k <= E <= SAO_BALANCE_MAX_EXPERTS. Workspace of
 * the forward: sao_balance_workspace_bytes(N, E, B), which never falls as one of them
 * grows; the backward needs the error word's 256 bytes only.
 */
SAO_API size_t sao_balance_workspace_bytes(int64_t N, int32_t E, int32_t B);
SAO_API sao_status sao_balance_loss_fwd(const void *logits, sao_dtype dt, const int32_t *expert_ids,
                                        const uint8_t *row_mask, const int32_t *cu_seqlens, int32_t B, int64_t N,
                                        int32_t E, int32_t k, int score, float *loss, int64_t *counts,
                                        float *prob_sums, int64_t *rows, void *ws, size_t ws_bytes,
                                        sao_stream_t stream);

/*
 * grad_logits = grad_loss[0] * d loss / d logits (counts are not differentiated):
 * with w_e = grad_loss E counts_e / (k n^2 segments), d x_te = s_te (w_e -
 * sum_j s_tj w_j), times 1 - sigmoid(x_te) for SAO_SCORE_SIGMOID; 0 on rows that
 * are not counted. counts and rows are the forward's, or sums of several ranks'.
 *   grad_logits [N, E] dt, overwritten; grad_loss is a device scalar
 */
SAO_API sao_status sao_balance_loss_bwd(const void *logits, sao_dtype dt, const uint8_t *row_mask,
                                        const int32_t *cu_seqlens, int32_t B, int64_t N, int32_t E, int32_t k,
                                        int score, const int64_t *counts, const int64_t *rows,
                                        const float *grad_loss, void *grad_logits, void *ws, size_t ws_bytes,
                                        sao_stream_t stream);

/* Most experts that sao_route_fwd/bwd take, and most of them a token. */
#define SAO_ROUTE_MAX_EXPERTS 1024
#define SAO_ROUTE_MAX_K 32
/* Most groups of experts. */
#define SAO_ROUTE_MAX_GROUPS 32

/* What a group of experts is chosen by. */
#define SAO_GROUP_MAX 0  /* its largest key */
#define SAO_GROUP_TOP2 1 /* the sum of its two largest keys */

/*
 * Routing to experts: each token's k experts and their weights (beside the balance
 * loss, which takes both logits and choices; the paper has no counterpart). Of the
 * logits x of a row,
 *   s_e = softmax(x)_e (SAO_SCORE_SOFTMAX) or sigmoid(x_e) (SAO_SCORE_SIGMOID; not
 *         divided by their sum, as the balance loss does)
 *   key_e = s_e + bias_e; the k experts of the largest keys, in falling order, equal
 *         keys by the lower index
 *   w_j = scale s_{e_j}, divided by the sum of the chosen s if renormalise != 0
 * With groups > 1 the experts form that many runs of E / groups; groups_kept of them
 * stay, by their largest key or the sum of their two largest (group_score), equal ones
 * by the lower index, and the choice is among their experts.
 * Choices are those of the exact scores: keys too near one another for fp32 are
 * compared in 64 bits, whose own rounding decides below that, keys without a bias by their logits. (Softmax and sigmoid keep
 * the logits' order, so experts whose scores are equal in any precision, as of
 * logits past 40, go by the logits too unless there is a bias.)
 * An expert of logit -inf, or of a bias that is -inf or NaN, is never chosen and counts for nothing in
 * its group (one with a single other expert is worth that one's key): where fewer than k are left, the
 * row's last ids are -1 with weight 0. Chosen scores that add up to 0 have weights 0 too.
 * replay != 0: expert_ids are given (a rollout's choices), each row's weights are those
 * of its ids, negative ones have none, and bias, groups and group_score are not used.
 * Ids of E or more have no weight either (and SAO_DEVERR_EXPERT_ID).
 *   logits [N, E] dt           bias [E] fp32 or NULL
 *   row_mask [N] uint8 or NULL: rows with 0 have ids -1 (not if given) and weights 0
 *   expert_ids [N, k] int32    output, or input (replay)
 *   weights [N, k] fp32        output
 * A row with a NaN, or under softmax with a +inf, has no scores: ids -1 (not if given), weights 0 (and
 * SAO_DEVERR_LOGITS). Neither has one that is -inf throughout, which is no error.
 * 1 <= k <= min(SAO_ROUTE_MAX_K, groups_kept E / groups), E <= SAO_ROUTE_MAX_EXPERTS, 1 <=
 * groups_kept <= groups <= SAO_ROUTE_MAX_GROUPS, groups divides E; scale finite.
 * Workspace of both calls: sao_route_workspace_bytes(N, E), which never falls as
 * one of them grows.
 */
SAO_API size_t sao_route_workspace_bytes(int64_t N, int32_t E);
SAO_API sao_status sao_route_fwd(const void *logits, sao_dtype dt, const float *bias, const uint8_t *row_mask,
                                 int64_t N, int32_t E, int32_t k, int score, int32_t groups, int32_t groups_kept,
                                 int group_score, int renormalise, float scale, int replay, int32_t *expert_ids,
                                 float *weights, void *ws, size_t ws_bytes, sao_stream_t stream);

/*
 * Gradient of sum_tj grad_weights[t, j] weights[t, j] in the logits (the choice is not
 * differentiated). With c = sum_j g_j w_j of the row:
 *   renormalised   softmax d x_j = w_j (g_j - c / scale), sigmoid the same times 1 - s_j;
 *                  0 for experts that were not chosen
 *   else           softmax d x_e = s_e (scale g_e - c), g_e = 0 for those that were not
 *                  chosen; sigmoid d x_j = g_j w_j (1 - s_j)
 *   expert_ids, weights   the forward's (ids as given, with replay); an id that a row
 *                  has twice gets both of its gradients
 *   grad_logits [N, E] dt   overwritten (0 on masked rows), or (accumulate != 0) added
 *                  to: to the balance loss's. A bf16 sum is rounded once more.
 * scale 0 gives gradients of 0, as do rows without scores.
 */
SAO_API sao_status sao_route_bwd(const void *logits, sao_dtype dt, const uint8_t *row_mask, int64_t N, int32_t E,
                                 int32_t k, int score, int renormalise, float scale, const int32_t *expert_ids,
                                 const float *weights, const float *grad_weights, void *grad_logits, int accumulate,
                                 void *ws, size_t ws_bytes, sao_stream_t stream);

/* Widest rows of sao_rms_norm_fwd/bwd. */
#define SAO_NORM_MAX_H 16384

/* What shares a scale in the 8-bit rows of sao_rms_norm_fwd. */
#define SAO_SCALE_NONE 0     /* no 8-bit rows */
#define SAO_SCALE_ROW 1      /* a row: scales [N] fp32 */
#define SAO_SCALE_BLOCK128 2 /* 128 columns: scales [N, ceil(h / 128)] fp32 */
#define SAO_SCALE_MX32 3     /* 32 columns: scales [N, ceil(h / 32)] uint8, 2^(scale - 127) */

/*
 * Root-mean-square norm, of the sum with a residual stream if there is one (in front
 * of the LM head: H = y; the paper has no counterpart):
 *   sum[t, c] = x + residual, rounded to dt; without a residual it is x
 *   rstd[t] = (mean_c sum[t, c]^2 + eps)^-1/2,   y[t, c] = sum[t, c] rstd[t] weight[c]
 * and in 8 bits y8 = e4m3(y (1 / scale)), y before its rounding to dt, to the nearest (ties
 * to even), with scale = max(amax / 448, 2^-126) of the row or the block, or the least power
 * of two 2^b >= amax / 448, -127 <= b. A NaN in y makes its scale NaN.
 *   x, residual, sum, y [N, h] dt     weight [h] w_dt     rstd [N] fp32
 *   y8 [N, h] uint8 (e4m3)            scales as `scaling` says
 * residual and sum are both given or both NULL; rstd and one of y and y8 may be NULL;
 * y8 and scales with scaling != SAO_SCALE_NONE only. sum may be x or residual; the
 * other outputs overlap nothing. Squares are summed in fp32: |sum| up to 2^56; small ones
 * keep their digits, whatever eps. (A row of zeros with eps 0 has no norm: NaN. An rstd past
 * fp32's range, of a root mean square below 2^-128, reads +inf.)
 * 1 <= h <= SAO_NORM_MAX_H; eps >= 0 and finite. The forward's workspace: the error word's 256
 * bytes; the backward's: sao_norm_workspace_bytes(N, h), which never falls as one of
 * them grows.
 */
SAO_API size_t sao_norm_workspace_bytes(int64_t N, int32_t h);
SAO_API sao_status sao_rms_norm_fwd(const void *x, const void *residual, sao_dtype dt, const void *weight,
                                    sao_dtype w_dt, float eps, int64_t N, int32_t h, void *sum, void *y, float *rstd,
                                    uint8_t *y8, void *scales, int scaling, void *ws, size_t ws_bytes,
                                    sao_stream_t stream);

/*
 * Gradients of the norm, given those of y and, past the norm, of sum:
 *   dx = dsum + rstd (weight dy - sum rstd^2 mean_c(weight dy sum))   (x's and residual's)
 *   dweight = sum_t dy sum rstd
 *   sum [N, h] dt, rstd [N]   the forward's (sum: x without a residual)
 *   dy, dsum [N, h] dt        dsum may be NULL (nothing behind the norm)
 *   dx [N, h] dt              may be dy or dsum
 *   dweight [h] fp32          overwritten or (accumulate != 0) added to; or NULL
 * Deterministic.
 */
SAO_API sao_status sao_rms_norm_bwd(const void *sum, sao_dtype dt, const void *weight, sao_dtype w_dt,
                                    const float *rstd, const void *dy, const void *dsum, int64_t N, int32_t h,
                                    void *dx, float *dweight, int accumulate, void *ws, size_t ws_bytes,
                                    sao_stream_t stream);

/* One tensor of a list on the host: n contiguous elements of device memory, aligned to
 * their size (vectorised paths: 16 bytes). data may be NULL if n is 0. */
typedef struct sao_tensor {
  void *data;
  int64_t n;
  sao_dtype dt;
} sao_tensor;

/*
 * Global norm of a step's gradients, in two calls so that data-parallel ranks with
 * gradients of their own can add up the first one's result (the paper has no
 * counterpart):
 *   sumsq[0] = sum over the tensors' elements of g^2                  [1] fp64 output
 *   norm[0] = sqrt(sumsq[0]), coef[0] = max_norm / norm where norm > max_norm, else 1
 *   out[i] = coef grads[i], with the fp32 coef, rounded to out's type   norm, coef [1] fp32
 * out NULL: in place, and nothing is read or written where coef is 1. Otherwise out[i]
 * has the elements of grads[i], of either type, and is grads[i] itself or overlaps none of the
 * tensors. Where sumsq is not finite (or negative) coef is NaN and the gradients are passed on
 * as they are: the step is to be dropped. (A norm past fp32's range reads +inf, with its coef.)
 * The lists are read before the calls return; they hold no tensor twice, nor two that
 * overlap. Sums are fp64 (each of 32 or 64 squares fp32 where those are in its range), in a
 * fixed order. max_norm > 0; +inf: only the norm.
 * Workspace: sao_grad_workspace_bytes(), whatever the lists.
 */
SAO_API size_t sao_grad_workspace_bytes(void);
SAO_API sao_status sao_grad_sumsq(const sao_tensor *grads, int32_t count, double *sumsq, void *ws, size_t ws_bytes,
                                  sao_stream_t stream);
SAO_API sao_status sao_grad_clip(const sao_tensor *grads, const sao_tensor *out, int32_t count, const double *sumsq,
                                 float max_norm, float *norm, float *coef, void *ws, size_t ws_bytes,
                                 sao_stream_t stream);

/*
 * Kernel timing for profiling. When enabled, every kernel the library
 * launches is bracketed by CUDA events on its stream; sao_profile_read
 * synchronises those events and returns, for up to `cap` kernel kinds, the
 * name (static string), the number of launches and the summed device
 * milliseconds since the last reset. Returns the number of kinds written.
 */
SAO_API void sao_profile_enable(int on);
SAO_API void sao_profile_reset(void);
SAO_API int sao_profile_read(const char **names, int64_t *launches, double *total_ms, int cap);

#ifdef __cplusplus
}
#endif

#endif /* SAO_H_ */
