/*
 * agrl.h -- C ABI of the fused policy-loss library for AMD MI355X (gfx950).
 *
 * The library computes, on one GPU, the trainer-side hot path of agentic RL
 * with GRPO and task advantage normalisation (AgentRL, arXiv 2510.04206):
 *
 *   agrl_task_adv_norm     per-trajectory action-token counts, GRPO group
 *                          advantages and task advantage normalisation
 *                          (Sec. 3.2; App. B.2 GRPO objective);
 *   agrl_policy_loss_fwd   logits H W^T by vocabulary tiles on the matrix
 *                          cores (never stored), log-softmax, the sampled
 *                          token's log-probability (App. B.1, token-level
 *                          factorisation of the action probability), ratio
 *                          against the behaviour policy and the clipped
 *                          surrogate, masked to action tokens and averaged
 *                          over them (App. B.2 PPO objective; App. A, the
 *                          DAPO objective's decoupled clip bounds and
 *                          token-level normalisation);
 *   agrl_policy_loss_bwd   dH and dW of that loss, recomputing the logits;
 *   agrl_sequence_mean_weights  per-token weights that turn the loss into the
 *                          sequence-level mean of App. B.2's GRPO objective;
 *
 * and what stands on both sides of it in a training step:
 *
 *   agrl_token_norm_fwd    layer or RMS norm of the token rows that become H;
 *   agrl_token_norm_bwd    its gradient, from the loss's dH;
 *   agrl_orthogonalize     Newton-Schulz orthogonalisation of matrices;
 *   agrl_muon_step         the optimiser step of weight matrices with it;
 *
 * and what stands between the packed token ids and that norm and knows of the packing:
 *
 *   agrl_token_embed_fwd   rows of the embedding, scaled;
 *   agrl_token_embed_bwd   its gradient, added up by token id;
 *   agrl_rotate_heads      query and key heads turned by their tokens' positions (and back);
 *   agrl_attention_fwd     causal attention within each sequence of the stream;
 *   agrl_attention_bwd     its gradients.
 *
 * Conventions for every entry point:
 *   - Array arguments are DEVICE pointers owned by the caller; the library
 *     allocates no memory.  Scalars and `opt` are host values.  `stream` is a
 *     hipStream_t passed as void* (NULL = the null stream).
 *   - Calls only enqueue work on `stream` and return; they never synchronise.
 *     Calls that share a workspace or an output are ordered by the caller when
 *     they are on different streams.
 *     Argument errors are reported synchronously, before anything is
 *     launched, and leave every output untouched.
 *   - Row-major, contiguous (where a call has row and matrix strides in its
 *     arguments: rows of consecutive elements).  H is [T, d]; W is [V, d] (the nn.Linear weight
 *     layout, logits = H W^T).  Row n of H is the hidden state that predicts
 *     token_id[n]; the caller shifts labels, the library never does.
 *   - Tokens with action_mask == 0 (environment observations, padding) are
 *     never read for H, token_id, adv_tok, old_logp, lse or logp.  Their
 *     outputs are logp = lse = 0 and dH row = +0.
 *   - Faults found on the device (an id out of range, more action tokens
 *     than max_act) set bits in a per-device error word; read it with
 *     agrl_get_device_error.  An action token whose token_id lies outside
 *     [0, V) poisons the call's outputs, so that a caller who does not read
 *     the word still sees the fault: that token's logp and lse are NaN, the
 *     loss is NaN, and in the backward its logit-gradient row is NaN, which
 *     makes its dH row and every row of dW NaN.  Other tokens' logp and lse
 *     are unaffected.  With more action tokens than max_act the loss is NaN
 *     and the other outputs are unspecified.
 *   - A NaN or +inf logit makes its token's logp and lse non-finite and the
 *     loss NaN; a -inf logit carries no weight.  A NaN old_logp on an action
 *     token makes the loss NaN.
 *   - Results are deterministic: every reduction has a fixed order, no
 *     floating-point atomics are used.  A repeated call keeps its bits.  The
 *     order of the sums of dH and dW may depend on the sizes, on max_act and
 *     g_chunk_bytes, on the number of action tokens and on the device's compute
 *     units: another bound or a partitioned device may change their last bits.
 */
#ifndef AGRL_H
#define AGRL_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  AGRL_OK = 0,
  AGRL_E_NULL = -1,        /* a required pointer is NULL */
  AGRL_E_SHAPE = -2,       /* a size is negative, zero where it must not be, or too large */
  AGRL_E_DTYPE = -3,       /* dtype is not AGRL_BF16 or AGRL_F32 */
  AGRL_E_FLAGS = -4,       /* an option or a clip bound is out of range */
  AGRL_E_WORKSPACE = -5,   /* workspace NULL or smaller than agrl_policy_loss_workspace_size */
  AGRL_E_HIP = -6,         /* the HIP runtime reported an error (see agrl_last_error) */
  AGRL_E_UNSUPPORTED = -7  /* a valid but unimplemented configuration */
} agrl_status;

typedef enum { AGRL_BF16 = 0, AGRL_F32 = 1 } agrl_dtype;

/* Options.  A zero-initialised struct (or opt == NULL) selects the defaults. */
typedef struct {
  int32_t std_ddof;      /* 0: population std in both normalisation stages (default); 1: sample std */
  float std_eps;         /* added to each std before dividing; 0 selects 1e-6 */
  float temperature;     /* logits are (H W^T) / temperature; 0 selects 1 */
  int32_t dw_accumulate; /* 0: dW is overwritten (default); 1: dW += gradient */
  /* Bound on the backward's logit-gradient buffers for one vocabulary chunk:
   * G, roundup(max_act, 256) * Vc * 2 bytes, for AGRL_BF16 (dW reads G
   * transposed); twice that at 4 bytes per element for AGRL_F32 (G, and as much
   * again for partial sums).
   * The backward walks the vocabulary in equal chunks of Vc columns (a
   * multiple of 256), as few as fit the bound; 0 selects 4 GiB.  The full
   * T x V logit gradient is held only when it fits the bound. */
  int64_t g_chunk_bytes;
  /* Optional instrumentation: NULL, or a host array of 8 hipEvent_t.  The
   * library records events[2k] on `stream` just before and events[2k+1] just
   * after its matrix-core launch k: 0 forward logits, 1 backward logit
   * recompute, 2 dW product, 3 dH product.  The dW and dH products run as
   * one launch, bracketed by events 4/5, and events 6/7 are recorded back
   * to back.  With several vocabulary chunks the last chunk's
   * launches are the ones bracketed. */
  void* const* phase_events;
  /* KL penalty against a reference policy (App. A: the PPO and GRPO
   * objectives subtract beta * D_KL).  Per action token, with l = logp and
   * r = ref_logp[t]: kl_estimator 0 (k3, default) KL = exp(r - l) - (r - l) - 1,
   * 1 (k1) KL = l - r.  The loss uses s - kl_beta * KL in place of the
   * surrogate s.  kl_beta = 0 disables it; otherwise ref_logp is a device
   * array of T fp32 values, read on action tokens. */
  float kl_beta;
  int32_t kl_estimator;
  const float* ref_logp;
  /* Per-token loss weights (device, T fp32, read on action tokens): the loss
   * becomes L = -sum_t w_t (s_t - kl_beta KL_t) in place of the token mean
   * -(1/N) sum_t (...), and n_norm is ignored.  Sequence-level aggregation
   * (App. B.2's GRPO form: a token mean per trajectory, then a mean over
   * trajectories) is w_t = 1 / (n_seq * n_traj(t)).  NULL: token mean. */
  const float* token_weight;
  /* agrl_task_adv_norm only: 1 drops every GRPO group whose rewards are all
   * equal (App. A, DAPO's dynamic sampling): its trajectories get advantage 0
   * and are left out of the task statistics.  Needs traj_group. */
  int32_t drop_uniform_groups;
  /* agrl_task_adv_norm only: NULL, or a device array of 2 * (n_group + n_task)
   * int32 (2 * n_task without traj_group) that the call uses as scratch.  With
   * it, the call records the lowest and the highest index of each group's and
   * each task's trajectories (a batch small enough for one workgroup does not
   * need them and leaves it as it is), and each group's and task's wave scans only that
   * index range instead of all n_traj trajectories: the stages then take work
   * proportional to the members' spans rather than n_group * n_traj and
   * n_task * n_traj (trajectories stored segment by segment make every span its
   * segment's size).  The results are bit-identical either way: the summation
   * order below does not depend on it.  Calls that overlap must not share it. */
  int32_t* adv_ranges;
} agrl_options;

/*
 * Advantage normalisation over a global batch of T_g tokens (Sec. 3.2).
 *
 *   traj_id[T_g]      int32, trajectory of each token, -1 for padding
 *   action_mask[T_g]  uint8, 1 for model-generated (action) tokens
 *   traj_task[n_traj] int32, task of each trajectory, in [0, n_task)
 *   traj_group[n_traj] int32, GRPO group (one sample's rollouts) of each
 *                     trajectory, in [0, n_group); NULL skips the group stage
 *   reward[n_traj]    fp32, one reward per trajectory
 * Outputs (all written):
 *   act_count[n_traj] int32, number of action tokens of each trajectory
 *   task_count[n_task] int64, number of action tokens of each task (N_i)
 *   task_mean, task_std [n_task] fp32, mean and std of the task's token-level
 *                     advantage set
 *   adv_traj[n_traj]  fp32, normalised advantage of each trajectory
 *   adv_tok[T_g]      fp32, adv_traj[traj_id[t]] on action tokens, 0 elsewhere
 *                     (NULL: not written)
 *
 * Group stage (App. B.2 GRPO advantage): A_hat = (R - mean_g R) / (std_g R + eps).
 * Task stage (Sec. 3.2): every action token of trajectory tau carries A_hat_tau;
 * mu_i and sigma_i are the mean and std of that token-level set of task i and
 * A_tilde = (A_hat - mu_i) / (sigma_i + eps).  A task without action tokens
 * gets mu = sigma = 0 and A_tilde = 0.
 *
 * Bit-exact fp32: every sum over a segment (a group or a task) deals its
 * terms to 64 partial sums by trajectory index mod 64, adds each partial in
 * ascending trajectory order, and combines the partials by an xor butterfly
 * (offsets 32, 16, 8, 4, 2, 1); products, quotients and the square root are
 * single correctly rounded operations.  Counts are exact integers.
 */
int agrl_task_adv_norm(int64_t T_g, int32_t n_traj, int32_t n_task, int32_t n_group,
                       const int32_t* traj_id, const uint8_t* action_mask,
                       const int32_t* traj_task, const int32_t* traj_group,
                       const float* reward, const agrl_options* opt, int32_t* act_count,
                       int64_t* task_count, float* task_mean, float* task_std, float* adv_traj,
                       float* adv_tok, void* stream);

/*
 * Per-token loss weights of the sequence-level aggregation.  App. B.2 writes
 * GRPO's objective as a mean over the responses of a token mean within each
 * response; for a packed micro-batch of T tokens this is
 *   seq_count[j]    = action tokens of trajectory j in this micro-batch
 *                     (action_mask != 0 and traj_id == j), int32
 *   n_seq           = trajectories with seq_count[j] > 0
 *   token_weight[t] = fp32(1 / (n_seq * seq_count[traj_id[t]])) on action
 *                     tokens with traj_id >= 0 (the quotient is formed in
 *                     fp64 and rounded once), 0 on every other token.
 * Passed as agrl_options.token_weight to the policy-loss calls, the loss
 * becomes -(1/n_seq) sum_j (1/seq_count[j]) sum_{t in j} (...).  A trajectory
 * cut by the packing counts only its tokens in this micro-batch.
 *   traj_id[T]       int32 trajectory of each token, -1 for padding (device)
 *   action_mask[T]   uint8 (device)
 *   seq_count[n_traj]  int32, written (device)
 *   token_weight[T]  fp32, written (device)
 * A traj_id >= n_traj sets ERR bit 2 of the device error word and the token
 * is ignored.  T = 0 writes seq_count only.
 */
int agrl_sequence_mean_weights(int64_t T, int32_t n_traj, const int32_t* traj_id,
                               const uint8_t* action_mask, int32_t* seq_count,
                               float* token_weight, void* stream);

/*
 * Bytes of device workspace the forward and backward calls need for a packed
 * micro-batch of T tokens of which at most max_act are action tokens
 * (max_act <= 0 means T).  The same workspace serves both calls.  Returns 0
 * for invalid sizes.
 */
size_t agrl_policy_loss_workspace_size(int64_t T, int64_t max_act, int32_t d, int32_t V,
                                       int32_t dtype, const agrl_options* opt);

/*
 * Vocabulary columns per backward chunk for these sizes and options (the same
 * arguments as agrl_policy_loss_workspace_size): a multiple of 256, at most
 * roundup(V, 256).  The backward recomputes the logits and forms G for
 * ceil(V / chunk) chunks in order; the last holds the remaining columns.
 * Returns 0 for invalid sizes.  Host-only; no device work.
 */
int64_t agrl_policy_loss_vocab_chunk(int64_t T, int64_t max_act, int32_t d, int32_t V,
                                     int32_t dtype, const agrl_options* opt);

/*
 * Forward of the token-level clipped policy loss over a packed micro-batch.
 *
 *   T, d, V         tokens, hidden size (multiple of 64), vocabulary size
 *   max_act         upper bound on the number of action tokens (<= 0: T)
 *   dtype           AGRL_BF16 (bf16 inputs, fp32 accumulation on the matrix
 *                   cores) or AGRL_F32
 *   H[T, d], W[V, d]  hidden states and LM head, in `dtype`
 *   token_id[T]     int32 sampled token of each position (read on action tokens)
 *   action_mask[T]  uint8
 *   adv_tok[T]      fp32 advantage of each token (e.g. agrl_task_adv_norm's adv_tok)
 *   old_logp[T]     fp32 log-probability of token_id under the behaviour policy
 *   clip_eps_low, clip_eps_high  ratio clipped to [1 - low, 1 + high],
 *                   0 <= low < 1, high >= 0
 *   n_norm          loss divisor; <= 0 uses the number of action tokens
 * Outputs:
 *   loss[1]         L = -(1/N) sum over action tokens of min(rho A, clip(rho) A),
 *                   rho = exp(logp - old_logp); 0 when N == 0
 *   logp[T], lse[T] fp32 log-probability of token_id and log-sum-exp of the
 *                   logits on action tokens, 0 elsewhere
 *   n_clip[2]       int64 {#tokens with A > 0 and rho > 1 + high,
 *                          #tokens with A < 0 and rho < 1 - low}; NULL: skipped
 */
int agrl_policy_loss_fwd(int64_t T, int64_t max_act, int32_t d, int32_t V, int32_t dtype,
                         const void* H, const void* W, const int32_t* token_id,
                         const uint8_t* action_mask, const float* adv_tok,
                         const float* old_logp, float clip_eps_low, float clip_eps_high,
                         int64_t n_norm, const agrl_options* opt, void* workspace,
                         size_t ws_bytes, float* loss, float* logp, float* lse, int64_t* n_clip,
                         void* stream);

/*
 * Backward of the same loss, scaled by grad_loss (the upstream dL).
 *
 * Arguments as for the forward, plus lse[T] and logp[T] as returned by the
 * forward on the same inputs.  With g_n = dL/dlogp_n = -(grad_loss/N) A_n rho_n
 * (0 for tokens whose clipped branch is active) and p the softmax of the
 * logits, the logit gradient is G[n, v] = g_n (1[v = y_n] - p[n, v]) / temperature and
 *   dH[T, d] fp32 = G W       (+0 rows for masked tokens)
 *   dW[V, d] fp32 = G^T H     (overwritten, or added to with opt->dw_accumulate)
 * dH and dW must be 16-byte aligned (AGRL_E_UNSUPPORTED otherwise): their rows
 * are written 16 bytes per lane.
 * The logits are recomputed tile by tile; G is rounded to `dtype` (bf16 for
 * AGRL_BF16) before the two products, which accumulate in fp32.
 */
int agrl_policy_loss_bwd(int64_t T, int64_t max_act, int32_t d, int32_t V, int32_t dtype,
                         const void* H, const void* W, const int32_t* token_id,
                         const uint8_t* action_mask, const float* adv_tok,
                         const float* old_logp, float clip_eps_low, float clip_eps_high,
                         int64_t n_norm, const agrl_options* opt, const float* lse,
                         const float* logp, float grad_loss, void* workspace, size_t ws_bytes,
                         float* dH, float* dW, void* stream);

/*
 * Forward-only token log-probabilities over a packed batch: log pi(a_t | s_t)
 * of every action token, the factorised log-probability of an action
 * (App. B.1), as needed for the old-policy denominator of the PPO ratio
 * (App. B.2) when it is recomputed on the trainer rather than taken from the
 * rollout engine.  The same tiles, partials and merge as agrl_policy_loss_fwd,
 * so logp and lse are bit-identical to that call's on the same inputs.
 *
 *   T, max_act, d, V, dtype, H, W, token_id, action_mask, opt: as for
 *                   agrl_policy_loss_fwd (opt->temperature divides the logits)
 *   workspace       at least agrl_token_logprob_workspace_size bytes (the
 *                   policy-loss workspace also serves)
 * Outputs:
 *   logp[T], lse[T] fp32 on action tokens, 0 elsewhere
 * Errors as for agrl_policy_loss_fwd; T == 0 enqueues nothing.
 */
size_t agrl_token_logprob_workspace_size(int64_t T, int64_t max_act, int32_t d, int32_t V,
                                         int32_t dtype, const agrl_options* opt);
int agrl_token_logprob(int64_t T, int64_t max_act, int32_t d, int32_t V, int32_t dtype,
                       const void* H, const void* W, const int32_t* token_id,
                       const uint8_t* action_mask, const agrl_options* opt, void* workspace,
                       size_t ws_bytes, float* logp, float* lse, void* stream);

/*
 * agrl_token_logprob without a workspace argument, for callers that cannot
 * allocate device memory around the call: code being captured into a HIP
 * graph, tight serving loops, harnesses that forbid allocation.  The same
 * kernels, outputs and errors as agrl_token_logprob; their workspace is a
 * fixed array of AGRL_NOALLOC_SCRATCH_BYTES of device memory that the library
 * holds on every GPU it runs on until the process ends.  The call allocates
 * nothing (no hipMalloc, no library routine that allocates); the caller still
 * passes the inputs and outputs.
 *   Arguments as for agrl_token_logprob, without workspace and ws_bytes.
 *   Sizes whose agrl_token_logprob_workspace_size exceeds the array are
 *   refused with AGRL_E_WORKSPACE before anything is launched.
 * Every call on one GPU uses that GPU's array, and an array keeps what the
 * last call left in it (nothing in it needs to start at zero: the kernels
 * write every value they read).  Calls that overlap on one GPU, from two
 * streams or two host threads, race on the array; serialise them.
 */
#define AGRL_NOALLOC_SCRATCH_BYTES (64ll << 20)
int agrl_token_logprob_noalloc(int64_t T, int64_t max_act, int32_t d, int32_t V, int32_t dtype,
                               const void* H, const void* W, const int32_t* token_id,
                               const uint8_t* action_mask, const agrl_options* opt, float* logp,
                               float* lse, void* stream);

/*
 * Layer or RMS norm of token rows: the final norm whose output is the policy
 * loss's H, and (backward) which takes its dH.  Per live row
 *   AGRL_NORM_LAYER  mean = (1/d) sum x, var = (1/d) sum (x - mean)^2,
 *                    rstd = 1/sqrt(var + eps), y = (x - mean) rstd weight + bias
 *   AGRL_NORM_RMS    rstd = 1/sqrt((1/d) sum x^2 + eps), y = x rstd weight + bias
 * Statistics, products and sums are fp32; y is rounded once to `dtype`.
 *   T, d             rows and row length, 1 <= d <= 16384 (AGRL_E_UNSUPPORTED above)
 *   dtype, w_dtype   type of x and y, and of weight and bias: AGRL_BF16 or AGRL_F32
 *   x[T, d]          rows ld_x >= d elements apart; y likewise with ld_y
 *   weight, bias[d]  NULL: 1, and 0
 *   action_mask[T]   uint8; NULL: every row is live.  Rows with mask 0 are never
 *                    read; their y is +0, their mean and rstd 0
 *   eps              finite, >= 0
 * Outputs: y, mean[T] (layer; NULL: not written), rstd[T] (NULL: not written).
 * x, y and the parameters may start at any element.  y may be x itself (the
 * same pointer and stride); arrays that overlap in another way are not
 * supported.  A constant row has y = bias up to rounding (layer).  A row with a
 * NaN or infinite element, or whose sum (layer) or sum of squares passes fp32's
 * range (elements around 1e19), is NaN as a whole, its rstd too; no other row is.
 */
enum { AGRL_NORM_LAYER = 0, AGRL_NORM_RMS = 1 };
int agrl_token_norm_fwd(int64_t T, int32_t d, int32_t kind, int32_t dtype, int32_t w_dtype,
                        const void* x, int64_t ld_x, const void* weight, const void* bias,
                        const uint8_t* action_mask, float eps, void* y, int64_t ld_y, float* mean,
                        float* rstd, void* stream);

/* Bytes of workspace for agrl_token_norm_bwd's sums over rows; 0 for invalid
 * sizes.  Host-only. */
size_t agrl_token_norm_bwd_workspace_size(int64_t T, int32_t d);

/*
 * Backward of agrl_token_norm_fwd.  With xh = (x - mean) rstd (RMS: x rstd) and
 * g = dy weight:
 *   dx      = rstd (g - (1/d) sum g - xh (1/d) sum (g xh))   (RMS: without sum g)
 *   dweight = sum over live rows of dy xh,  dbias = sum over live rows of dy
 *   dy[T, d]      in dy_dtype (the policy loss's dH is AGRL_F32), rows ld_dy apart
 *   mean, rstd    as the forward left them (mean is not read for RMS)
 *   accumulate    0: dweight and dbias are overwritten, 1: added to
 *   workspace     4-byte aligned; not needed when dweight and dbias are NULL
 * Outputs: dx[T, d] in `dtype`, rows ld_dx apart (+0 on masked rows, whose x, dy,
 * mean and rstd are never read); dweight[d], dbias[d] fp32 (NULL: not formed).
 * With T = 0, or no live row, dweight and dbias are 0 (or keep their values).
 * dx may be x or dy itself where type and stride agree.
 */
int agrl_token_norm_bwd(int64_t T, int32_t d, int32_t kind, int32_t dtype, int32_t w_dtype,
                        int32_t dy_dtype, const void* x, int64_t ld_x, const void* weight,
                        const uint8_t* action_mask, const void* dy, int64_t ld_dy,
                        const float* mean, const float* rstd, int32_t accumulate, void* workspace,
                        size_t ws_bytes, void* dx, int64_t ld_dx, float* dweight, float* dbias,
                        void* stream);

/*
 * Newton-Schulz orthogonalisation of a stack of `batch` matrices G [m, n]:
 *   X = G / (|G|_F + eps)
 *   `steps` times: A = X X^T, B = b A + c A A, X = a X + B X    (m <= n;
 *   for m > n the same on the transpose, X = a X + X B with A = X^T X)
 *   O = X
 * the odd polynomial a s + b s^3 + c s^5 applied to G's singular values, `steps`
 * times.  The coefficients must keep every singular value s, which start in [0, 1],
 * below 3.9 and |b s^2 + c s^4| + max(|a|, |b + c| / 2) below 15: beyond, the operands'
 * range overflows and the result is not finite.
 */
typedef struct {
  int32_t steps;     /* 0 selects 5 */
  float a, b, c;     /* all 0 selects 3.4445, -4.7750, 2.0315 */
  float eps;         /* 0 selects 1e-7 */
} agrl_ns_options;

/* Bytes of workspace for agrl_orthogonalize and agrl_muon_step (out_dtype: the
 * type of O or of the parameter); 0 for invalid sizes.  Host-only. */
size_t agrl_orthogonalize_workspace_size(int64_t batch, int64_t m, int64_t n, int32_t out_dtype);

/*
 *   batch, m, n      0 in any of them enqueues nothing; m, n <= 2^20, the smaller
 *                    <= 65536, batch <= 65535
 *   dtype            type of G: AGRL_BF16 or AGRL_F32; rows ld_g >= n elements apart,
 *                    matrices stride_g apart (not read for batch 1)
 *   out_dtype        type of O: AGRL_BF16 or AGRL_F32; ld_o, stride_o likewise
 *                    (any strides that keep O's rows apart: matrix after matrix, or
 *                    rows of the matrices in turn, ld_o >= (batch - 1) stride_o + n)
 *   ns               NULL or options (zero-initialised: the defaults)
 *   workspace        256-byte aligned, agrl_orthogonalize_workspace_size bytes
 * G and O may start at any element and must not overlap.
 * Precision goes by out_dtype.  AGRL_F32: operands of 22 bits (two fp16 numbers each,
 * three fp16 products for one of theirs) and fp32 sums, 1e-7 to 2e-5 of O's norm: 0.2 to
 * 1.4 times what fp32 products are off by on noise, less than they on large matrices of
 * repeated entries, up to 1e-6 where they hardly round (the identity).  AGRL_BF16 with
 * min(m, n) <= 128: the same, rounded.  AGRL_BF16 of more: operands rounded to fp16 (11
 * bits), the iterate held in 22, fp32 sums.  Besides O's own rounding that is 1e-4 to 2e-3
 * of O's norm where the roundings average, as in a gradient's noise.  Where entries repeat
 * (blocks of one value, diagonal matrices) they add up: 5e-3 in the middle and up to 3e-2
 * among 1 to 256 equal blocks, 6e-2 at the worst to first order (the default polynomial).
 * An fp32 O has none of that.  |G|_F is summed in 64 bits.  A zero matrix gives 0; a
 * NaN or infinite entry makes its whole matrix NaN, and no other.
 */
int agrl_orthogonalize(int64_t batch, int64_t m, int64_t n, int32_t dtype, const void* G,
                       int64_t ld_g, int64_t stride_g, int32_t out_dtype,
                       const agrl_ns_options* ns, void* workspace, size_t ws_bytes, void* O,
                       int64_t ld_o, int64_t stride_o, void* stream);

/*
 * One optimiser step for a stack of weight matrices [m, n]:
 *   momentum <- mu momentum + grad
 *   u        =  grad + mu momentum (nesterov 1) or momentum (0)
 *   param    <- (1 - lr weight_decay) param - lr scale O(u)
 * with O as above.  grad as G above; param [m, n] in param_dtype, updated in place,
 * rows ld_param and matrices stride_param apart; momentum fp32, contiguous
 * [batch, m, n], 4-byte aligned.  scale 0 selects sqrt(max(1, m / n)).  A bf16
 * parameter is rounded to nearest once per step.  The three must not overlap.
 */
int agrl_muon_step(int64_t batch, int64_t m, int64_t n, int32_t grad_dtype, const void* grad,
                   int64_t ld_grad, int64_t stride_grad, int32_t param_dtype, void* param,
                   int64_t ld_param, int64_t stride_param, float* momentum, float lr, float mu,
                   int32_t nesterov, float weight_decay, float scale, const agrl_ns_options* ns,
                   void* workspace, size_t ws_bytes, void* stream);

/*
 * Embedding of a packed stream: y[n] = scale * weight[token_id[n]].
 *   T, d, V           tokens, row length (<= 2^20), rows of the embedding
 *   w_dtype, dtype    type of weight and of y: AGRL_BF16 or AGRL_F32; y is rounded once
 *   weight[V, d]      contiguous; token_id[T] int32
 *   live_mask[T]      uint8; NULL: every token is live.  A token with mask 0 is not read (nor
 *                     its id); its y is +0
 *   scale             finite
 *   y[T, d]           rows ld_y >= d elements apart
 * weight and y may start at any element.  A live token_id outside [0, V) sets bit 1 of the
 * device error word and makes its row NaN.
 */
int agrl_token_embed_fwd(int64_t T, int32_t d, int32_t V, int32_t w_dtype, int32_t dtype,
                         const void* weight, const int32_t* token_id, const uint8_t* live_mask,
                         float scale, void* y, int64_t ld_y, void* stream);

/* Bytes of workspace for agrl_token_embed_bwd; 0 for invalid sizes.  Host-only. */
size_t agrl_token_embed_bwd_workspace_size(int64_t T, int32_t d, int32_t V);

/*
 * Gradient of the embedding: dweight[v] = scale * sum of dy[n] over the live tokens n with
 * token_id[n] = v, in fp32, in an order that the ids fix.
 *   V                 <= 2^31 - 1024; ceil(T / 32) ceil(d / 1024) (T <= 256: T of them), and ceil(V / 8) with accumulate 0,
 *                     below 2^24 together
 *   dy[T, d]          in dy_dtype, rows ld_dy >= d elements apart, from any element
 *   accumulate        0: every row of dweight is written (0 where no token has its id); 1: the
 *                     sums are added, rows without a token are not touched.  A tied head's
 *                     gradient: agrl_policy_loss_bwd first, then this with accumulate 1
 *   workspace         256-byte aligned, agrl_token_embed_bwd_workspace_size bytes
 *   dweight[V, d]     fp32, contiguous, 4-byte aligned
 * A live token_id outside [0, V) sets bit 1 of the device error word and adds nothing.  T = 0
 * writes zeros (accumulate 0) or nothing.
 */
int agrl_token_embed_bwd(int64_t T, int32_t d, int32_t V, int32_t dy_dtype,
                         const int32_t* token_id, const uint8_t* live_mask, const void* dy,
                         int64_t ld_dy, float scale, int32_t accumulate, void* workspace,
                         size_t ws_bytes, float* dweight, void* stream);

/*
 * Heads [T, n_head, d] in the two calls below: `ld` elements between tokens, `head` between
 * heads, the d elements of a head adjacent, from any element.  Inputs may have any strides that are
 * not negative (0 repeats a head or a token); the heads of an output must not overlap.
 *
 * Rotation by position: of each head's first `rot` elements (even, <= d) the pairs
 * (i, i + rot / 2), or (2 i, 2 i + 1) with interleaved = 1, are turned by the angle
 * position * base^(-2 i / rot):  (p, q) -> (p cos - q sin, p sin + q cos).  Elements from rot on are
 * copied.  inverse = 1 turns back, which is the gradient of the rotation.
 *   T, n_head, d      d <= 512 (AGRL_E_UNSUPPORTED above)
 *   dtype             type of x and y: AGRL_BF16 or AGRL_F32; angles are formed in 64 bits, the
 *                     rest in 32, y is rounded once
 *   position[T]       int32, any value; NULL: the token's number
 *   base              finite, > 0
 *   y                 may be x itself (the same strides); arrays that overlap in another way
 *                     are not supported
 */
int agrl_rotate_heads(int64_t T, int32_t n_head, int32_t d, int32_t rot, int32_t dtype,
                      const void* x, int64_t ld_x, int64_t head_x, const int32_t* position,
                      double base, int32_t interleaved, int32_t inverse, void* y, int64_t ld_y,
                      int64_t head_y, void* stream);

/*
 * Causal attention within each sequence of a packed stream of T tokens:
 *   S = scale q k^T over the keys of the token's sequence up to the token itself,
 *   o = softmax(S) v,  lse = log sum exp S
 *   n_head, n_kv      query heads; key heads, a divisor: query head h reads key head h / (n_head / n_kv);
 *                     ceil(T / 128) n_head < 2^24
 *   d                 head size, <= 128 (AGRL_E_UNSUPPORTED above)
 *   dtype             type of q, k, v and o: AGRL_BF16 or AGRL_F32
 *   q [T, n_head, d]; k, v [T, n_kv, d]
 *   seq_start[n_seq + 1]  int32: sequence i is the tokens seq_start[i] .. seq_start[i + 1] - 1; it may
 *                     be empty.  Tokens before the first offset and from the last one on belong to no
 *                     sequence: their values do not matter, their o is +0 and their lse 0.  n_seq = 0:
 *                     no token belongs to one.  Offsets that decrease or leave [0, T] set bit 32 of
 *                     the device error word; what o holds is then unspecified
 *   scale             2^-60 to 2^60
 * Outputs: o [T, n_head, d]; lse [n_head, T] fp32 (NULL: not written; the backward needs it).
 * Products of bf16 inputs and all sums are fp32, P is rounded to `dtype` before it meets v, o once.
 * Scores may have any size that fp32 holds: the largest weight of a row is 1, the others are as exact as fp32 holds the
 * differences of scores.  Sums of weights times v are fp32, weights up to 2^8 before the row is divided: the keys of a row
 * times 2^8 |v| should stay within its range.
 * No token of another sequence and no later one of its own reaches a row, not even a NaN or
 * infinite one; an element of v that is not finite makes what counts it NaN or infinite.
 */
int agrl_attention_fwd(int64_t T, int32_t n_seq, int32_t n_head, int32_t n_kv, int32_t d,
                       int32_t dtype, const void* q, int64_t ld_q, int64_t head_q, const void* k,
                       int64_t ld_k, int64_t head_k, const void* v, int64_t ld_v, int64_t head_v,
                       const int32_t* seq_start, float scale, void* o, int64_t ld_o,
                       int64_t head_o, float* lse, void* stream);

/* Bytes of workspace for agrl_attention_bwd; 0 for invalid sizes.  Host-only. */
size_t agrl_attention_bwd_workspace_size(int64_t T, int32_t n_head, int32_t n_kv, int32_t d,
                                         int32_t dtype);

/*
 * Gradients of agrl_attention_fwd.  With P = exp(S - lse), D = sum over d of dout o and
 * dS = P (dout v^T - D):  dv = P^T dout, dq = scale dS k, dk = scale dS^T q; dk and dv are the sums over
 * the query heads that share a key head (in a fixed order).
 *   o, lse            as the forward left them (P is as exact as fp32 holds S and lse, so a lse formed in another way makes it
 *                     off by exp of its difference); dout [T, n_head, d] in `dtype`
 *   workspace         256-byte aligned, agrl_attention_bwd_workspace_size bytes
 * Outputs in `dtype`: dq [T, n_head, d], dk and dv [T, n_kv, d] (+0 on tokens of no sequence); they may be
 * parts of one array [T, n_head + 2 n_kv, d].  P and dS are rounded to `dtype` before they
 * meet dout, k and q; sums are fp32.
 */
int agrl_attention_bwd(int64_t T, int32_t n_seq, int32_t n_head, int32_t n_kv, int32_t d,
                       int32_t dtype, const void* q, int64_t ld_q, int64_t head_q, const void* k,
                       int64_t ld_k, int64_t head_k, const void* v, int64_t ld_v, int64_t head_v,
                       const int32_t* seq_start, float scale, const void* o, int64_t ld_o,
                       int64_t head_o, const float* lse, const void* dout, int64_t ld_do,
                       int64_t head_do, void* workspace, size_t ws_bytes, void* dq, int64_t ld_dq,
                       int64_t head_dq, void* dk, int64_t ld_dk, int64_t head_dk, void* dv,
                       int64_t ld_dv, int64_t head_dv, void* stream);

/* Text for a status code (static storage). */
const char* agrl_status_string(int status);

/* Message of the last AGRL_E_* returned on this host thread ("" if none). */
const char* agrl_last_error(void);

/*
 * Synchronises `stream`, then reads and clears the current device's error
 * word into *code (0 = no fault; bits: 1 token id, 2 trajectory id, 4 task
 * id, 8 group id, 16 more action tokens than max_act, 32 sequence offsets).
 */
int agrl_get_device_error(void* stream, int32_t* code);

#ifdef __cplusplus
}
#endif

#endif /* AGRL_H */
