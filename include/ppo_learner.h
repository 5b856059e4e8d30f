/*
 * ppo_learner.h - C ABI of the MI355X PPO learner library (libppo_learner.so).
 *
 * One context = the dedicated learner GPU of the paper's disaggregated
 * set-up (Sec. III-B, Fig. 2b, Algorithm 2): it owns the experience buffer
 * of depth images + proprioception, the actor-critic parameters, their Adam
 * state and all workspaces, and runs TrainPPO (Algorithm 2, last step) and
 * the stereo-RGB distillation update (Sec. I, Sec. III-C) on them.
 *
 * Conventions
 *  - Every function returns 0 or a negative PPO_E* code; ppo_last_error()
 *    gives the text of the last failure on that context.  No exceptions and
 *    no aborts cross this boundary.  Arguments are validated before any HIP
 *    call is made.
 *  - Pointers named d_* are DEVICE pointers owned by the caller; they must
 *    stay valid until the work enqueued by the call has run on the context's
 *    stream.  Pointers named h_* / host_* are HOST pointers.  The library
 *    never frees or keeps caller memory.
 *  - The library owns everything it allocates (in ppo_create) and releases it
 *    in ppo_destroy.  ppo_buffer_write / ppo_gae / ppo_update /
 *    distill_update allocate nothing.
 *  - Work is enqueued on the HIP stream given to ppo_create (NULL = the
 *    default stream).  Calls that fill host memory synchronise that stream;
 *    all others return as soon as the work is enqueued.
 *  - A flat sample index is s = t*num_envs + n.
 *  - Canonical parameter order (fp32): for each conv layer W[Co][Ci][3][3],
 *    b[Co]; for each hidden layer W[out][in], b[out] (the first hidden
 *    layer's input is [flatten(view0) in (c,h,w) order, flatten(view1), ...,
 *    proprio]); action head W[A][h], b[A]; and, with a value head, w_v[h],
 *    b_v, logstd[A].
 */
#ifndef PPO_LEARNER_H
#define PPO_LEARNER_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define PPO_OK 0
#define PPO_EINVAL (-1) /* null pointer, NaN / out-of-range hyper-parameter            */
#define PPO_ESHAPE (-2) /* geometry the kernels do not support, or sizes do not divide */
#define PPO_ESTATE (-3) /* calls out of order (e.g. ppo_gae before all steps written)  */
#define PPO_EHIP (-4)   /* a HIP runtime call failed                                   */
#define PPO_ENOMEM (-5) /* device or host allocation failed                            */

#define PPO_MAX_LAYERS 8

typedef struct ppo_ctx ppo_ctx; /* opaque, library-owned */

/* Network and buffer geometry.  The network is the feed-forward actor-critic
 * of the benchmark configurations: a stack of 3x3 stride-2 pad-1 convolutions
 * with ReLU on each view (shared weights), flatten, concatenate proprioception,
 * ReLU hidden layers, a linear Gaussian-mean head and (optionally) a scalar
 * value head with a state-independent log-std vector (cf. the CNN -> concat
 * proprio -> MLP sketch of Sec. III-C, Fig. 3). */
typedef struct {
  int32_t num_envs, horizon;         /* N, T */
  int32_t n_views, in_c, in_h, in_w; /* 1 x 1xHxW depth, or 2 x 3xHxW stereo RGB */
  int32_t obs_dtype;                 /* element type the CALLER passes to ppo_buffer_write: 0 fp32, 1 bf16 */
  int32_t proprio_dim, act_dim;      /* P (multiple of 8), A (<= 31) */
  int32_t n_conv, conv_ch[PPO_MAX_LAYERS]; /* channel counts, each a multiple of 8 */
  int32_t conv_k, conv_stride, conv_pad;   /* must be 3, 2, 1 */
  int32_t n_fc, fc_dim[PPO_MAX_LAYERS];    /* hidden widths, each a multiple of 8, n_fc >= 1 */
  int32_t has_value_head;            /* 1 actor-critic (PPO), 0 distillation student */
  int32_t max_chunk;                 /* samples per forward/backward pass inside a minibatch; 0 = default */
  /* (n_conv - 1) + n_fc + 1 head + 2 with the auxiliary head below + 1 with an embedding + lstm_layers must be at
   * most 12 (else PPO_ESHAPE). */
  /* The deployed student's extra MLP head (Sec. IV-C: "an extra MLP head that predicts the position of the
   * object"): with aux_hidden > 0 (a multiple of 8; students only) the last aux_dim (1 .. act_dim-1) output
   * columns are  W_a2 relu(W_a1 h + b_a1) + b_a2  on the last hidden layer h, and the linear head has
   * act_dim - aux_dim rows.  The targets stay in the last aux_dim columns of the action slot; ppo_hparams.aux_dim
   * must equal this aux_dim and aux_coef weighs their error.  Canonical order: W_a1[aux_hidden][h], b_a1,
   * W_a2[aux_dim][aux_hidden], b_a2 after everything else.  0: no such head. */
  int32_t aux_hidden, aux_dim;
  /* The paper's own teacher (Sec. III-C, Fig. 3): layer normalisation after every convolution (over the C*H*W
   * values of a sample, eps 1e-5, gain and shift per channel, before the ReLU; canonical: g[Co], s[Co] after each
   * conv bias), embed_dim > 0: a linear layer flatten -> embed_dim per view (no activation; canonical W[E][flat],
   * b[E] after the convolutions) whose output is concatenated with the proprioception, and lstm_layers LSTM
   * layers of lstm_units units (gate order i, f, g, o; canonical per layer W_ih[4H][in], W_hh[4H][H], b[4H])
   * between that concatenation and the hidden layers.  With lstm_layers > 0 ppo_update trains on minibatches
   * of whole environments (back-propagation through the T steps of the horizon, the state reset where a done
   * flag is set, initial state from ppo_buffer_write_state) and num_envs must be divisible by
   * hp.minibatches.  All zero: the feed-forward network of the benchmark configurations. */
  int32_t layer_norm, embed_dim, lstm_layers, lstm_units;
} ppo_net_desc;

typedef struct {
  float gamma, lambda;          /* used by ppo_gae only through its own arguments; kept for logging */
  float clip_eps;               /* > 0 */
  float vclip_eps;              /* <= 0: value clipping off */
  float vf_coef, ent_coef;
  float lr, beta1, beta2, adam_eps;
  float max_grad_norm;          /* > 0: global gradient-norm clipping, g *= min(1, c / (||g|| + 1e-6)), before every Adam step; <= 0: off */
  float desired_kl;             /* > 0 (ppo_update only): KL-adaptive learning rate.  Before each Adam step the rate
                                   follows the minibatch's approx_kl = mean((rho-1) - log rho), the sampled estimate of
                                   KL(behaviour policy || current policy): approx_kl > 2 desired_kl divides it by 1.5
                                   (not below lr_min), approx_kl < desired_kl / 2 multiplies it by 1.5 (not above
                                   lr_max).  The rate starts from `lr` and lives on the device (no host round trip);
                                   ppo_mb_stats.lr reports what each step used.  <= 0: off, every step uses `lr`.
                                   The paper gives no schedule (Sec. III-C); this is the common one of on-policy code. */
  float lr_min, lr_max;         /* bounds of the adaptive rate; 0 < lr_min <= lr_max when desired_kl > 0 */
  float aux_coef;               /* distill_update with aux_dim > 0: weight of the auxiliary columns' error (>= 0) */
  int32_t epochs, minibatches;  /* num_envs*horizon must be divisible by minibatches */
  int32_t norm_adv;             /* 1: advantages normalised once per update over the whole rollout,
                                   (A - mean) / (population std + 1e-8); 0: raw advantages */
  int32_t lr_carry;             /* with desired_kl > 0: 1 = start from the rate the previous adaptive update of this
                                   context ended with (if there was one; else from `lr`), 0 = start from `lr` */
  int32_t aux_dim;              /* distill_update: the last aux_dim (< act_dim) head columns are an auxiliary output,
                                   0 = none; see distill_update */
  uint64_t seed;                /* permutation stream seed */
} ppo_hparams;

/* One record per optimiser step, in order epoch-major. */
typedef struct {
  float pi_loss, v_loss, entropy, approx_kl, clip_frac, grad_norm, total_loss;
  int32_t nonfinite; /* 1 if the total loss was not finite */
  float lr;          /* learning rate this step's Adam update used */
} ppo_mb_stats;

/* Create a learner for `desc` on the current HIP device; all device memory and the
 * pinned staging of the parameter read-back are allocated here.  `hip_stream` is a hipStream_t (may be NULL).  Parameters
 * start at zero: load them with ppo_set_params. */
int ppo_create(ppo_ctx** out, const ppo_net_desc* desc, void* hip_stream);
int ppo_destroy(ppo_ctx* ctx);
const char* ppo_last_error(const ppo_ctx* ctx); /* ctx may be NULL: error of the last failed ppo_create */

int64_t ppo_param_count(const ppo_ctx* ctx);
/* Device bytes held by the experience buffer's image part (Sec. III-B sizing example). */
int64_t ppo_buffer_image_bytes(const ppo_ctx* ctx);

/* Parameters / gradients / optimiser state in canonical order, HOST fp32 arrays of
 * n = ppo_param_count() elements.  All synchronise.  ppo_get_grads returns the gradient
 * of the last minibatch processed.  Setting parameters or optimiser state is the
 * checkpoint/resume path: after get -> (new ctx) set, the next update is bit-identical (with
 * desired_kl > 0 and lr_carry = 1 the adaptive rate below belongs to the state as well). */
int ppo_set_params(ppo_ctx* ctx, const float* h_params, int64_t n);
int ppo_get_params(ppo_ctx* ctx, float* h_params, int64_t n);
int ppo_get_grads(ppo_ctx* ctx, float* h_grads, int64_t n);
int ppo_set_opt_state(ppo_ctx* ctx, const float* h_m, const float* h_v, int64_t n, int64_t step, int64_t update_idx);
int ppo_get_opt_state(ppo_ctx* ctx, float* h_m, float* h_v, int64_t n, int64_t* step, int64_t* update_idx);

/* The KL-adaptive learning rate a context carries between updates (hp.desired_kl > 0, hp.lr_carry = 1): part of
 * a checkpoint beside the optimiser state.  get: *h_live = 1 and *h_lr = the rate the last adaptive update ended
 * with, or *h_live = 0 (no adaptive update has run; *h_lr = 0).  set with live = 1 installs `lr` (> 0) as that
 * rate, live = 0 forgets it (the next adaptive update starts from hp.lr).  Both synchronise. */
int ppo_get_adaptive_lr(ppo_ctx* ctx, float* h_lr, int32_t* h_live);
int ppo_set_adaptive_lr(ppo_ctx* ctx, float lr, int32_t live);

/* Append the step-t record of all N environments to the trajectory buffer
 * (Algorithm 2: D <- D u {(obs, actions, rew, done)}), plus the behaviour
 * policy's log-prob and value that PPO needs.  Device inputs:
 *   d_obs     [N][n_views][in_c][in_h][in_w], fp32 or bf16 per desc.obs_dtype
 *   d_proprio [N][P] fp32     d_action [N][A] fp32 (for distillation: the teacher's action)
 *   d_logp, d_value, d_reward [N] fp32, d_done [N] uint8   (may all be NULL for a distillation student)
 * Images are narrowed to bf16 (round to nearest even) and stored channel-last.
 * t must be in [0, T); writing t = 0 starts a new rollout. */
int ppo_buffer_write(ppo_ctx* ctx, int32_t t, const void* d_obs, const float* d_proprio, const float* d_action,
                     const float* d_logp, const float* d_value, const float* d_reward, const uint8_t* d_done);

/* ppo_buffer_write for the environments [env_offset, env_offset + count) of step t only; every array
 * holds `count` rows.  This is the landing call for observations that arrive from several producers
 * (the simulator GPUs of Fig. 2b each own a range of environments and send their slice once per
 * step): the ranges may come in any order; step t counts as written once the ranges received for it
 * cover [0, N); within a rollout a write into a complete step starts that step afresh.  A range that
 * arrives while ALL T steps are complete is the first slice of the next rollout: every step then counts
 * as unwritten until its own ranges have covered [0, N) again (to replace a whole step of a complete
 * rollout in place use ppo_buffer_write).  count = 0 is a no-op; a range outside [0, N) is PPO_EINVAL. */
int ppo_buffer_write_range(ppo_ctx* ctx, int32_t t, int32_t env_offset, int32_t count, const void* d_obs, const float* d_proprio,
                           const float* d_action, const float* d_logp, const float* d_value, const float* d_reward,
                           const uint8_t* d_done);

/* Policy step of the collection loop (Algorithm 2: the policy maps the stacked observations of all
 * environments to actions; the record is appended once the simulators have stepped).  Stores the
 * step-t observations like ppo_buffer_write, runs the network forward on them with the current
 * parameters and samples the diagonal-Gaussian policy,
 *   a = mu + exp(logstd) * xi,   logp = sum_j [-((a_j-mu_j)/sigma_j)^2/2 - logstd_j - ln(2 pi)/2],
 * with the standard-normal draws xi supplied by the caller (d_noise [N][A] fp32, device).  Action,
 * log-prob and value go into the step-t slab and, where the pointers are not NULL, to the DEVICE
 * arrays d_action [N][A], d_logp [N], d_value [N] (fp32), which may lie in the memory of d_obs or
 * d_proprio but not of each other.  The step counts as written only after
 * ppo_buffer_write_outcome(t).  Actor-critic contexts only (else PPO_ESTATE); t = 0 starts a new rollout. */
int ppo_act(ppo_ctx* ctx, int32_t t, const void* d_obs, const float* d_proprio, const float* d_noise, float* d_action,
            float* d_logp, float* d_value);
/* Reward and termination flag of step t (device, [N] fp32 / uint8), known only after the
 * simulators have stepped (Algorithm 2: obs, rew, done <- step(actions)); completes a record
 * begun by ppo_act, or replaces these two fields of a record written by ppo_buffer_write.
 * PPO_ESTATE when step t holds no record. */
int ppo_buffer_write_outcome(ppo_ctx* ctx, int32_t t, const float* d_reward, const uint8_t* d_done);

/* Recurrent nets (lstm_layers > 0): the LSTM state of every environment at the START of the rollout in the
 * buffer (the state the acting policy had when it took step 0), DEVICE fp32 arrays [lstm_layers][N][lstm_units];
 * NULL = zeros.  Kept until the next call; a new context starts from zeros.  PPO_ESTATE for a feed-forward net. */
int ppo_buffer_write_state(ppo_ctx* ctx, const float* d_h0, const float* d_c0);

/* Read back the step-t images as stored (bf16) into a DEVICE array in the caller's layout
 * [N][n_views][in_c][in_h][in_w] (bf16).  Test hook for the write path. */
int ppo_buffer_read_obs(ppo_ctx* ctx, int32_t t, void* d_obs_bf16);

/* Generalised advantage estimation over the buffer, per environment, reverse in time:
 *   delta_t = r_t + gamma (1-d_t) V_{t+1} - V_t,  A_t = delta_t + gamma lambda (1-d_t) A_{t+1},  R_t = A_t + V_t
 * with V_T = d_last_value[n] (device, [N] fp32).  Needs all T steps written (else PPO_ESTATE). */
int ppo_gae(ppo_ctx* ctx, const float* d_last_value, float gamma, float lambda);
/* Copy advantages and returns ([T][N] fp32) to DEVICE arrays (either may be NULL). */
int ppo_get_adv_ret(ppo_ctx* ctx, float* d_adv, float* d_ret);

/* The permutation the next update will use for `epoch` (device kernel, result copied to
 * HOST int32[N*T]); minibatch m is entries [m*B, (m+1)*B).  A recurrent net shuffles whole environments:
 * the first N entries are then a permutation of 0..N-1 and the rest of h_perm is left untouched. */
int ppo_permutation(ppo_ctx* ctx, uint64_t seed, uint64_t update_idx, uint64_t epoch, int32_t* h_perm);

/* ppo_permutation for callers that cannot allocate device memory (code under HIP graph capture, tight serving
 * loops, harnesses that forbid hipMalloc): needs no context and calls no hipMalloc / hipFree or any allocating
 * routine.  The same kernels write the permutation of 0..S-1 for (seed, update_idx, epoch) into the DEVICE array
 * d_perm [S] (int32, caller-owned), enqueued on hip_stream (a hipStream_t, may be NULL); nothing synchronises.
 * Their scratch (none up to 8192 units; beyond, histogram, bucket starts and bucket-ordered indices) lives in a
 * static device array of the library, 4.4 MiB per GPU the library is used on, resolved once per device on the first call there (or by
 * ppo_create).  S <= PPO_STATIC_PERM_MAX (else PPO_ESHAPE); S = 0 is a no-op.  All calls on one GPU share that
 * array: two calls whose work overlaps in time on one GPU (different streams, or different threads) race;
 * calls on one stream are ordered and safe.  Errors are reported through ppo_last_error(NULL). */
#define PPO_STATIC_PERM_MAX (1 << 20)
int ppo_permutation_static(int64_t S, uint64_t seed, uint64_t update_idx, uint64_t epoch, int32_t* d_perm, void* hip_stream);

/* TrainPPO (Algorithm 2): epochs x minibatches of forward, clipped-surrogate + value +
 * entropy loss, backward and one Adam step each.  Needs ppo_gae (else PPO_ESTATE).
 * host_stats: HOST array [epochs*minibatches] or NULL (NULL = fully asynchronous). */
int ppo_update(ppo_ctx* ctx, const ppo_hparams* hp, ppo_mb_stats* host_stats);

/* Distillation update of a student (has_value_head = 0): MSE between the student's
 * action and the teacher action stored in the buffer's action slot; no GAE needed.
 * With hp->aux_dim = X > 0 the last X head columns are an auxiliary regression output (the deployed
 * student's object-position output, Sec. IV-C) whose target sits in the same columns of the action
 * slot; the paper gives no weighting, the loss taken is
 *   L = mean_b[ 1/(A-X) sum_{j<A-X} e_bj^2 ] + aux_coef * mean_b[ 1/X sum_{j>=A-X} e_bj^2 ],
 * and the two means are reported as pi_loss and v_loss.  X = 0: the mean over batch and all A columns. */
int distill_update(ppo_ctx* ctx, const ppo_hparams* hp, ppo_mb_stats* host_stats);

/* Forward only, on `count` buffer samples given by DEVICE int32 indices d_idx (NULL = samples
 * 0..count-1): action means to d_mu [count][A] fp32 and values to d_v [count] fp32 (may be NULL). */
int ppo_forward(ppo_ctx* ctx, const int32_t* d_idx, int64_t count, float* d_mu, float* d_v);

/* ---------------------------------------------------------------------------------------------------------------
 * Operators of a policy that answers in tokens (a categorical head over a vocabulary, sequences of uneven length).
 *
 * They need no context and allocate nothing: every array is the caller's, results included.  Work is enqueued on
 * hip_stream (a hipStream_t, may be NULL) of the CURRENT device, where all arrays must lie; nothing synchronises, and
 * every call may be recorded into a graph.  d_ws is scratch of at least the bytes that the *_ws_bytes function gives
 * for the same sizes (0: d_ws may be NULL), 16-byte aligned; nothing is kept in it between calls, and two calls whose work may overlap in time
 * need two of them (so do two captured graphs that may).  Errors are reported through ppo_last_error(NULL); arguments are
 * checked before any HIP call.  The same call gives the same results, bit for bit, every time (the order in which a row is added
 * up goes by its length, its alignment and the number of rows).  An empty call (no rows, tokens or
 * sequences) is allowed; the array pointers that it would read may then be NULL.
 *
 * `dtype` is the type of the large arrays: 0 fp32, 1 bf16, 2 fp16; everything else is fp32 or as declared, and every sum
 * is held in fp32 or more.  Rows may lie `ld` elements apart (ld >= their length); elements between them are neither
 * read nor written.  Arrays need the alignment of their element type only.
 * --------------------------------------------------------------------------------------------------------------- */
#define PPO_TOKEN_MAX_VOCAB (1 << 24)
#define PPO_TOKEN_MAX_ROWS ((1 << 24) - 1) /* rows of one call; half as many pairs */

/* Dropout whose mask is a function of (seed, layer, row id, column) and is never stored, so that the pass that collects
 * a rollout, every later pass over the same samples in any order, and the backward pass drop the same units:
 *   y = keep ? x * 65536 / (65536 - q) : 0  (+ residual),   q = round(65536 p), 0 <= p <= 1.
 * Column c of a row with id r is kept where the 16-bit field c % 4 (from the low end) of output c / 4 of the SplitMix64
 * stream of (seed, layer, r) - the streams that ppo_permutation sorts - is at least q.  A dropped x is not looked at
 * (NaN included).  d_row_ids: int64 [rows], e.g. flat sample indices; NULL: a row's id is its number.  The backward pass
 * is the same call on the gradient without d_residual.  d_y may be d_x or d_residual (with the same row stride). */
int ppo_dropout(int32_t dtype, int64_t rows, int64_t cols, const void* d_x, int64_t ld_x, const int64_t* d_row_ids,
                const void* d_residual, int64_t ld_residual, double p, uint64_t seed, uint64_t layer, void* d_y, int64_t ld_y,
                void* hip_stream);

/* Log-probability of the chosen token and entropy of every row of logits, z = logits / temperature:
 *   logp = z_t - log sum_j exp z_j,   H = -sum_j p_j log p_j   (a term with p_j = 0 counts 0: logits may be -infinity).
 * d_target int32 [rows].  A row is IDLE if its target lies outside [0, vocab) - its logits are not read then - or if all of
 * its logits are -infinity: logp and H are 0.  A NaN or +infinity among the logits of any other row gives NaN.
 * d_entropy may be NULL.  d_stat (may be NULL): fp32 [rows][2], what the backward pass needs of the row. */
int64_t ppo_token_logp_ws_bytes(int64_t rows, int64_t vocab);
int ppo_token_logp(int32_t dtype, int64_t rows, int64_t vocab, const void* d_logits, int64_t ld, const int32_t* d_target,
                   float temperature, float* d_logp, float* d_entropy, float* d_stat, void* d_ws, int64_t ws_bytes, void* hip_stream);
/* Gradient of sum_r (dlogp_r logp_r + dentropy_r H_r) by the logits, rounded once to their type:
 *   dlogits_j = [dlogp ([j = t] - p_j) - dentropy p_j (log p_j + H)] / temperature;   0 in idle rows.
 * d_stat and d_entropy as ppo_token_logp left them; d_dentropy NULL (then d_entropy is not read): no entropy term.
 * d_dlogits may be d_logits (with the same row stride). */
int ppo_token_logp_backward(int32_t dtype, int64_t rows, int64_t vocab, const void* d_logits, int64_t ld, const int32_t* d_target,
                            float temperature, const float* d_stat, const float* d_dlogp, const float* d_entropy,
                            const float* d_dentropy, void* d_dlogits, int64_t ld_d, void* hip_stream);

/* The clipped policy loss on tokens (ppo_update's, for a categorical head) with a KL term against a reference policy, and
 * its gradient, in one pass over the logits.  With rho = exp(logp - logp_old) and x = logp_ref - logp, a token's loss is
 *   l = -min(rho A, clip(rho, 1 - clip_lo, 1 + clip_hi) A) + kl_coef (exp x - x - 1) - ent_coef H
 * (exp x - x - 1: the non-negative one-sample estimate of KL(policy || reference)), and L = scale sum_r weight_r l_r over
 * the rows that are not idle.  At ties the unclipped branch carries the gradient.  A weight of 0 hides no term that is infinite or no
 * number: rows that do not count (padding) have a target outside [0, vocab). */
typedef struct {
  float temperature;      /* > 0, and large enough for 2 / temperature to be finite */
  float clip_lo, clip_hi; /* >= 0; clip_lo <= 1 */
  float kl_coef;          /* >= 0; without d_logp_ref it must be 0.  0 with one: the estimate is reported only */
  float ent_coef;         /* 0: the entropy is neither computed nor reported; ent_coef * scale must be finite */
  float scale;            /* e.g. 1 / number of tokens; a loss scale for fp16 gradients */
} ppo_token_hparams;
/* Inputs [rows]: d_target, d_logp_old, d_adv; d_logp_ref, d_weight may be NULL (no KL; weights 1).  They are not read in idle
 * rows.  Outputs: d_dlogits (dL/dlogits; may be d_logits with the same row stride), d_logp [rows] (may be NULL), d_stats [8]:
 *   0 L, 1..3 its weighted sums scale sum w (-min(..)), scale sum w (exp x - x - 1), scale sum w H, then over the rows that are
 *   not idle 4 mean of (rho - 1) - log rho, 5 share with rho outside the clip range, 6 their number, 7 1 if L is not finite. */
int64_t ppo_token_loss_ws_bytes(int64_t rows, int64_t vocab);
int ppo_token_loss(int32_t dtype, int64_t rows, int64_t vocab, const void* d_logits, int64_t ld, const int32_t* d_target,
                   const float* d_logp_old, const float* d_logp_ref, const float* d_adv, const float* d_weight,
                   const ppo_token_hparams* hp, void* d_dlogits, int64_t ld_d, float* d_logp, float* d_stats, void* d_ws,
                   int64_t ws_bytes, void* hip_stream);

/* Sequences of the calls below are packed one behind the other: sequence k holds the tokens [d_offsets[k], d_offsets[k+1])
 * (int64, non-decreasing, inside [0, tokens]; a sequence may be empty; tokens <= 2^34, sequences <= 2^30).  Offsets outside [0, tokens] are taken as its
 * nearer end, and of decreasing ones the results are unspecified; no memory outside the arrays is touched either way.
 * d_mask: uint8 [tokens], 0 = the token is passed over (a prompt, a tool's answer) and its inputs may be anything; NULL: none.
 * (Tokens whose row was idle in ppo_token_logp, with a log-probability of 0, belong there.)
 *
 * Preference loss on `pairs` pairs of sequences, k chosen and pairs + k rejected, from the tokens' log-probabilities.
 * S = sum (logp - logp_ref) over a sequence's unmasked tokens (their mean if length_mean), D = S_chosen - S_rejected:
 *   kind 0:  l = -(1 - label_smoothing) log sigmoid(beta D) - label_smoothing log sigmoid(-beta D)
 *   kind 1:  l = (D - 1 / (2 beta))^2
 * L = scale sum_k l_k over the pairs with an unmasked token in both sequences.  d_logp_ref, d_margin may be NULL.
 * Outputs: d_dlogp [tokens] (dL/dlogp; 0 for masked tokens and tokens of no sequence), d_margin [pairs] (beta D; 0 for a pair
 * that does not count), d_stats [7]: 0 L, then over the pairs that count 1 share with D > 0, 2 mean beta D, 3, 4 mean beta S of
 * the chosen and of the rejected, 5 their number, 6 1 if L is not finite. */
typedef struct {
  int32_t kind, length_mean;
  float beta;            /* > 0 */
  float label_smoothing; /* in [0, 1]; used by kind 0 */
  float scale;           /* e.g. 1 / pairs */
} ppo_pair_hparams;
int64_t ppo_pair_ws_bytes(int64_t pairs, int64_t tokens);
int ppo_pair_loss(int64_t pairs, int64_t tokens, const float* d_logp, const float* d_logp_ref, const uint8_t* d_mask,
                  const int64_t* d_offsets, const ppo_pair_hparams* hp, float* d_dlogp, float* d_margin, float* d_stats,
                  void* d_ws, int64_t ws_bytes, void* hip_stream);

/* ppo_gae over packed sequences: with ' the next unmasked token of the sequence,
 *   A_t = r_t + gamma V' - V_t + gamma lambda A',   R_t = A_t + V_t;
 * behind a sequence's last unmasked token A' = 0 and V' = d_last_value[k] (fp32 [sequences], the value of the state behind a
 * sequence that was cut off; NULL: 0, every sequence ended).  Masked tokens and tokens of no sequence get 0. */
int64_t ppo_token_gae_ws_bytes(int64_t sequences, int64_t tokens);
int ppo_token_gae(int64_t sequences, int64_t tokens, const float* d_reward, const float* d_value, const uint8_t* d_mask,
                  const int64_t* d_offsets, const float* d_last_value, double gamma, double lambda, float* d_adv, float* d_ret,
                  void* d_ws, int64_t ws_bytes, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif
