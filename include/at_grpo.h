/*
 * at_grpo.h -- C ABI of the MI355X (gfx950) AT-GRPO policy-loss library.
 *
 * The library computes, on one GPU, the per-token policy loss of AT-GRPO
 * (arXiv 2510.11062): agent- and turn-wise grouped advantages (Alg. 1, Phase 1; Eq. 1),
 * log pi_theta(token) from the LM head (the ratio below Eq. 2), the clipped surrogate with
 * masked averaging per policy (Eq. 2; per-model batches B_m of Sec. 3) and its gradients
 * with respect to the final hidden states and the head weights.  Beside that, of the layers in front of
 * the head: norms and rotation of queries and keys with their gradient, a paged cache of the rollout's keys
 * and values, and attention over it.
 *
 * Conventions common to every call
 *   - Pointers are DEVICE pointers unless the comment says "host".  The caller owns every
 *     buffer; the library never allocates, frees or keeps a pointer after the call returns.
 *   - All work is enqueued on `hip_stream` (a hipStream_t cast to void*; NULL = default
 *     stream).  No call synchronises with the host.  Scalar results live in device memory.
 *   - `workspace` is caller-provided device scratch of at least at_grpo_workspace_bytes()
 *     bytes, 256-byte aligned.  Its first int32 is an error word: 0, or the bit-or of
 *     AT_GRPO_DATA_* flags raised by data that is only visible on the device.  Offending
 *     elements are treated as masked out.  Read it after synchronising the stream.  (The calls on queries,
 *     keys and the cache use the first word as scratch: they raise their flags in `data_error`.)
 *   - Return value: an at_grpo_status.  Argument errors are detected on the host before
 *     anything is launched; nothing is thrown and nothing aborts.
 *   - Matrices are row-major and dense.  `hidden` is [n_tok, H]; each head W is [V, H].
 *   - dtype AT_GRPO_BF16 requires H % 64 == 0; AT_GRPO_F32 requires H % 32 == 0.
 */
#ifndef AT_GRPO_H_
#define AT_GRPO_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  AT_GRPO_OK = 0,
  AT_GRPO_EINVAL = 1,       /* null pointer, non-positive size, inconsistent arguments */
  AT_GRPO_EUNSUPPORTED = 2, /* dtype / shape the kernels do not cover                 */
  AT_GRPO_EWORKSPACE = 3,   /* workspace missing, misaligned or too small             */
  AT_GRPO_EHIP = 4,         /* a HIP runtime call or kernel launch failed             */
  AT_GRPO_ESCRATCH = 5      /* input too large for the library's fixed scratch array  */
} at_grpo_status;

typedef enum { AT_GRPO_F32 = 0, AT_GRPO_BF16 = 1 } at_grpo_dtype;

/* How Eq. (2)'s expectation over the per-model batch is taken (the paper writes a mean over
 * groups and candidates; credit is per response token, Sec. 4.1):
 *   TOKEN_MEAN           loss_m = -(1/n_m) sum_t l_t          over the n_m response tokens of B_m
 *   SEQ_MEAN_TOKEN_MEAN  loss_m = -(1/R_m) sum_r (1/len_r) sum_{t in r} l_t                  */
typedef enum { AT_GRPO_AGG_TOKEN_MEAN = 0, AT_GRPO_AGG_SEQ_MEAN_TOKEN_MEAN = 1 } at_grpo_agg;

/* F_norm of Eq. (1): the group's standard deviation (plus eps_std), or 1. */
typedef enum { AT_GRPO_NORM_STD = 0, AT_GRPO_NORM_NONE = 1 } at_grpo_norm;

/* May be or'ed into a `norm` argument by a caller whose group buffers all hold
 * min(R, number of keys) entries (seg_offsets one more): the call then also writes the entries
 * behind the last group and behind the last listed response (0; -1 for best), so that the buffers
 * need not be cleared first.  Without it nothing is written there. */
enum { AT_GRPO_NORM_FILL = 256 };

/* Which responses form a group in Eq. (1): the paper's agent- and turn-wise key, or one of the two
 * groupings it argues against (Sec. 4.1, Fig. 3; Sec. 5.3), kept for comparison runs. */
typedef enum {
  AT_GRPO_GROUP_BY_AGENT_TURN = 0, /* (e, i, t): AT-GRPO, Alg. 1                                      */
  AT_GRPO_GROUP_BY_TRAJECTORY = 1, /* e alone: every candidate of a task in one group (GRPO on the MAS) */
  AT_GRPO_GROUP_BY_PARALLEL = 2    /* (e, i, t) at t = 0, one group per candidate at t > 0: what
                                      sampling K whole trajectories in parallel yields               */
} at_grpo_group_by;

/* Bits of the device error word (workspace[0]). */
enum {
  AT_GRPO_DATA_ID_RANGE = 1,     /* env/agent/turn id outside its extent              */
  AT_GRPO_DATA_REWARD = 2,       /* non-finite reward (the response then takes no part) */
  AT_GRPO_DATA_TOKEN_RANGE = 4,  /* token_id outside [0, V) on an unmasked row        */
  AT_GRPO_DATA_SEQLENS = 8,      /* cu_seqlens not monotone within [0, n_tok]         */
  AT_GRPO_DATA_AGENT_RANGE = 16, /* resp_agent / head_of_agent entry out of range     */
  AT_GRPO_DATA_PAGE = 32,        /* page id outside the cache, or a token behind its page table */
  AT_GRPO_DATA_POSITION = 64     /* position outside the rotation table               */
};

/* Bits of clip_mask[t] (Eq. 2's clip, decided in log space on d = logp - old_logp, one fp32
 * subtraction, against lo = (float)log1p(-eps_low) and hi = (float)log1p(eps_high)). */
enum {
  AT_GRPO_CLIP_LOW = 1,       /* d < lo : ratio below 1 - eps_low                    */
  AT_GRPO_CLIP_HIGH = 2,      /* d > hi : ratio above 1 + eps_high                   */
  AT_GRPO_CLIP_ZERO_GRAD = 4  /* min() selects the clipped branch: no gradient       */
};

/* Which call a workspace is sized for. */
typedef enum {
  AT_GRPO_CALL_GROUP_ADVANTAGE = 0,
  AT_GRPO_CALL_TOKEN_LOGPROB = 1,
  AT_GRPO_CALL_POLICY_LOSS_FWD = 2,
  AT_GRPO_CALL_POLICY_LOSS_BWD = 3,
  AT_GRPO_CALL_SURROGATE = 4,
  AT_GRPO_CALL_HEAD_UPDATE = 5,  /* size does not depend on the other arguments */
  AT_GRPO_CALL_DIAGNOSTICS = 6,
  AT_GRPO_CALL_TOKEN_ENTROPY = 7,
  AT_GRPO_CALL_POLICY_LOSS_FWD_BWD = 8,
  AT_GRPO_CALL_QK_NORM_ROPE_BWD = 9 /* size does not depend on the other arguments */
} at_grpo_call;

/*
 * A batch of rollout tokens (Alg. 1 Phase 2: the per-model batches B_m, all models at once).
 * Row t of `hidden` is the final hidden state that predicts token_id[t].  Response r owns rows
 * [cu_seqlens[r], cu_seqlens[r+1]); rows owned by no response, and rows with mask 0, take no
 * part (packed layout: mask == NULL; padded layout: fixed-size slots plus mask).  With
 * n_heads > 1 the rows of response r go to head head_of_agent[resp_agent[r]] (the role
 * mapping sigma of Sec. 3); with n_heads == 1 both arrays may be NULL.
 */
typedef struct {
  int32_t dtype;             /* at_grpo_dtype of hidden and W                            */
  int32_t H, V, n_heads;     /* n_heads in [1, 16]                                       */
  int64_t n_tok;             /* rows of hidden / token_id / mask (padding included)      */
  int32_t n_resp;            /* R                                                        */
  int32_t n_agent;           /* length of head_of_agent (ignored if n_heads == 1)        */
  const int64_t* cu_seqlens; /* [R+1] device                                             */
  const void* hidden;        /* [n_tok, H] device                                        */
  const void* const* W;      /* HOST array of n_heads device pointers, each [V, H]       */
  const int32_t* token_id;   /* [n_tok] device, sampled token, 0 <= id < V               */
  const uint8_t* mask;       /* [n_tok] device or NULL (all ones)                        */
  const int32_t* resp_agent; /* [R] device or NULL                                       */
  const int32_t* head_of_agent; /* [n_agent] device or NULL                              */
} at_grpo_batch;

/*
 * Agent- and turn-wise grouping and group-relative advantages.
 * Alg. 1 ("Define group key g <- hash(e, i, t) and compute advantages"), Sec. 4.1
 * "Agent- and Turn-wise Grouping", Eq. (1).
 *
 * key(r) = (env_id[r] * n_agent + agent_id[r]) * n_turn + turn_id[r]; groups are numbered
 * densely in ascending key order; keys that do not occur produce no group.
 *   group_id[R]      dense group of each response (-1 for a response with an id out of range or a
 *                    non-finite reward: it joins no group, gets advantage 0 and does not touch the
 *                    statistics of the others)
 *   n_groups[1]      G
 *   seg_offsets[G+1] CSR offsets into perm; the buffer must hold min(R, n_env*n_agent*n_turn)+1
 *   perm[R]          responses sorted by key, ties in ascending original index (stable)
 *   adv[R]           (reward - mean_g) / (std_g + eps_std)   [NORM_STD]   or reward - mean_g
 *                    [NORM_NONE]; std uses divisor n_g - ddof (0 if that is <= 0); a group
 *                    whose rewards are all the same fp32 value gets exactly 0
 *   group_mean[G], group_std[G]  optional (NULL to skip)
 * ddof is 0 or 1.  Arithmetic is fp32, two passes (mean, then squared deviations): groups of up to 16
 * members are summed sequentially in perm order, larger ones as 64 lane-strided partial sums (member
 * j of the group goes to partial j mod 64) that are combined in a fixed order; either way the result
 * does not depend on the order in which the responses arrive or on the run.
 */
int at_grpo_group_advantage(int32_t n_resp, int32_t n_env, int32_t n_agent, int32_t n_turn,
                            const int32_t* env_id, const int32_t* agent_id, const int32_t* turn_id,
                            const float* reward, float eps_std, int32_t ddof, int32_t norm,
                            int32_t* group_id, int32_t* n_groups, int32_t* seg_offsets,
                            int32_t* perm, float* adv, float* group_mean, float* group_std,
                            void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * at_grpo_group_advantage under another grouping key (`group_by`, see at_grpo_group_by): everything
 * else, including the canonical numbering (ascending key), is the same.
 *   TRAJECTORY  key = e: agent_id and turn_id are only range-checked; seg_offsets needs min(R, n_env) + 1
 *   PARALLEL    key = ((e * n_agent + i) * n_turn + t) * n_sample + (t > 0 ? sample_id[r] : 0), with
 *               sample_id[R] the candidate index c in [0, n_sample): every group at t > 0 is a single
 *               response and gets advantage 0 (the degenerate case Sec. 4.1 describes);
 *               seg_offsets needs min(R, n_env * n_agent * n_turn * n_sample) + 1 entries
 * sample_id and n_sample are ignored otherwise.  Workspace: at_grpo_group_advantage_keyed_workspace_bytes.
 */
int at_grpo_group_advantage_keyed(int32_t group_by, int32_t n_resp, int32_t n_env, int32_t n_agent,
                                  int32_t n_turn, int32_t n_sample, const int32_t* env_id,
                                  const int32_t* agent_id, const int32_t* turn_id, const int32_t* sample_id,
                                  const float* reward, float eps_std, int32_t ddof, int32_t norm,
                                  int32_t* group_id, int32_t* n_groups, int32_t* seg_offsets, int32_t* perm,
                                  float* adv, float* group_mean, float* group_std, void* workspace,
                                  size_t workspace_bytes, void* hip_stream);
size_t at_grpo_group_advantage_keyed_workspace_bytes(int32_t group_by, int32_t n_resp, int32_t n_env,
                                                     int32_t n_agent, int32_t n_turn, int32_t n_sample);

/*
 * The same with the step in front of it: agent-wise credit assignment, Eq. (3) of Sec. 4.1,
 *   reward[r] = alpha * r_team[r] + r_loc[r]     (one fp32 multiplication, then one fp32 addition)
 * feeds Eq. (1), and the greedy choice of tree-structured sampling (Alg. 1, "c* <- arg max_c r^(c)")
 * is taken on the same groups:
 *   reward[R]   output, the mixed reward (also what adv, group_mean, group_std are computed from)
 *   best[G]     optional (NULL to skip): response index of the candidate with the largest reward of
 *               each group, the lowest response index among equal rewards; the buffer must hold
 *               min(R, n_env*n_agent*n_turn) entries
 * r_team[R], r_loc[R] are inputs; reward may be one of them itself (mixed in place), in whole; alpha must be
 * finite.  Every other argument, the workspace size
 * (AT_GRPO_CALL_GROUP_ADVANTAGE) and the error behaviour are those of at_grpo_group_advantage; a
 * non-finite mixed reward raises AT_GRPO_DATA_REWARD.
 */
int at_grpo_group_advantage_mixed(int32_t n_resp, int32_t n_env, int32_t n_agent, int32_t n_turn,
                                  const int32_t* env_id, const int32_t* agent_id, const int32_t* turn_id,
                                  const float* r_team, const float* r_loc, float alpha, float eps_std,
                                  int32_t ddof, int32_t norm, float* reward, int32_t* group_id,
                                  int32_t* n_groups, int32_t* seg_offsets, int32_t* perm, float* adv,
                                  float* group_mean, float* group_std, int32_t* best, void* workspace,
                                  size_t workspace_bytes, void* hip_stream);

/*
 * at_grpo_group_advantage for callers that cannot allocate device memory or hand over a workspace
 * (code under HIP graph capture, tight serving loops, harnesses that forbid hipMalloc): the scratch
 * is a fixed array of at_grpo_static_scratch_bytes() bytes (2 MiB) in the library's own device
 * memory, which every GPU the library runs on holds until the process ends.  The call allocates and
 * frees nothing.  Same inputs, outputs, arithmetic and results as at_grpo_group_advantage, plus
 *   data_error[1]  optional device output (NULL to skip): the error word of this call (AT_GRPO_DATA_*)
 * Limit: about 12 * n_resp + 8 * n_env * n_agent * n_turn bytes must not exceed
 * at_grpo_static_scratch_bytes() = 2 MiB (65 536 responses over 65 536 keys fit, as does every workload of the paper's shape); beyond it the call
 * returns AT_GRPO_ESCRATCH and launches nothing.
 * All calls on one GPU share that GPU's array: calls that may overlap on one GPU (different streams
 * or threads) race and must be serialised by the caller.  Everything the kernels need cleared is
 * cleared by the call itself with fill kernels (no memset nodes), so it may be captured in a graph;
 * the first call on a device looks the array's address up and should be made outside a capture.
 */
size_t at_grpo_static_scratch_bytes(void);
int at_grpo_group_advantage_static(int32_t n_resp, int32_t n_env, int32_t n_agent, int32_t n_turn,
                                   const int32_t* env_id, const int32_t* agent_id, const int32_t* turn_id,
                                   const float* reward, float eps_std, int32_t ddof, int32_t norm,
                                   int32_t* group_id, int32_t* n_groups, int32_t* seg_offsets,
                                   int32_t* perm, float* adv, float* group_mean, float* group_std,
                                   int32_t* data_error, void* hip_stream);

/*
 * log pi_theta(token_id[t]) and the log-sum-exp of the head logits for every participating row
 * (the policy probability inside r(theta) below Eq. 2).  Logits z[t, v] = <hidden[t], W_m[v]>
 * are produced tile by tile on the matrix cores and reduced on the fly; they are never written
 * to memory.  Rows that take no part get logp = lse = 0.
 *   logp[n_tok], lse[n_tok] (lse may be NULL)
 */
int at_grpo_token_logprob(const at_grpo_batch* batch, float* logp, float* lse,
                          void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * Clipped surrogate of Eq. (2) given log-probs (the stage after the head):
 *   d_t = logp_t - old_logp_t,  r_t = exp(d_t),  A_t = adv[response of t]
 *   l_t = min(r_t A_t, clip(r_t, 1 - eps_low, 1 + eps_high) A_t)
 *   loss[m] = - sum_{t in B_m} w_t l_t      (w_t per `agg`)
 *   clip_mask[n_tok], n_valid[n_heads] (participating rows per head)
 * Only the batch's layout fields are used (n_tok, n_resp, cu_seqlens, mask, token_id for the
 * range check, resp_agent, head_of_agent, n_heads, V); hidden and W may be NULL.
 * The reduction is a fixed-order tree: results are bit-reproducible.
 */
int at_grpo_surrogate_from_logp(const at_grpo_batch* batch, const float* logp, const float* old_logp,
                                const float* adv, float eps_low, float eps_high, int32_t agg,
                                float* loss, uint8_t* clip_mask, int32_t* n_valid,
                                void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * at_grpo_token_logprob plus a monitor: the entropy of the next-token distribution at every
 * participating row, H_t = - sum_v p_v ln p_v = lse_t - sum_v p_v z_v, from one more partial sum per
 * vocabulary tile in the same pass (the paper trains with entropy coefficient 0, App. C.1; nothing in
 * the loss uses it).  Rows that take no part get 0.
 *   logp[n_tok], lse[n_tok] (may be NULL), entropy[n_tok]
 * Workspace: AT_GRPO_CALL_TOKEN_ENTROPY.
 */
int at_grpo_token_entropy(const at_grpo_batch* batch, float* logp, float* lse, float* entropy,
                          void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * Monitors of the clipped-ratio update of Eq. (2), per policy, over the same participating rows as
 * at_grpo_surrogate_from_logp (the paper reports none of them; its entropy coefficient is 0 and Eq. 2
 * carries no KL term):
 *   counts[n_heads][4]  rows, rows with d < lo, rows with d > hi, rows on the clipped branch
 *                       (AT_GRPO_CLIP_LOW / _HIGH / _ZERO_GRAD counted), d = logp - old_logp in fp32
 *   stats[n_heads][2]   mean of exp(d) - 1 - d (sample estimate of KL(pi_old || pi_theta)), mean exp(d)
 * Sums are taken in a fixed order.  Workspace: AT_GRPO_CALL_DIAGNOSTICS (needs batch->n_resp only).
 */
int at_grpo_surrogate_diagnostics(const at_grpo_batch* batch, const float* logp, const float* old_logp,
                                  const float* adv, float eps_low, float eps_high, int32_t* counts,
                                  float* stats, void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * Forward of the policy loss: at_grpo_token_logprob followed by at_grpo_surrogate_from_logp.
 * Outputs logp[n_tok], lse[n_tok] (both are needed by the backward), loss[n_heads],
 * clip_mask[n_tok], n_valid[n_heads].
 */
int at_grpo_policy_loss_fwd(const at_grpo_batch* batch, const float* old_logp, const float* adv,
                            float eps_low, float eps_high, int32_t agg,
                            float* loss, float* logp, float* lse, uint8_t* clip_mask, int32_t* n_valid,
                            void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * Backward of sum_m grad_loss[m] * loss[m] (grad_loss == NULL means all ones):
 *   g_t = -w_t A_t r_t [unclipped branch selected] grad_loss[m]
 *   dZ[t, v]     = g_t (1[v = token_id[t]] - exp(z[t, v] - lse_t))     (logits recomputed)
 *   d_hidden[t]  = sum_v dZ[t, v] W_m[v]          dtype of hidden, [n_tok, H]; rows that take
 *                                                  no part or have g_t = 0 are exactly 0
 *   dW[m][v]     = sum_t dZ[t, v] hidden[t]       fp32 [V, H] per head; dW is a HOST array of
 *                                                  n_heads device pointers; overwritten, or
 *                                                  added to when accumulate_dW != 0
 * logp and lse are the forward's outputs.  Rows with g_t = 0 are skipped entirely.
 */
int at_grpo_policy_loss_bwd(const at_grpo_batch* batch, const float* old_logp, const float* adv,
                            const float* logp, const float* lse,
                            float eps_low, float eps_high, int32_t agg, const float* grad_loss,
                            void* d_hidden, float* const* dW, int32_t accumulate_dW,
                            void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * One training step's worth of Eq. (2): at_grpo_policy_loss_fwd followed by at_grpo_policy_loss_bwd
 * (same arguments, same outputs, same error behaviour), computed from ONE pass over the logits.  For
 * AT_GRPO_BF16, rows whose response has a non-zero advantage (only they can carry gradient) have their
 * logits produced once: with the reference c_t = z[t, token_id[t]] (one dot product per row) the forward
 * tile writes e[t, v] = exp(z[t, v] - c_t) in bf16, as dZ would be written, and
 *   lse_t = c_t + ln S_t,  S_t = sum_v e[t, v],   dZ[t, v] = a_t (e[t, v] - S_t 1[v = token_id[t]]),
 *   a_t = -g_t / S_t
 * so that d_hidden and dW follow from e by two contractions and a per-row factor, without recomputing the
 * logits.  A launch in which some S_t leaves [1, 2^60) (the sampled token about e^88 times less likely than
 * the mode, or non-finite inputs) is redone by the two-pass kernels, on the device, without host
 * involvement.  Rows of zero-advantage responses only get logp / lse.  AT_GRPO_F32 runs the two calls one
 * after the other.  Results agree with the two-call sequence to rounding (e and the scaled hidden rows are
 * rounded to bf16 where that path rounds dZ).  Workspace: AT_GRPO_CALL_POLICY_LOSS_FWD_BWD.
 */
int at_grpo_policy_loss_fwd_bwd(const at_grpo_batch* batch, const float* old_logp, const float* adv,
                                float eps_low, float eps_high, int32_t agg, const float* grad_loss,
                                float* loss, float* logp, float* lse, uint8_t* clip_mask, int32_t* n_valid,
                                void* d_hidden, float* const* dW, int32_t accumulate_dW,
                                void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * Hyper-parameters of the head update (App. C.1: Adam, learning rate 1e-6, weight decay 0.01,
 * gradient clipping at 1.0; beta1, beta2 and eps are not stated there: 0.9, 0.999, 1e-8 are the
 * customary values).
 */
typedef struct {
  float lr, beta1, beta2, eps;
  float weight_decay;
  float max_grad_norm; /* 0 disables clipping                                                    */
  int32_t step;        /* 1 for the first update (bias correction 1 - beta^step)                 */
  int32_t decoupled;   /* 1: w <- w (1 - lr wd) before the step; 0: g <- g + wd w (L2 penalty)   */
} at_grpo_adam;

/*
 * "Update policy m" of Alg. 1 (Phase 2) for the head weights, with App. C.1's recipe:
 *   norm  = L2 norm of dW over all n_heads heads together
 *   g     = dW * min(1, max_grad_norm / (norm + 1e-6))
 *   m     <- beta1 m + (1 - beta1) g,   v <- beta2 v + (1 - beta2) g^2
 *   w     <- w - lr wd w - (lr / (1 - beta1^step)) m / (sqrt(v / (1 - beta2^step)) + eps)
 * (decoupled form; the coupled form adds wd w to g instead).  All arithmetic is fp32.
 *   W        HOST array of n_heads device pointers, each [V, H] in `dtype`, updated in place
 *   W_master HOST array of device pointers to the fp32 weights that are stepped, each [V, H];
 *            required for AT_GRPO_BF16 (W then receives their bf16 rounding, nearest-even);
 *            ignored for AT_GRPO_F32 (W itself is stepped)
 *   dW       HOST array of device pointers, fp32 [V, H] (what at_grpo_policy_loss_bwd produced,
 *            possibly accumulated over several mini-batches); read only
 *   m, v     HOST arrays of device pointers, fp32 [V, H], Adam moments, updated in place
 *   opt      host pointer
 *   grad_norm[2]  device output: the norm before clipping, and the factor applied
 * Every device pointer must be 16-byte aligned; H % 4 == 0.  Workspace: AT_GRPO_CALL_HEAD_UPDATE.
 * The norm is reduced in a fixed order, so results are reproducible run to run.
 */
int at_grpo_head_update(int32_t dtype, int32_t H, int32_t V, int32_t n_heads, void* const* W,
                        float* const* W_master, const float* const* dW, float* const* m,
                        float* const* v, const at_grpo_adam* opt, float* grad_norm,
                        void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * ---- In front of the head: queries, keys and the rollout's cache ---------------------------------
 * Tree sampling (Alg. 1 / "Tree-structured Sampling") draws the K candidates of a group from one prompt,
 * and the step then trains on all of them.  The calls below are the attention side of such a policy: norms
 * and rotation of queries and keys (with the gradient that training needs), the same on the way into a
 * paged cache, and attention that reads a prompt's keys and values once for the candidates that share it.
 *
 * Norms and rotation have a gradient here; the attention has none: these calls serve the rollout and the training pass's
 * norms, whose attention is the caller's.
 *
 * They have no error word of their own in a workspace: where `data_error` is not NULL the AT_GRPO_DATA_*
 * bits of offending elements are or'ed into that int32 in device memory, which the caller clears when it
 * likes (once per rollout, say).
 */

/* Rows of heads: element (t, h, d) lies at data + t * token_stride + h * head_stride + d (in elements of the
 * call's dtype).  Queries, keys and values may therefore be views of one projection's output, or stand head
 * by head.  data must be 16-byte aligned and both strides multiples of 16 bytes. */
typedef struct {
  void* data;
  int64_t token_stride, head_stride;
} at_grpo_rows;

/* Which elements of a head are rotated together, for i < rot_dim / 2: (i, i + rot_dim / 2), or (2 i, 2 i + 1). */
typedef enum { AT_GRPO_ROPE_HALF = 0, AT_GRPO_ROPE_INTERLEAVED = 1 } at_grpo_rope_layout;

/* How frequencies f_i = base^(-2 i / rot_dim) are scaled for contexts longer than `trained` positions. */
typedef enum {
  AT_GRPO_ROPE_PLAIN = 0,  /* f_i                                                                        */
  AT_GRPO_ROPE_LINEAR = 1, /* f_i / factor                                                               */
  AT_GRPO_ROPE_BASE = 2,   /* base * factor^(rot_dim / (rot_dim - 2)) in place of base; rot_dim > 2       */
  AT_GRPO_ROPE_PARTS = 3   /* f_i (g + (1 - g) / factor), g = clamp((turns_i - slow) / (fast - slow), 0, 1),
                              turns_i = trained * f_i / (2 pi): fast turning pairs keep their frequency   */
} at_grpo_rope_scaling;

typedef struct {
  int32_t rot_dim;    /* even, > 0                                                                       */
  int32_t scaling;    /* at_grpo_rope_scaling                                                            */
  double base;        /* > 0                                                                             */
  double factor;      /* >= 1 (ignored by PLAIN)                                                         */
  double trained, slow, fast; /* PARTS: > 0, and slow < fast                                             */
  double magnitude;   /* cos and sin are multiplied by it; > 0                                           */
} at_grpo_rope;

/*
 * The rotation table that the calls below read, computed in 64 bits and rounded once:
 *   table[n_pos][rot_dim / 2][2] = magnitude * (cos, sin)(p f_i), fp32, 16-byte aligned, p < n_pos
 */
int at_grpo_rope_table(const at_grpo_rope* rope, int32_t n_pos, float* table, void* hip_stream);

/* What a layer does to its queries and keys. */
typedef struct {
  int32_t dtype, D;         /* at_grpo_dtype of rows and weights; D % 8 == 0, 8 <= D <= 256              */
  int32_t rot_dim, layout;  /* even, 0 <= rot_dim <= D (0: no rotation); at_grpo_rope_layout             */
  int32_t n_pos;            /* positions in the table                                                    */
  float eps;                /* >= 0                                                                      */
  const float* table;       /* [n_pos][rot_dim / 2][2]; may be NULL where rot_dim == 0                   */
  const void* q_weight;     /* [D], 16-byte aligned, or NULL: queries are not normed                     */
  const void* k_weight;     /* [D], or NULL: keys are not normed                                         */
} at_grpo_norm_rope;

/*
 * Norm of every head's row and rotation by its token's position, in one pass:
 *   u = x / sqrt(mean(x^2) + eps) * weight     (u = x without a weight)
 *   y_a = c u_a - s u_b,  y_b = c u_b + s u_a  for the pairs (a, b) of the layout, (c, s) = table[position[t]]
 *   y_d = u_d for d >= rot_dim
 * in fp32, rounded once.  q [n_tok, Hq, D], k [n_tok, Hk, D]; Hk == 0 (or Hq == 0) leaves one of them out.
 * An output may be its input itself (same data and strides) or lie apart from it: one that meets it otherwise is
 * AT_GRPO_EINVAL (views of one buffer that do not meet have the same strides).  A token whose position lies
 * outside the table raises AT_GRPO_DATA_POSITION and gets rows of zeros.  n_tok == 0 is no error and does nothing.
 */
int at_grpo_qk_norm_rope(const at_grpo_norm_rope* layer, int32_t n_tok, int32_t Hq, int32_t Hk,
                         const at_grpo_rows* q, const at_grpo_rows* k, const int32_t* position,
                         const at_grpo_rows* q_out, const at_grpo_rows* k_out, int32_t* data_error,
                         void* hip_stream);

/*
 * Its gradient.  With g the rotated-back gradient of a row (g_a = c dy_a + s dy_b, g_b = c dy_b - s dy_a),
 * r = 1 / sqrt(mean(x^2) + eps) and n = x r:
 *   dx = r (g weight - n mean(g weight n)),   d_weight = sum over all rows of g n     (dx = g without a weight)
 *   dq, dk as q, k (dq may be dq_out or q itself, dk dk_out or k);  dq_weight[D], dk_weight[D] fp32, overwritten, required
 *   where the layer has the weight.
 * Tokens whose position lies outside the table get zeros and add nothing.  Sums are taken in a fixed order.
 * Workspace: AT_GRPO_CALL_QK_NORM_ROPE_BWD.
 */
int at_grpo_qk_norm_rope_bwd(const at_grpo_norm_rope* layer, int32_t n_tok, int32_t Hq, int32_t Hk,
                             const at_grpo_rows* dq_out, const at_grpo_rows* dk_out, const at_grpo_rows* q,
                             const at_grpo_rows* k, const int32_t* position, const at_grpo_rows* dq,
                             const at_grpo_rows* dk, float* dq_weight, float* dk_weight, int32_t* data_error,
                             void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * A paged cache and the sequences of a batch in it.  Sequence s has length[s] tokens of its own; token i of them
 * lies in page pages[s][i / page_size] at place i % page_size.  With groups, sequences group_seq[g] ..
 * group_seq[g + 1] - 1 (the candidates of one turn) stand behind the prefix of group g: prefix_len[g] tokens
 * (the prompt), laid out the same way through prefix_pages[g]; any prefix_len will do, a page that the prefix
 * does not fill is not shared with what follows.  A sequence in no group has no prefix.
 * The last cu_q[s + 1] - cu_q[s] own tokens of a sequence are its new ones: rows cu_q[s] .. of the calls' q, k, v.
 * Token i of sequence s stands at position prefix_len + i.
 */
typedef struct {
  int32_t dtype, Hk, D;          /* of the cache; D as above                                             */
  int32_t page_size;             /* a power of two, 8 .. 65536; Hk * page_size * D <= 2^30               */
  int32_t n_pages;               /* > 0                                                                  */
  int32_t n_seq, max_pages;      /* rows and columns of pages                                            */
  int32_t n_group, max_prefix_pages; /* rows and columns of prefix_pages; n_group == 0: no prefixes      */
  void *k, *v;                   /* [n_pages, Hk, page_size, D], 16-byte aligned                         */
  const int32_t* pages;          /* [n_seq, max_pages]; entries behind a sequence's length are not read  */
  const int32_t* length;         /* [n_seq], 0 .. max_pages * page_size                                  */
  const int32_t* cu_q;           /* [n_seq + 1], not falling; NULL: one new token in every sequence      */
  const int32_t* group_seq;      /* [n_group + 1], not falling                                           */
  const int32_t* prefix_len;     /* [n_group], 0 .. max_prefix_pages * page_size                         */
  const int32_t* prefix_pages;   /* [n_group, max_prefix_pages]                                          */
} at_grpo_kv;

/*
 * The new tokens' keys, normed and rotated by their positions as at_grpo_qk_norm_rope does, and their values as
 * they are go into the cache; their queries, normed and rotated, to q_out (Hq == 0: none).  `length` already
 * counts the new tokens.  Rows q [n_tok, Hq, D], k and v [n_tok, kv->Hk, D].  A token that belongs to no sequence,
 * or that the entries of group_seq in front of it and behind it do not enclose, since they fall or leave their
 * range (AT_GRPO_DATA_SEQLENS), whose position lies outside the table (AT_GRPO_DATA_POSITION) or whose page is
 * none of the cache's (AT_GRPO_DATA_PAGE) is left out of the cache, and its q_out rows are zeros.
 */
int at_grpo_kv_append(const at_grpo_kv* kv, const at_grpo_norm_rope* layer, int32_t n_tok, int32_t Hq,
                      const at_grpo_rows* q, const at_grpo_rows* k, const at_grpo_rows* v,
                      const at_grpo_rows* q_out, int32_t* data_error, void* hip_stream);

/*
 * Attention of the new tokens' queries over the cache, Hq a multiple of Hk (query head h reads key head
 * h / (Hq / Hk)):
 *   out[t, h] = sum_i p_i v_i,  p = softmax over the visible tokens i of scale <q[t, h], k_i>
 *   lse[t, h] = ln sum_i exp(scale <q[t, h], k_i>)      (fp32 [n_tok, Hq]; NULL to skip)
 * Visible are the whole prefix of the sequence's group and its own tokens: with causal != 0 up to and with the
 * query's own place (length - new tokens + its number among the new ones), with causal == 0 all of them.  The
 * prefix of a group is read once for all its sequences.  A query that sees nothing gets out 0 and lse -inf.
 * Tokens in a page that is none of the cache's are not seen (AT_GRPO_DATA_PAGE); a length out of range counts as
 * 0, and where cu_q or group_seq fall or leave their range no sequence sees anything (AT_GRPO_DATA_SEQLENS).
 * What a query does not see does not reach its results, infinities and NaN included: what lies in the cache behind
 * a sequence's length, tokens of other sequences, and with causal != 0 those behind the query.
 * out may not share memory with q (AT_GRPO_EINVAL); both may be views of one buffer, of the same strides.
 * Weights are divided by their sum at the end: the values of V times 2^8 times the visible tokens have to stay in fp32's
 * range.
 * max_q (host): an upper bound of the new tokens of one sequence; it picks the kernel, results do not depend on
 * it but for rounding.  scale > 0.  Scores and sums are fp32; bf16 weights are rounded to bf16 for the product
 * with v.  Workspace: at_grpo_prefix_attention_workspace_bytes (0 on invalid arguments; no pointer in kv is read).
 * More than some 6 * 10^7 pairs of a key head with a sequence, group or tile of 16 to 128 rows are
 * AT_GRPO_EUNSUPPORTED.
 */
int at_grpo_prefix_attention(const at_grpo_kv* kv, int32_t n_tok, int32_t Hq, const at_grpo_rows* q, float scale,
                             int32_t causal, int32_t max_q, const at_grpo_rows* out, float* lse,
                             int32_t* data_error, void* workspace, size_t workspace_bytes, void* hip_stream);
size_t at_grpo_prefix_attention_workspace_bytes(const at_grpo_kv* kv, int32_t n_tok, int32_t Hq, int32_t max_q);

/*
 * Bytes of workspace a call needs.  `batch` may be NULL for AT_GRPO_CALL_GROUP_ADVANTAGE; the
 * id extents are ignored for the other calls.  Only sizes are read from `batch` (H, V, n_heads,
 * dtype, n_tok, n_resp); no pointer in it is dereferenced.  With the other sizes as they are, a batch of
 * fewer responses never needs more.  Returns 0 on invalid arguments.
 */
size_t at_grpo_workspace_bytes(int32_t which_call, const at_grpo_batch* batch, int32_t n_resp,
                               int32_t n_env, int32_t n_agent, int32_t n_turn);

/* Static description of a status code. */
const char* at_grpo_status_string(int32_t status);

/* Library version, major * 10000 + minor * 100 + patch. */
int32_t at_grpo_version(void);

/*
 * Optional per-kernel timing with HIP events recorded on the call's stream (a measurement aid,
 * off by default; it keeps process-wide state and is not thread-safe).
 *   at_grpo_profile_enable(1) starts recording, (0) stops and drops what was recorded.
 *   at_grpo_profile_read synchronises the recorded events and returns, for kernel class
 *   `which` (0 .. at_grpo_profile_classes()-1), the number of launches and their total
 *   duration in milliseconds since recording started; the name is a static string.  Small fp32
 *   batches compute both gradients of the head in one launch, which counts as "head_dh", and in the
 *   one-call step their loss beside the backward's preparation, which counts as "token_prep" ("surrogate"
 *   has no launch there).  Calls on queries, keys and the cache count as "rope", attention as "attention".
 */
int at_grpo_profile_enable(int32_t on);
int32_t at_grpo_profile_classes(void);
int at_grpo_profile_read(int32_t which, const char** name, int64_t* launches, double* total_ms);

#ifdef __cplusplus
}
#endif
#endif /* AT_GRPO_H_ */
