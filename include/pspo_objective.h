/*
 * pspo_objective.h -- training objectives through the LM head beside the clipped
 * loss of pspo.h, each with its gradient in one call: the clipped policy loss with
 * a penalty on the divergence from a reference policy, a preference loss on pairs
 * of sequences, and distillation from a teacher's top logits.  Same library and
 * conventions as pspo.h (device pointers owned by the caller, caller's stream, no
 * allocation, no synchronisation, no memset, errors seen by the host returned
 * before anything is enqueued; every call can be captured into a HIP graph).
 *
 * For every row i (hidden row h_i, of N; the head W [V, d])
 *   z_i = W h_i / temperature,  p_i = softmax(z_i),
 * a loss that depends on the rows through some entries of log p_i has the gradient
 *   G_i = d loss / d (W h_i) = a_i p_i, except at those entries,
 *   d_hidden[i] = G_i W,  d_w_head = sum_i G_i^T h_i.
 *
 * Rows left out: a row of weight 0 (any sign) takes no part.  Nothing else of it is
 * read, so that its other values may be anything (NaN, ids out of range); its loss
 * term, d_hidden row and per-token outputs are 0.  A row that has an invalid id
 * raises the error bit, takes no part either and has NaN in its per-token outputs.
 *
 * Precision: logits and softmax sums are float32 sums of exact bf16 products (a logit
 * at an id float32 sums of eight products each, added in float64; its entry joins the
 * sum in float64 from that logit), per-row terms and the loss float64.  A log-prob is
 * never positive, and 1 - p at an id keeps its relative accuracy as p goes to 1.  The
 * softmax entries (with the entries of G at the ids in their places) and, for d_w_head,
 * the hidden rows times their factors are rounded to bf16, the matrix cores' operand
 * type, once each (a row's largest entry at an id is kept exact); sums of the gradient
 * products are float32.  For up to 48 rows of d <= 3584 and up to 64 of d <= 1536
 * d_w_head takes the hidden rows as they are.
 *
 * Memory: the softmax entries of all N rows are kept in the workspace, 2 bytes each
 * (2.5 GB at 8,192 rows of V = 152064), instead of being computed a second time; a call
 * of more than 64 rows without gradients writes and reserves them too.
 *
 * Every result is deterministic: the same arguments give the same bits.  The order of
 * a row's sums follows from N and from its place among the rows.
 * "First N rows": rows behind them are left as they were.  N = 0 is valid (loss 0,
 * d_w_head zeroed unless it is added to).  Outputs and workspaces must not alias
 * inputs or each other.
 */
#ifndef PSPO_OBJECTIVE_H_
#define PSPO_OBJECTIVE_H_

#include "pspo.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Flags of the three calls (PSPO_ACCUMULATE_DW, with float32 d_w_head, adds to it). */
#define PSPO_OBJ_DH_F32   2048u /* d_hidden in float32 instead of bf16 */
#define PSPO_OBJ_DW_F32   4096u /* d_w_head in float32 instead of bf16 */
/* Flag of pspo_preference_fwd_bwd. */
#define PSPO_PREF_AVERAGE 8192u /* a sequence's log ratio is its tokens' weighted mean, not their sum */

/* Estimators of the divergence from the reference at a sampled token, u = log p - log p_ref. */
#define PSPO_KL_K1 1   /* u */
#define PSPO_KL_K2 2   /* u^2 / 2 */
#define PSPO_KL_K3 3   /* exp(-u) - 1 + u */

/* Preference losses of a pair, u = ratio(chosen) - ratio(rejected). */
#define PSPO_PREF_SIGMOID 0   /* -(1 - smoothing) log s(beta u) - smoothing log s(-beta u), s the logistic function */
#define PSPO_PREF_SQUARED 1   /* (u - 1 / (2 beta))^2 */

/*
 * Bytes of device workspace each call below needs for up to N rows (host-only, pure
 * function; 0 for sizes that the calls refuse).  grads: whether a gradient is wanted (a
 * size asked for with them serves calls without them too).
 */
size_t pspo_policy_loss_workspace_bytes(int32_t N, int32_t d, int32_t V, int32_t grads);
size_t pspo_preference_workspace_bytes(int32_t N, int32_t d, int32_t V, int32_t R, int32_t P, int32_t grads);
size_t pspo_distill_workspace_bytes(int32_t N, int32_t d, int32_t V, int32_t k, int32_t grads);

/*
 * Clipped policy loss with a penalty on the divergence from a reference policy: with
 * l_i = log p_i(target_i), rho_i = exp(l_i - logp_old_i), A_i = advantage[seq_id[i]],
 * u_i = l_i - logp_ref_i,
 *   loss = loss_scale * sum_i weight_i (kl_coef kl(u_i) - min(rho_i A_i, clip(rho_i) A_i)),
 * clip to [1 - eps_low, 1 + eps_high]; at rho on the border the gradient passes, as in
 * pspo_loss_fwd_bwd, which computes this loss without the penalty (recomputing logits
 * instead of keeping softmax entries, and with the target entries of G in float32).
 *
 *  hidden     device, bf16 bits [N, d]; w_head: device, bf16 bits [V, d]; d % 8 == 0.
 *  target     device, int32 [N]; logp_old, weight: device, float32 [N]; seq_id: device,
 *             int32 [N] in [0, R); advantage: device, float32 [R].
 *  logp_ref   device, float32 [N], or NULL (then kl_coef must be 0).
 *  kl_kind    PSPO_KL_K1, _K2 or _K3;  temperature > 0;  eps_low, eps_high in [0, 1).
 *  flags      PSPO_OBJ_DH_F32 | PSPO_OBJ_DW_F32 | PSPO_ACCUMULATE_DW or 0.
 *  loss       device, float64 [1] out.
 *  d_hidden   device, [N, d] out, or NULL (not wanted).
 *  d_w_head   device, [V, d] out, or NULL (not wanted: a frozen head).
 *  logp_new   device, float32 [N] out, or NULL.
 *  stats      device, float64 [4] out, or NULL: { loss_scale sum weight s (the clipped
 *             gain), loss_scale sum weight kl (0 without logp_ref), #rows whose gain is
 *             clipped, #rows that take part }.
 *  err_flag   device, int32 [1] or NULL: PSPO_DEVERR_TARGET, PSPO_DEVERR_SEQ_ID,
 *             PSPO_DEVERR_NONFINITE (a value of a row that takes part is not finite).
 *  workspace  device, 256-byte aligned; contents on entry ignored.
 * Sizes: N <= 2^23, V <= 2^21, d <= 2^20, and N d, N V, V d <= 2^36 (PSPO_ERR_UNSUPPORTED
 * beyond).  Device pointers of matrices 16-byte aligned.
 */
int pspo_policy_loss_fwd_bwd(const uint16_t* hidden, const uint16_t* w_head, const int32_t* target,
                             const float* logp_old, const float* logp_ref, const float* weight,
                             const int32_t* seq_id, const float* advantage, int32_t N, int32_t d, int32_t V,
                             int32_t R, float eps_low, float eps_high, float kl_coef, int32_t kl_kind,
                             float temperature, float loss_scale, uint32_t flags, double* loss, void* d_hidden,
                             void* d_w_head, float* logp_new, double* stats, int32_t* err_flag, void* workspace,
                             size_t workspace_bytes, hipStream_t stream);

/*
 * Preference loss on pairs of sequences: with l_i as above,
 *   ratio_r = sum_{i in r} weight_i (l_i - logp_ref_i)
 *             (PSPO_PREF_AVERAGE: divided by sum_{i in r} weight_i, 0 where that is 0),
 *   loss    = loss_scale * sum_q pair_loss(ratio[chosen_q] - ratio[rejected_q]).
 * A sequence may stand in any number of pairs.
 *
 *  cu_seqlens device, int32 [R + 1], non-decreasing: sequence r is rows cu[r] .. cu[r+1] - 1.
 *             Rows outside every sequence get their log-prob and zero gradient, take no part
 *             otherwise and may hold values that are not finite.  Offsets that decrease or lie
 *             outside [0, N] raise PSPO_DEVERR_SEQ_ID and are clamped to [0, N].
 *  chosen, rejected  device, int32 [P] in [0, R); a pair with an index outside raises
 *             PSPO_DEVERR_SEQ_ID and counts nothing (its margin is NaN).
 *  logp_ref   device, float32 [N], or NULL (zeros).
 *  weight     device, float32 [N], or NULL (ones).
 *  kind       PSPO_PREF_SIGMOID or PSPO_PREF_SQUARED; beta > 0; smoothing in [0, 1]
 *             (PSPO_PREF_SIGMOID only).
 *  seq_ratio  device, float32 [R] out, or NULL: ratio_r.
 *  margin     device, float32 [P] out, or NULL: beta (ratio[chosen] - ratio[rejected]).
 *  Other arguments as above; flags also PSPO_PREF_AVERAGE.  P = 0 and R = 0 are valid;
 *  R <= 2^23 and R P <= 2^36 (PSPO_ERR_UNSUPPORTED beyond).  Every sequence looks at
 *  every pair (10^5 of each: some 5 ms).
 */
int pspo_preference_fwd_bwd(const uint16_t* hidden, const uint16_t* w_head, const int32_t* target,
                            const float* logp_ref, const float* weight, const int32_t* cu_seqlens,
                            const int32_t* chosen, const int32_t* rejected, int32_t N, int32_t d, int32_t V,
                            int32_t R, int32_t P, int32_t kind, float beta, float smoothing, float temperature,
                            float loss_scale, uint32_t flags, double* loss, void* d_hidden, void* d_w_head,
                            float* logp_new, float* seq_ratio, float* margin, int32_t* err_flag, void* workspace,
                            size_t workspace_bytes, hipStream_t stream);

/*
 * Distillation from a teacher's top logits: with q_i the softmax of row i's teacher
 * values / temperature over the ids of its list (log-probs serve as well as logits),
 *   loss = loss_scale * sum_i weight_i kl_i,   kl_i = sum_j q_ij (log q_ij - log p_i(id_ij)),
 * p_i over the whole vocabulary.  (A factor temperature^2, where it is wanted, belongs
 * into loss_scale.)
 *
 *  topk_ids   device, int32 [N, k]: ids in [0, V), or negative: no entry.  An id that
 *             stands in a list more than once has the sum of its probabilities.  An id
 *             >= V raises PSPO_DEVERR_TARGET and the row takes no part.
 *  topk_logit device, float32 [N, k]: an entry of -inf is none either; values of
 *             negative ids are not read.  A list without entries leaves its row out.
 *  k          1 .. 64.
 *  weight     device, float32 [N], or NULL (ones).
 *  kl         device, float32 [N] out, or NULL: kl_i.
 *  Other arguments as above.
 */
int pspo_distill_fwd_bwd(const uint16_t* hidden, const uint16_t* w_head, const int32_t* topk_ids,
                         const float* topk_logit, const float* weight, int32_t N, int32_t d, int32_t V, int32_t k,
                         float temperature, float loss_scale, uint32_t flags, double* loss, void* d_hidden,
                         void* d_w_head, float* kl, int32_t* err_flag, void* workspace, size_t workspace_bytes,
                         hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* PSPO_OBJECTIVE_H_ */
