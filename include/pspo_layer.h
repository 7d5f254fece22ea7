/*
 * pspo_layer.h -- the token-wise operators of a policy's transformer layers on
 * packed prefix tokens, in the same library and under the same conventions as
 * pspo.h (device pointers owned by the caller, caller's stream, no allocation,
 * no synchronisation, no memset, errors seen by the host returned before
 * anything is enqueued; every call can be captured into a HIP graph).
 *
 * Algorithm 1 runs the policy's layers "only for t <= H": on the rows that
 * pspo_pack_prefixes lays out.  The calls read that layout's own arrays: the
 * rotation takes positions from seq_id and cu_seqlens, the dropout takes its
 * counter from src_row, so that a kept token's mask is the same whichever
 * cutoffs were drawn, and the same in the passes under the old and the new
 * policy that the importance ratio compares.
 *
 * "First N rows": every call reads and writes rows 0 .. N-1 of its per-token
 * tensors and leaves the rows behind them as they were.  N = 0 is valid; the
 * gradients of weights are then zero.  Outputs and workspaces must not alias
 * inputs or each other.
 *
 * Every result is deterministic: the same arguments give the same bits.  A
 * token's head norms and dropout do not depend on the other tokens of the call;
 * its feed-forward block does in rounding (see pspo_gated_ffn_fwd).
 */
#ifndef PSPO_LAYER_H_
#define PSPO_LAYER_H_

#include "pspo.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types of the calls that take one. */
#define PSPO_TYPE_BF16 0
#define PSPO_TYPE_F32  1

/* Flags of pspo_qk_norm_rope_*. */
#define PSPO_ROPE_INTERLEAVED 1u /* pairs (2 i, 2 i + 1); default: pairs (i, i + rot_dim / 2) */
#define PSPO_QK_NO_NORM       2u /* rotation only: no norm, and the weights must be NULL */

/*
 * Norms of queries and keys for each head with the position rotation, in one
 * pass.  For a head x of D = head_dim entries of token n:
 *   z   = w * x / sqrt(mean(x^2) + eps)
 *   out = z with its first rot_dim entries turned pair by pair by the angles
 *         pos_n * inv_freq[i], i < rot_dim / 2:
 *         (a, b) -> (a cos - b sin, a sin + b cos).
 * The angle is formed in float64 (positions of any size), everything else in
 * float32, with one rounding to the output's type.  (A head whose sum of
 * squares passes float32, entries of 1e18 and more, is normed to zeros.)
 *
 *  q, k          device [N rows]: token n's heads at q + n * q_stride, heads
 *                contiguous ([heads, D]); strides in elements, >= heads * D, so q
 *                and k may be parts of a fused projection's rows.  16-byte
 *                aligned rows.  heads_k = 0 (k NULL) is valid, heads_q >= 1.
 *  q_weight,     device [D] of the same type, 16-byte aligned, or NULL (all ones).
 *  k_weight
 *  inv_freq      device, float32 [rot_dim / 2] (NULL iff rot_dim = 0).
 *  positions     device, int32 [N], or NULL: then
 *                pos_n = first_pos[r] + n - cu_seqlens[r], r = seq_id[n].
 *  seq_id, cu_seqlens, first_pos   device, int32 [N], [R+1], [R]; first_pos may
 *                be NULL (zeros).  Not read when positions is given or rot_dim = 0.
 *                A seq_id outside [0, R) raises PSPO_DEVERR_SEQ_ID and is turned
 *                by position 0.
 *  head_dim      a multiple of 8, at most 512; rot_dim a multiple of 16, <= head_dim.
 *  q_out, k_out  device, [N, heads, D] contiguous, of the same type.
 *  err_flag      device, int32 [1] or NULL.
 */
int pspo_qk_norm_rope_fwd(const void* q, const void* k, int64_t q_stride, int64_t k_stride,
                          const void* q_weight, const void* k_weight, const float* inv_freq,
                          const int32_t* positions, const int32_t* seq_id, const int32_t* cu_seqlens,
                          const int32_t* first_pos, int32_t N, int32_t R, int32_t heads_q, int32_t heads_k,
                          int32_t head_dim, int32_t rot_dim, float eps, int32_t type, uint32_t flags,
                          void* q_out, void* k_out, int32_t* err_flag, hipStream_t stream);

/* Bytes of device workspace pspo_qk_norm_rope_bwd needs for N tokens (host-only), enough for fewer too;
 * 0 for sizes it refuses. */
size_t pspo_qk_norm_rope_workspace_bytes(int32_t N, int32_t head_dim);

/*
 * Its gradient, from the inputs (nothing of the forward is kept): with
 * dz = out's gradient turned back and xhat = x / sqrt(mean(x^2) + eps),
 *   dw = sum over tokens and heads of dz xhat,
 *   dx = (dz w - xhat mean(dz w xhat)) / sqrt(mean(x^2) + eps).
 *  dq_out, dk_out  device, [N, heads, D] contiguous, of the same type.
 *  dq, dk          device, [N, heads, D] contiguous, of the same type, out.
 *  dq_weight,      device, float32 [D] out, or NULL (not wanted; must be NULL
 *  dk_weight       where the weight is).  Sums in a fixed order, no atomics.
 */
int pspo_qk_norm_rope_bwd(const void* dq_out, const void* dk_out, const void* q, const void* k,
                          int64_t q_stride, int64_t k_stride, const void* q_weight, const void* k_weight,
                          const float* inv_freq, const int32_t* positions, const int32_t* seq_id,
                          const int32_t* cu_seqlens, const int32_t* first_pos, int32_t N, int32_t R,
                          int32_t heads_q, int32_t heads_k, int32_t head_dim, int32_t rot_dim, float eps,
                          int32_t type, uint32_t flags, void* dq, void* dk, float* dq_weight,
                          float* dk_weight, int32_t* err_flag, void* workspace, size_t workspace_bytes,
                          hipStream_t stream);

/*
 * Dropout with the residual sum; the mask is drawn again wherever it is needed
 * and never stored:
 *   y[n][c] = residual[n][c] + (kept(n, c) ? x[n][c] * 2^16 / T : 0),
 *   T = clamp(floor((1 - p) 2^16 + 1/2), 1, 2^16),   kept iff word < T,
 * word = 16 bits of Philox4x32-10(counter = (row, 1 + c / 8, lo32(offset),
 * hi32(offset)), key = (lo32(seed), hi32(seed))): of output word (c % 8) / 2 the
 * low half for even c, the high half for odd c; row = row_ids[n] (taken as 32
 * unsigned bits) or n.  An entry is kept with probability T / 2^16 exactly and
 * scaled by its inverse (rounded to float32), so the mean is unbiased.
 * pspo_sample_cutoffs draws from counters with 0 in the second place, so one
 * seed and offset may serve both.
 *
 *  x, residual  device, [N, d] of `type`, 16-byte aligned, d % 8 == 0;
 *               residual may be NULL (zeros).
 *  row_ids      device, int32 [N] or NULL: e.g. the packer's src_row.
 *  p            in [0, 1).
 *  y            device, [N, d] of `type` out.
 */
int pspo_dropout_add_fwd(const void* x, const void* residual, const int32_t* row_ids, int32_t N, int32_t d,
                         double p, uint64_t seed, uint64_t offset, int32_t type, void* y, hipStream_t stream);

/*
 * Its gradient: dx[n][c] = kept(n, c) ? dy[n][c] * 2^16 / T : 0 (the residual's
 * gradient is dy itself).  dy of type dy_type, dx of type dx_type.
 */
int pspo_dropout_bwd(const void* dy, const int32_t* row_ids, int32_t N, int32_t d, double p, uint64_t seed,
                     uint64_t offset, int32_t dy_type, int32_t dx_type, void* dx, hipStream_t stream);

/* Activations of pspo_gated_ffn_*. */
#define PSPO_ACT_SILU      0   /* g / (1 + exp(-g)) */
#define PSPO_ACT_GELU_TANH 1   /* g (1 + tanh(sqrt(2/pi) (g + 0.044715 g^3))) / 2 */

/* Flags of pspo_gated_ffn_bwd (PSPO_ACCUMULATE_DW, with float32 weight gradients, adds to them). */
#define PSPO_FFN_DW_F32   256u /* weight gradients in float32 instead of bf16 */
/* Flags of pspo_gated_ffn_workspace_bytes. */
#define PSPO_FFN_BACKWARD 512u /* the backward call's workspace instead of the forward's */
#define PSPO_FFN_PREACT  1024u /* ... with the forward's pre-activations given */

/* Bytes of device workspace the calls below need for N tokens (host-only); 0 for sizes they refuse.
 * The size for N tokens serves every call of fewer (same d, f and flags).  Up to 256 MB of it hold
 * the sums of products that are split along K. */
size_t pspo_gated_ffn_workspace_bytes(int32_t N, int32_t d, int32_t f, uint32_t flags);

/*
 * The gated feed-forward block: for every token x (a row of d entries)
 *   g = Wg x,  u = Wu x,  h = act(g) * u,  y = Wd h.
 * Sums in float32; h is rounded to bf16 (the operand of the last product), y once.
 * The order of a token's sums follows from N and from its place among the rows (tiles, K
 * parts), so y of the same token may differ in rounding between calls of different N: passes
 * whose ratio is taken should run on the same rows.
 *
 *  x             device, bf16 bits [N, d] row-major, 16-byte aligned.
 *  w_gate, w_up  device, bf16 bits [f, d] row-major.
 *  w_down        device, bf16 bits [d, f] row-major.
 *  d, f          multiples of 8, at most 2^20.
 *  y             device, bf16 bits [N, d] out.
 *  preact        device, float32 [N, 2 f] out (g, then u, of each token), or NULL: what
 *                the backward needs besides its inputs.
 *  workspace     device, 256-byte aligned, its contents need not be kept.
 */
int pspo_gated_ffn_fwd(const uint16_t* x, const uint16_t* w_gate, const uint16_t* w_up, const uint16_t* w_down,
                       int32_t N, int32_t d, int32_t f, int32_t act, uint16_t* y, float* preact,
                       void* workspace, size_t workspace_bytes, hipStream_t stream);

/*
 * Its gradient: with dh = Wd^T dy,
 *   dg = dh * u * act'(g),  du = dh * act(g)   (rounded to bf16),
 *   dx = Wg^T dg + Wu^T du,  dWg = sum dg x^T,  dWu = sum du x^T,  dWd = sum dy h^T.
 *  dy            device, bf16 bits [N, d].
 *  preact        what the forward wrote, or NULL: computed again (in the workspace).
 *  dx            device, bf16 bits [N, d] out.
 *  dw_gate, dw_up, dw_down   device, of the weights' shapes, out: bf16, or float32
 *                with PSPO_FFN_DW_F32; N = 0 writes (or adds) zeros and takes workspace NULL.
 */
int pspo_gated_ffn_bwd(const uint16_t* dy, const uint16_t* x, const uint16_t* w_gate, const uint16_t* w_up,
                       const uint16_t* w_down, const float* preact, int32_t N, int32_t d, int32_t f,
                       int32_t act, uint32_t flags, uint16_t* dx, void* dw_gate, void* dw_up, void* dw_down,
                       void* workspace, size_t workspace_bytes, hipStream_t stream);

#ifdef __cplusplus
}  /* extern "C" */
#endif

#endif  /* PSPO_LAYER_H_ */
