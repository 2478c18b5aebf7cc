/*
 * moepd_balance.h -- the router's load-balance loss, its per-expert counts and
 * its gradient, over the logits and top-k indices of moe_route or
 * moe_route_from_hidden (moe_phase_view: logits, topk_idx) or a caller's own.
 *
 * The paper's rollouts train the model that they run (Section 2); its router
 * picks the top-k experts of each token (Section 7.1).  The loss that keeps
 * such a router's experts evenly used is, for a sequence s with T_s live tokens,
 *   f_se = E / (k T_s) * c_se       c_se: slots of its live tokens at expert e
 *   P_se = 1 / T_s * sum_t p_te     p_t = softmax(logits_t) over the pool
 *   loss = coef / S' * sum_s sum_e f_se P_se
 * over the S' sequences with a live token (0 if there is none; even routing
 * gives coef).  The counts are constants of the gradient:
 *   d loss / d logits_tj = coef / (S' T_s) * p_tj (f_sj - sum_e f_se p_te).
 *
 * A token is live unless its mask byte is 0; a masked token's logits, whatever
 * they hold, and indices are not used, and its gradient is 0.  A logit of minus
 * infinity excludes its expert (probability and gradient 0); a live token whose
 * logits are all minus infinity has probability 0 everywhere.  Other infinities
 * and NaN in a live token's logits give NaN.
 *
 * Conventions: as in moepd.h, on the current device; no state, no allocation, no
 * synchronisation, and deterministic results (no float atomics).  Sums and probabilities are float32.
 */
#ifndef MOEPD_BALANCE_H
#define MOEPD_BALANCE_H

#include "moepd.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Bytes of the workspace of moe_balance_loss (256-byte aligned device memory;
 * its contents need not be set and mean nothing afterwards; calls that overlap
 * need one each).  T in [0, 2^24], E in [1, 1024], S in [1, 65536].
 * Errors: MOE_ERR_INVALID_ARG. */
int moe_balance_workspace(int32_t T, int32_t E, int32_t S, int64_t* bytes);

/* The loss and the counts.
 * logits: device [T, E] of logits_dtype (MOE_DTYPE_F32 or MOE_DTYPE_BF16), rows
 * logits_stride elements apart (0: E).  topk_idx: device [T, k] int32 (an index
 * outside [0, E) counts for no expert; k <= 16).  token_mask: device [T] bytes
 * or NULL (all live).  seq_offsets: device [S + 1] int32, ascending, sequence s
 * has the tokens [seq_offsets[s], seq_offsets[s + 1]), which may be none; tokens
 * before the first and from the last on belong to no sequence; NULL with S = 1:
 * all tokens.
 * loss: device [1] float; counts: device [S, E] int32; live: device [S + 1]
 * int32, each sequence's live tokens, then S'.  All are written, T = 0 included.
 * Errors: MOE_ERR_INVALID_ARG, MOE_ERR_CAPACITY (workspace too small),
 * MOE_ERR_HIP. */
int moe_balance_loss(const void* logits, int32_t logits_dtype, int64_t logits_stride, const int32_t* topk_idx,
                     const uint8_t* token_mask, const int32_t* seq_offsets, int32_t S, int32_t T, int32_t E, int32_t k,
                     float coef, float* loss, int32_t* counts, int32_t* live, void* workspace, int64_t workspace_bytes,
                     hipStream_t stream);

/* The gradient in the logits, from the counts and live tokens of
 * moe_balance_loss on the same arguments.  grad: device [1] float, the gradient
 * of the loss (NULL: 1).  dlogits: device [T, E] of logits_dtype, rows
 * dlogits_stride elements apart (0: E); with accumulate it is added to (in
 * float32, rounded once), else written, zeros where there is no gradient.
 * dlogits may be logits itself when not accumulating, with the same stride.
 * Errors: MOE_ERR_INVALID_ARG, MOE_ERR_HIP. */
int moe_balance_loss_backward(const void* logits, int32_t logits_dtype, int64_t logits_stride,
                              const uint8_t* token_mask, const int32_t* seq_offsets, int32_t S, int32_t T, int32_t E,
                              int32_t k, float coef, const int32_t* counts, const int32_t* live, const float* grad,
                              void* dlogits, int64_t dlogits_stride, int32_t accumulate, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* MOEPD_BALANCE_H */
