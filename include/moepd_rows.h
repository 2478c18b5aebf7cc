/*
 * moepd_rows.h -- token rows into expert order and, weighted, back, with the
 * gradients of both and of the gate: the dispatch's data movement and the
 * combine of moepd.h over buffers that the caller holds, for training and for
 * rows that leave the library between the two.
 *
 * The paper's rollouts train the model that they run (Section 2); dispatch and
 * combine carry a token's row to the experts that the gate picked and back
 * (Section 2.2).  With a layout of moe_dispatch_layout_noalloc (row_of_slot,
 * token_of_row), j over the slots of token t that have a row r(t, j):
 *   rows[r] = x[token_of_row[r]]
 *   out[t] = sum_j w[t,j] y[r(t,j)]
 *   dy[r(t,j)] = w[t,j] dout[t],   dw[t,j] = sum_h dout[t,h] y[r(t,j),h]
 * and dx[t] = sum_j drows[r(t,j)], the gather's gradient, is the combine without
 * weights.  The gate's weights are softmaxes over a token's k picked logits, so
 *   dlogits[t, idx[t,j]] = w[t,j] (dw[t,j] - sum_i w[t,i] dw[t,i]).
 * The loss of a slot whose expert lives on another GPU reaches dw there: dw is
 * summed over the GPUs before moe_gate_backward.
 *
 * Conventions: as in moepd.h (status codes, borrowed device pointers, host
 * validation before anything is enqueued, no allocation, no synchronisation, a
 * non-null stream; the calls may be captured into a graph), on the current
 * device; no state, and deterministic results: sums are float32 and taken in slot
 * order, results in bf16 rounded once.  T in [0, 2^24], k in [1, 16], hidden in
 * [1, 2^20], rows in [0, 2^31 - 512].  Types are MOE_DTYPE_F32 or MOE_DTYPE_BF16.
 * Strides are in elements, at least the row's width, or 0 for exactly that;
 * pointers need their element's alignment.  No buffer that is written may overlap
 * another argument.
 */
#ifndef MOEPD_ROWS_H
#define MOEPD_ROWS_H

#include "moepd.h"

#ifdef __cplusplus
extern "C" {
#endif

/* out[r] = x[token_of_row[r]] in dtype, bit for bit, for r below rows; an index outside [0, T)
 * gives a row of zeros.  row_count: device int32, the rows in use (clamped to [0, rows]; a
 * layout's offsets[E_loc]), past which nothing is written, or NULL for all.
 * Errors: MOE_ERR_INVALID_ARG, MOE_ERR_HIP. */
int moe_rows_gather(const void* x, int32_t dtype, int64_t x_stride, int32_t T, const int32_t* token_of_row,
                    const int32_t* row_count, int64_t rows, int32_t hidden, void* out, int64_t out_stride,
                    hipStream_t stream);

/* out[t] = sum_j w[t,j] y[row_of_slot[t,j]].  A slot whose row is outside [0, rows) adds
 * nothing, whatever its weight holds; a token without rows gets zeros.  w: device [T, k]
 * float, or NULL: 1.  row_of_slot: device [T, k] int32.  Every row of out is written.
 * Errors: MOE_ERR_INVALID_ARG, MOE_ERR_HIP. */
int moe_rows_combine(const void* y, int32_t y_dtype, int64_t y_stride, int64_t rows, const float* w,
                     const int32_t* row_of_slot, int32_t T, int32_t k, int32_t hidden, void* out, int32_t out_dtype,
                     int64_t out_stride, hipStream_t stream);

/* The combine's gradients.  dout: [T, hidden] of dout_dtype.  dy: rows of dy_dtype; those of no
 * slot are not written, and no two slots may name one row.  dw: device [T, k] float, 0 for a
 * slot without a row; or NULL, when y may be NULL too.  w NULL: 1.
 * Errors: MOE_ERR_INVALID_ARG, MOE_ERR_HIP. */
int moe_rows_combine_backward(const void* dout, int32_t dout_dtype, int64_t dout_stride, const void* y, int32_t y_dtype,
                              int64_t y_stride, int64_t rows, const float* w, const int32_t* row_of_slot, int32_t T,
                              int32_t k, int32_t hidden, void* dy, int32_t dy_dtype, int64_t dy_stride, float* dw,
                              hipStream_t stream);

/* The gate's gradient in the logits.  topk_idx: device [T, k] int32 (an index outside [0, E)
 * gets no gradient), topk_w, dw: device [T, k] float; E in [1, 1024], k at most E.  dlogits:
 * [T, E] of dlogits_dtype; with accumulate it is added to (in float32, rounded once: beside
 * moe_balance_loss_backward's), else written, zeros where no slot points.
 * Errors: MOE_ERR_INVALID_ARG, MOE_ERR_HIP. */
int moe_gate_backward(const int32_t* topk_idx, const float* topk_w, const float* dw, int32_t T, int32_t E, int32_t k,
                      void* dlogits, int32_t dlogits_dtype, int64_t dlogits_stride, int32_t accumulate,
                      hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* MOEPD_ROWS_H */
