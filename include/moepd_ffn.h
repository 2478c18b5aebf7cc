/*
 * moepd_ffn.h -- the gated feed-forward block of an expert layer with its
 * backward pass, over rows that the caller holds: what moe_expert_ffn (moepd.h)
 * computes inside a context, for training and for experts outside one.
 *
 * The paper's rollouts train the model that they run (Section 2); its experts
 * are gated blocks between dispatch and combine (Section 2.2).  For the rows of
 * group (expert) e, with W1, W3 the rows [0, I), [I, 2I) of w_gate_up's matrix e and
 * W2 w_down's:
 *   g = x W1^T,  u = x W3^T,  h = silu(g) * u,  y = h W2^T,  s = 1 / (1 + e^-g)
 *   dh = dy W2,  dg = dh * u * s * (1 + g (1 - s)),  du = dh * g * s
 *   dx = dg W1 + du W3,  dW1 = dg^T x,  dW3 = du^T x,  dW2 = dy^T h.
 * One call runs both projections, the activation and the product; one runs dh
 * and everything that follows from it element by element; g, u, dh never pass
 * through memory in between.
 *
 * Rows of a matrix lie side by side; gate_up and dgate_up are [rows, 2I], gate
 * (dg) in the columns [0, I) and up (du) in [I, 2I).  Products and sums are
 * float32.  Results in bf16 are rounded once, to nearest even; h and dgate_up, the
 * operands of the products that follow, are such results.  A gate of
 * minus infinity takes the limits (h, dg and du are 0 where u and dh are finite), one of
 * plus infinity too (s is 1, dg = dh u).
 *
 * Arguments that the calls share:
 *   rows     [0, 2^31 - 512]; sizes the launch, and picks the tiles as for groups of
 *            rows / groups rows (a weight gradient's parts too): room far above the rows
 *            in use costs the speed of tiles for longer groups, and sums in their order
 *   groups   [1, 1024], and offsets: device [groups + 1] int32, ascending; group
 *            g has the rows [offsets[g], offsets[g + 1]) (values are clamped to [0,
 *            rows]; a dispatch's offsets), which may be none.  Rows of no group
 *            are not written.  NULL with groups = 1: all rows.
 *   hidden   H, inter I: multiples of 8 in [8, 32768], H I at most 2^28
 *   dtype    MOE_DTYPE_BF16 or MOE_DTYPE_F32: of x, h, dy, gate_up, dgate_up and
 *            the weights.  Results with a type of their own are MOE_DTYPE_F32, or
 *            MOE_DTYPE_BF16 where dtype is.
 * Strides are in elements, multiples of 8, at least the row's width and at most
 * 2^20, or 0 for exactly that; pointers are 16-byte aligned.  w_gate_up: [groups,
 * 2I, H], w_down: [groups, H, I].  No buffer that is written may overlap another
 * argument.  A launch of more than 2^31 - 2^16 workgroups (one for each tile of at
 * least 32 rows and 32 columns) is refused with MOE_ERR_INVALID_ARG.
 *
 * Conventions: as in moepd.h (status codes, borrowed device pointers, host
 * validation before anything is enqueued, no allocation, no synchronisation, a
 * non-null stream; the calls may be captured into a graph), on the current
 * device.  The calls have no state; results are deterministic.
 */
#ifndef MOEPD_FFN_H
#define MOEPD_FFN_H

#include "moepd.h"

#ifdef __cplusplus
extern "C" {
#endif

/* h = silu(g) * u, from the unrounded g and u.  x: [rows, H], x_stride apart.
 * gate_up: g and u for the backward pass, or NULL where none follows.
 * Errors: MOE_ERR_INVALID_ARG, MOE_ERR_HIP. */
int moe_ffn_gate_up(const void* x, int64_t x_stride, int64_t rows, const void* w_gate_up, int32_t groups,
                    const int32_t* offsets, int32_t hidden, int32_t inter, int32_t dtype, void* gate_up, void* h,
                    hipStream_t stream);

/* y = h W2^T, rows of y_dtype y_stride apart.
 * Errors: MOE_ERR_INVALID_ARG, MOE_ERR_HIP. */
int moe_ffn_down(const void* h, int64_t rows, const void* w_down, int32_t groups, const int32_t* offsets, int32_t hidden,
                 int32_t inter, int32_t dtype, void* y, int32_t y_dtype, int64_t y_stride, hipStream_t stream);

/* dgate_up from dy ([rows, H], dy_stride apart) and the kept gate_up; and, unless
 * NULL, h anew from the kept gate_up, for programs that keep gate_up alone.
 * Errors: MOE_ERR_INVALID_ARG, MOE_ERR_HIP. */
int moe_ffn_down_backward(const void* dy, int64_t dy_stride, int64_t rows, const void* w_down, const void* gate_up,
                          int32_t groups, const int32_t* offsets, int32_t hidden, int32_t inter, int32_t dtype,
                          void* dgate_up, void* h, hipStream_t stream);

/* dx = dgate_up [W1; W3], rows of dx_dtype dx_stride apart.
 * Errors: MOE_ERR_INVALID_ARG, MOE_ERR_HIP. */
int moe_ffn_gate_up_backward(const void* dgate_up, int64_t rows, const void* w_gate_up, int32_t groups,
                             const int32_t* offsets, int32_t hidden, int32_t inter, int32_t dtype, void* dx,
                             int32_t dx_dtype, int64_t dx_stride, hipStream_t stream);

/* Bytes of the workspace of moe_ffn_weight_grad for these sizes: at most 2^27, often 0.
 * Errors: MOE_ERR_INVALID_ARG. */
int moe_ffn_weight_workspace(int64_t rows, int32_t groups, int32_t m, int32_t n, int64_t* bytes);

/* The gradient of a group's weights, dw[g] = sum over its rows r of a[r]^T b[r]: with a
 * = dgate_up (m = 2I), b = x (n = H) of w_gate_up; with a = dy (m = H), b = h (n =
 * I) of w_down.  a: [rows, m], b: [rows, n], of dtype, their strides apart; m, n:
 * multiples of 8 in [8, 65536], m n at most 2^29.  dw: [groups, m, n] of dw_dtype; with
 * accumulate it is added to (in float32, rounded once), else written, zeros for a
 * group without rows.  workspace: 256-byte aligned device memory of at least
 * moe_ffn_weight_workspace's bytes (NULL where that is 0), whose contents need
 * not be set and mean nothing afterwards; calls that overlap need one each.
 * Errors: MOE_ERR_INVALID_ARG, MOE_ERR_CAPACITY (workspace too small), MOE_ERR_HIP. */
int moe_ffn_weight_grad(const void* a, int64_t a_stride, const void* b, int64_t b_stride, int64_t rows, int32_t groups,
                        const int32_t* offsets, int32_t m, int32_t n, int32_t dtype, void* dw, int32_t dw_dtype,
                        int32_t accumulate, void* workspace, int64_t workspace_bytes, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* MOEPD_FFN_H */
