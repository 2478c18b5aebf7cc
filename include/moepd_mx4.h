/*
 * moepd_mx4.h -- MX FP4 (4-bit) matrices and their products: the operators
 * below the expert layer of moepd.h, for 4-bit weights and activations.
 *
 * The paper runs BF16 and FP8 checkpoints (Section 7.1); 4-bit blocks halve
 * the weight bytes a decode batch streams and double the matrix cores' rate.
 *
 * Format (OCP microscaling, FP4): E2M1 codes (magnitudes 0, 0.5, 1, 1.5, 2, 3,
 * 4, 6; bit 3 is the sign) with one E8M0 scale byte per 32 consecutive values
 * of a row: value = E2M1(code) * 2^(scale - 127).  Quantizing a block takes
 * the exponent X = floor(log2(max |v|)) - 2, clamped to [-127, 127] (-127 for
 * an all-zero block), and the codes v / 2^X rounded to nearest, ties to even,
 * magnitudes above 6 to 6.  A block that holds a NaN or an infinity gets the
 * scale 0xFF, E8M0's NaN: all its values, and every product with it, are NaN.
 *
 * An MX FP4 matrix of `rows` x `cols` is held in the order in which the matrix
 * cores read it, with Kp = cols rounded up to a multiple of 256 (code 0, scale
 * 0 past cols) and Rp = rows rounded up to a multiple of 32:
 *   codes  [Rp / 32][Kp / 32][32 rows][16 bytes], value 2 i of a block of 32 in
 *          the low half of byte i, value 2 i + 1 in the high half;
 *   scales [Rp / 32][Kp / 256][2][32 rows][4 bytes], entry (b, h, r, s) the
 *          scale of row r's block 8 b + 2 s + h.
 * moe_mx4_size gives the bytes of both.  Weight matrices of several groups
 * (experts) are one matrix: group g's rows follow group g - 1's, with no
 * padding between groups.
 *
 * Conventions: as in moepd.h (status codes, borrowed device pointers, host
 * validation before anything is enqueued, no allocation, no synchronisation,
 * a non-null stream; the calls may be captured into a graph).  These calls
 * have no state: any number may run at a time on any streams of the current
 * device, and results are deterministic.  Code and scale buffers are 16-byte aligned; other pointers
 * need their element's alignment.  Strides are in elements, at least the row's
 * width, or 0 for exactly that.
 */
#ifndef MOEPD_MX4_H
#define MOEPD_MX4_H

#include "moepd.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Limits: rows in [0, 2^31 - 32], cols / n / k in [1, 2^20], groups in
 * [1, 1024]. */
#define MOE_MX4_MAX_COLS (1 << 20)
#define MOE_MX4_MAX_GROUPS 1024

/* Bytes of the code and scale buffers of a rows x cols matrix.
 * Errors: MOE_ERR_INVALID_ARG (null output, size out of range). */
int moe_mx4_size(int64_t rows, int32_t cols, int64_t* code_bytes, int64_t* scale_bytes);

/* Quantize rows to an MX FP4 matrix.
 * x: device rows of `cols` values in x_dtype (MOE_DTYPE_F32 or MOE_DTYPE_BF16),
 * x_stride apart.  row_index: device [rows] int32, row r is quantized from
 * x[row_index[r]] (a dispatch's token_of_row gathers tokens into expert order),
 * a negative index gives a row of zeros; or NULL for r itself.  row_count:
 * device int32, the rows in use (clamped to [0, rows]; a dispatch's
 * offsets[E_loc]), or NULL for all; blocks of 32 rows past it are not written,
 * and its last block is filled up with zero rows.
 * Errors: MOE_ERR_INVALID_ARG, MOE_ERR_HIP. */
int moe_mx4_quantize(const void* x, int32_t x_dtype, int64_t x_stride, int64_t rows, int32_t cols,
                     const int32_t* row_index, const int32_t* row_count, uint8_t* codes, uint8_t* scales,
                     hipStream_t stream);

/* The matrix of a checkpoint's row-major codes ([rows, cols / 2] bytes, value
 * 2 i of a row in the low half of byte i) and scales ([rows, cols / 32]), cols
 * a multiple of 32, in the held order.  in_codes is 16-byte aligned.
 * Errors: MOE_ERR_INVALID_ARG, MOE_ERR_HIP. */
int moe_mx4_pack(const uint8_t* in_codes, const uint8_t* in_scales, int64_t rows, int32_t cols, uint8_t* codes,
                 uint8_t* scales, hipStream_t stream);

/* The values of an MX FP4 matrix, rows of `cols` values out_stride apart, in
 * float32 or bf16 (exact in both; a value past bf16's range is infinite).
 * Errors: MOE_ERR_INVALID_ARG, MOE_ERR_HIP. */
int moe_mx4_dequantize(const uint8_t* codes, const uint8_t* scales, int64_t rows, int32_t cols, void* out,
                       int32_t out_dtype, int64_t out_stride, hipStream_t stream);

/* Products with the transposed weights of each row's group:
 *   out[r][c] = sum_k a[r][k] w[g n + c][k], g the group of row r,
 * products and sums in float32, rounded once to out_dtype (MOE_DTYPE_F32 or
 * MOE_DTYPE_BF16).  a: [rows, k]; w: [groups n, k].  offsets: device [groups +
 * 1] int32, group g has the rows [offsets[g], offsets[g + 1]) (ascending;
 * values are clamped to [0, rows]); rows of no group are not written.  NULL
 * with groups = 1: all rows.  Rows of one call are at most `rows`, which also
 * sizes the launch; the tile schedule is read from offsets on the device.
 * k is the width of both matrices (their zero padding is multiplied along).
 * Errors: MOE_ERR_INVALID_ARG (also where the launch would take more than 2^31 -
 * 2^16 workgroups, one for each tile of at least 32 rows and columns), MOE_ERR_HIP. */
int moe_mx4_gemm(const uint8_t* a, const uint8_t* a_scales, int64_t rows, const uint8_t* w, const uint8_t* w_scales,
                 int32_t groups, const int32_t* offsets, int32_t n, int32_t k, void* out, int32_t out_dtype,
                 int64_t out_stride, hipStream_t stream);

/* The gate/up product with SwiGLU: with w [groups 2n, k] (a group's rows [0, n)
 * gate, [n, 2n) up), out[r][c] = silu(gate) * up in float32, then rounded once
 * to out_dtype: MOE_DTYPE_F32, MOE_DTYPE_BF16, or MOE_DTYPE_FP4 (n a multiple
 * of 32): out is the code buffer and out_scales the scale buffer of a rows x n
 * matrix, out_stride 0.  out_scales is NULL for the other types.  Everything
 * else as for moe_mx4_gemm. */
int moe_mx4_gemm_swiglu(const uint8_t* a, const uint8_t* a_scales, int64_t rows, const uint8_t* w,
                        const uint8_t* w_scales, int32_t groups, const int32_t* offsets, int32_t n, int32_t k,
                        void* out, uint8_t* out_scales, int32_t out_dtype, int64_t out_stride, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* MOEPD_MX4_H */
