/*
 * moepd_adamw.h -- an AdamW step over many tensors at once, with states in 32 bits
 * or in 8.
 *
 * The paper's rollouts train the model that they run (Section 2).  For each
 * element, with g = grad * grad_scale and the step's number t:
 *   m = beta1 m + (1 - beta1) g,   v = beta2 v + (1 - beta2) g^2
 *   p = p - lr (m / (1 - beta1^t) / (sqrt(v / (1 - beta2^t)) + eps) + weight_decay p)
 * in float32.  p is the master where there is one, and the parameter its rounding;
 * else the parameter itself (which, in bf16, loses updates below half a step of its own).
 * The root and the quotient hold for every float32 v and eps, those below the normal numbers
 * included.  What v adds up to below 2^-150 is 0 there: with an eps of 0 such an element divides by
 * 0, and one whose m and v are both 0 becomes NaN.
 *
 * States in 8 bits: an expert's weights are most of a model's memory, and 32-bit
 * states take four times that of its bf16 weights.  A block of 32 consecutive values
 * (the last may be shorter) holds one code byte each and one E8M0 scale byte S, a
 * factor of 2^(S - 127):
 *   m: OCP E4M3 codes; the scale puts the block's largest magnitude into [128, 256)
 *   v: codes of its square root, five exponent bits e above three mantissa bits f:
 *      (1 + f / 8) 2^(e - 30), or f / 8 2^-29 where e is 0; the largest into [1, 2)
 * with S clamped to [0, 254], 0 for an all-zero block; a block with a NaN or an
 * infinity gets S = 255 and codes 0, and all its values are NaN.  Codes are rounded at
 * random, up with the probability of the part cut off (to nearest, a v that changes by
 * less than half a code would never change), from 16 bits each: q / step + r / 2^16
 * rounded down, r the upper (m) and lower (v) half of a word that depends on seed, t, the
 * tensor's place in the table and the element's place in the tensor alone:
 *   mix(i ^ key),  key = mix(mix(mix(seed) + t) + tensor) (+ i / 2^32, mixed, past 2^32)
 *   mix(a): a ^= a >> 16, a *= 0x6A09E667, a ^= a >> 15, a *= 0xBB67AE85, a ^= a >> 16.
 * A v above 0 keeps at least the smallest code, so that no m meets a v of 0.
 *
 * Conventions: as in moepd.h (status codes, borrowed device pointers, host
 * validation before anything is enqueued, no synchronisation and no allocation after
 * the create call, a non-null stream; moe_adamw_step and moe_adamw_read may be
 * captured into a graph, which must not be replayed after moe_adamw_destroy).
 * Results are deterministic.
 */
#ifndef MOEPD_ADAMW_H
#define MOEPD_ADAMW_H

#include "moepd.h"

#ifdef __cplusplus
extern "C" {
#endif

/* One tensor of n elements (0 to 2^40).  Pointers need their element's alignment; 16
 * bytes let rows be read in whole vectors. */
typedef struct moe_adamw_tensor {
  void* param;        /* [n] of param_dtype */
  float* master;      /* [n], or NULL */
  const void* grad;   /* [n] of grad_dtype, read only */
  void* m;            /* [n] float, or codes (bytes) */
  void* v;            /* [n] float, or codes (bytes) */
  uint8_t* m_scales;  /* [ceil(n / 32)], or NULL for 32 bits */
  uint8_t* v_scales;  /* the same */
  int64_t n;
  double weight_decay;
  int32_t param_dtype; /* MOE_DTYPE_F32 or MOE_DTYPE_BF16 */
  int32_t grad_dtype;  /* the same */
} moe_adamw_tensor_t;

typedef struct moe_adamw moe_adamw_t;

/* The table of `count` tensors (1 to 65536) on the current device, with states of
 * state_bits (32 or 8).  The buffers are borrowed: they stay where they are for the table's
 * lifetime, and none may overlap another.  Waits for the table's copy; not for use while a
 * stream captures.  Errors:
 * MOE_ERR_INVALID_ARG, MOE_ERR_OOM, MOE_ERR_HIP; *out is then NULL and nothing is left
 * allocated. */
int moe_adamw_create(const moe_adamw_tensor_t* tensors, int32_t count, int32_t state_bits, moe_adamw_t** out);

/* One step over the whole table, one launch.  beta1, beta2 in [0, 1), eps >= 0.  lr: device
 * [1] float; step: device [1] int32, t, counted from 1 (both read by the enqueued work, so
 * a captured step follows them).  grad_scale: device [1] float, or NULL: 1; where it is not
 * finite, nothing is changed (a loss scaler's skipped step).  seed: of the random rounding of
 * 8-bit states.  Steps on one table are ordered by the caller.  The current device has to
 * be the table's.  Errors: MOE_ERR_INVALID_ARG, MOE_ERR_HIP. */
int moe_adamw_step(moe_adamw_t* table, double beta1, double beta2, double eps, const float* lr, const int32_t* step,
                   const float* grad_scale, uint32_t seed, hipStream_t stream);

/* The states of tensor `index` as values: m, and the square root of v, [n] each in
 * MOE_DTYPE_F32 or MOE_DTYPE_BF16 (states of 8 bits are exact in both, a value past bf16's
 * range is infinite or 0); either may be NULL.  Errors: MOE_ERR_INVALID_ARG, MOE_ERR_HIP. */
int moe_adamw_read(moe_adamw_t* table, int32_t index, void* m, void* root_v, int32_t dtype, hipStream_t stream);

/* Waits for the steps and reads enqueued on the table, then frees it; never touches the
 * tensors.  NULL is a no-op. */
int moe_adamw_destroy(moe_adamw_t* table);

#ifdef __cplusplus
}
#endif

#endif /* MOEPD_ADAMW_H */
