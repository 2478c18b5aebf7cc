// MX FP4 blocks on gfx950: the held order of a matrix, block exponents, and
// conversions (see include/moepd_mx4.h for the format).
//
// Why this order.  v_mfma_scale_f32_32x32x64_f8f6f4 with FP4 operands takes,
// in lane l, the 32 values K [32 h, 32 h + 32) of row l % 32 (h = l / 32): 16
// bytes.  A block of 32 rows therefore holds, for each block of 32 values along
// K, 32 rows x 16 bytes = 512 contiguous bytes, and one operand of one MFMA is
// 1 KB of consecutive memory, read by one 16-byte load per lane, straight
// into registers or, by DMA, into LDS where the lanes read it back with no bank
// conflict and no swizzle.  The scales of 256 values go together: lane l's four
// bytes are those of the four MFMAs, whose byte select picks them, so one
// 4-byte load per lane serves four MFMAs with no shifting.  Rows of a
// product's tile need not start at a multiple of 32: a lane's row only sets its
// base address.
#pragma once

#include "common.h"
#include "mx4_form.h"

namespace moepd {

__host__ __device__ inline int mx4_slices(int cols) { return (cols + kMx4Slice - 1) / kMx4Slice; }

// Scale byte of a block from the bits of its largest magnitude (as a
// float32): floor(log2 amax) - 2 + 127, at least 0; 255 for NaN and infinity.
__device__ __forceinline__ uint32_t mx4_scale_byte(uint32_t amax_bits) {
  const uint32_t ef = amax_bits >> 23;
  return ef >= 255u ? 255u : ef < 2u ? 0u : ef - 2u;
}

// 2^(byte - 127) as a float: 2^-127 is subnormal, 255 gives NaN.
__device__ __forceinline__ float mx4_scale(uint32_t byte) {
  return __uint_as_float(byte == 0u ? 0x00400000u : byte == 255u ? 0x7fc00000u : byte << 23);
}

// Eight values to eight codes under a block's scale (value i in bits 4i; RNE,
// magnitudes above 6 to 6).  NaN blocks hold zero codes.
__device__ __forceinline__ uint32_t mx4_codes8(const float (&v)[8], uint32_t byte) {
  const float s = mx4_scale(byte);
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[0], v[1], s, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2], v[3], s, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[4], v[5], s, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[6], v[7], s, 3);
  return byte == 255u ? 0u : w;
}

}  // namespace moepd
