// MX FP4 matrices: quantizing rows, packing a checkpoint's codes, and the
// values back (include/moepd_mx4.h).  All three move memory once, which is what
// bounds them, and for few rows the launch and three dependent loads (4 us for 64 rows
// of 7168).  A workgroup handles 32 rows x 256 values, the unit that is contiguous in
// the held order.
#include "kernels.h"
#include "moepd_mx4.h"
#include "mx4.h"

namespace moepd {

namespace {

constexpr int kUnitWords = 8 * 132;  // LDS words of a unit: a 32-value block of 32 rows, 128 words and 4 of padding

// Units of a launch are walked with a grid stride, by two rounds of what the GPU holds
// (2048 workgroups): a launch sized by a batch's capacity, of which a GPU's share may be an
// eighth, then ends with its rows (65,536 rows of 7168, 8192 in use: 25 us, one
// workgroup for each unit 55; all of 8243 in use 24 and 26).
inline unsigned unit_grid(long long units) { return (unsigned)(units < 4096 ? units : 4096); }

// Quantize.  A row's 256 values are read by half a wave, 8 consecutive values
// to a lane, so four lanes share a block and find its maximum with two quad
// permutations; the unit's codes cross LDS to leave as 4 KB of consecutive memory.
// 8243 rows of 7168 bf16 values gathered from 8192 24 us (6.2 TB/s of rows in and codes
// out, some of the rows from the memory-side cache), 12,289 x 2559 float32 25 us (5.7).
template <bool BF16>
__global__ __launch_bounds__(256) void mx4_quantize_kernel(const void* __restrict__ x, long long x_stride,
                                                           long long rows, int cols, int slices, long long units,
                                                           const int32_t* __restrict__ row_index,
                                                           const int32_t* __restrict__ row_count,
                                                           uint8_t* __restrict__ codes, uint8_t* __restrict__ scales) {
  __shared__ uint32_t words[kUnitWords];
  __shared__ uint8_t bytes[kMx4SliceScales];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int c8 = lane & 31;
  for (long long unit = blockIdx.x; unit < units; unit += gridDim.x) {
    const long long rb = unit / slices;
    const int kt = (int)(unit - rb * slices);
    // the row count and the indices are read together
    int index[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const long long row = rb * kMx4Rows + 8 * wave + 2 * i + (lane >> 5);
      index[i] = row_index && row < rows ? row_index[row] : -1;
    }
    const long long count = row_count ? *row_count : rows, used = count < rows ? count : rows;
    if (rb * kMx4Rows >= used) break;  // units ascend, so the whole workgroup is done
    const int col = kt * kMx4Slice + c8 * 8;
    float v[4][8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const long long row = rb * kMx4Rows + 8 * wave + 2 * i + (lane >> 5);
      const long long src = row >= used ? -1 : row_index ? index[i] : row;
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] = 0.f;
      if (src >= 0) {
        const long long at = src * x_stride + col;
        if (col + 8 <= cols) {
          if constexpr (BF16) {
            const u32x4 u = *reinterpret_cast<const u32x4_any*>(static_cast<const uint16_t*>(x) + at);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              v[i][2 * j] = __uint_as_float(u[j] << 16);
              v[i][2 * j + 1] = __uint_as_float(u[j] & 0xffff0000u);
            }
          } else {
            const u32x4 a = *reinterpret_cast<const u32x4_any*>(static_cast<const float*>(x) + at);
            const u32x4 b = *reinterpret_cast<const u32x4_any*>(static_cast<const float*>(x) + at + 4);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              v[i][j] = __uint_as_float(a[j]);
              v[i][4 + j] = __uint_as_float(b[j]);
            }
          }
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (col + j < cols) {
              if constexpr (BF16) v[i][j] = bf16_to_f32(static_cast<const uint16_t*>(x)[at + j]);
              else v[i][j] = static_cast<const float*>(x)[at + j];
            }
        }
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      // magnitudes as bits order like the floats, infinity and NaN above all
      uint32_t m = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const uint32_t b = __float_as_uint(v[i][j]) & 0x7fffffffu;
        m = b > m ? b : m;
      }
      m = dpp_step<true, 0xB1, 0xF>(m);  // quad_perm [1,0,3,2]
      m = dpp_step<true, 0x4E, 0xF>(m);  // quad_perm [2,3,0,1]
      const uint32_t byte = mx4_scale_byte(m);
      const int r = 8 * wave + 2 * i + (lane >> 5), c = c8 >> 2;
      words[c * 132 + r * 4 + (c8 & 3)] = mx4_codes8(v[i], byte);
      if ((c8 & 3) == 0) bytes[((c & 1) * 32 + r) * 4 + (c >> 1)] = (uint8_t)byte;
    }
    __syncthreads();
    const int t = threadIdx.x;
    store16(codes + unit * kMx4SliceBytes + t * 16, *reinterpret_cast<const u32x4*>(&words[(t >> 5) * 132 + (t & 31) * 4]));
    if (t < 64)
      reinterpret_cast<uint32_t*>(scales + unit * kMx4SliceScales)[t] = reinterpret_cast<const uint32_t*>(bytes)[t];
    __syncthreads();
  }
}

// A checkpoint's row-major codes and scales: thread t moves block t / 32 of row
// t % 32.
__global__ __launch_bounds__(256) void mx4_pack_kernel(const uint8_t* __restrict__ in_codes,
                                                       const uint8_t* __restrict__ in_scales, long long rows,
                                                       int blocks, int slices, long long units,
                                                       uint8_t* __restrict__ codes, uint8_t* __restrict__ scales) {
  const int t = threadIdx.x, c = t >> 5, r = t & 31;
  for (long long unit = blockIdx.x; unit < units; unit += gridDim.x) {
    const long long rb = unit / slices;
    const int kt = (int)(unit - rb * slices);
    const long long row = rb * kMx4Rows + r;
    const bool in = row < rows && kt * 8 + c < blocks;
    u32x4 q = {0u, 0u, 0u, 0u};
    uint8_t s = 0;
    if (in) {
      q = load16(in_codes + (row * blocks + kt * 8 + c) * 16);
      s = in_scales[row * blocks + kt * 8 + c];
    }
    store16(codes + unit * kMx4SliceBytes + t * 16, q);
    scales[unit * kMx4SliceScales + ((c & 1) * 32 + r) * 4 + (c >> 1)] = s;
  }
}

// The values: the unit's codes cross LDS so that half a wave writes a row's 256
// values together (past the caches' keeping).  8243 x 7168 to bf16 35 us (4.2 TB/s).
template <bool BF16>
__global__ __launch_bounds__(256) void mx4_dequantize_kernel(const uint8_t* __restrict__ codes,
                                                             const uint8_t* __restrict__ scales, long long rows,
                                                             int cols, int slices, long long units,
                                                             void* __restrict__ out, long long out_stride) {
  __shared__ uint32_t words[kUnitWords];
  __shared__ uint32_t bytes[kMx4SliceScales / 4];
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6, c8 = lane & 31;
  for (long long unit = blockIdx.x; unit < units; unit += gridDim.x) {
    const long long rb = unit / slices;
    const int kt = (int)(unit - rb * slices);
    *reinterpret_cast<u32x4*>(&words[(t >> 5) * 132 + (t & 31) * 4]) = load16(codes + unit * kMx4SliceBytes + t * 16);
    if (t < 64) bytes[t] = reinterpret_cast<const uint32_t*>(scales + unit * kMx4SliceScales)[t];
    __syncthreads();
    const int col = kt * kMx4Slice + c8 * 8, c = c8 >> 2;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = 8 * wave + 2 * i + (lane >> 5);
      const long long row = rb * kMx4Rows + r;
      if (row >= rows || col >= cols) continue;
      const uint32_t w = words[c * 132 + r * 4 + (c8 & 3)];
      const float s = mx4_scale((bytes[(c & 1) * 32 + r] >> (8 * (c >> 1))) & 255u);
      float v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        // E2M1 magnitude m: 0, 0.5, then (2 + (m & 1)) 2^(m / 2 - 2)
        const uint32_t m = (w >> (4 * j)) & 7u;
        const float mag = m < 2u ? 0.5f * (float)m : __uint_as_float((((m >> 1) + 126u) << 23) | ((m & 1u) << 22));
        v[j] = ((w >> (4 * j)) & 8u ? -mag : mag) * s;
      }
      const long long at = row * out_stride + col;
      if (col + 8 <= cols) {
        if constexpr (BF16) {
          u32x4_any q;
#pragma unroll
          for (int j = 0; j < 4; ++j)
            q[j] = (uint32_t)f32_to_bf16(v[2 * j]) | ((uint32_t)f32_to_bf16(v[2 * j + 1]) << 16);
          __builtin_nontemporal_store(q, reinterpret_cast<u32x4_any*>(static_cast<uint16_t*>(out) + at));
        } else {
          u32x4_any a, b;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            a[j] = __float_as_uint(v[j]);
            b[j] = __float_as_uint(v[4 + j]);
          }
          __builtin_nontemporal_store(a, reinterpret_cast<u32x4_any*>(static_cast<float*>(out) + at));
          __builtin_nontemporal_store(b, reinterpret_cast<u32x4_any*>(static_cast<float*>(out) + at + 4));
        }
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (col + j < cols) {
            if constexpr (BF16) static_cast<uint16_t*>(out)[at + j] = f32_to_bf16(v[j]);
            else static_cast<float*>(out)[at + j] = v[j];
          }
      }
    }
    __syncthreads();
  }
}

inline bool aligned(const void* p, size_t a) { return (uintptr_t)p % a == 0; }

}  // namespace

hipError_t launch_mx4_quantize(const void* x, bool bf16, long long x_stride, long long rows, int cols,
                               const int32_t* row_index, const int32_t* row_count, uint8_t* codes, uint8_t* scales,
                               hipStream_t s) {
  if (rows <= 0) return hipSuccess;
  const int slices = mx4_slices(cols);
  const long long units = (rows + kMx4Rows - 1) / kMx4Rows * slices;
  auto go = [&](auto k) {
    k<<<dim3(unit_grid(units)), 256, 0, s>>>(x, x_stride, rows, cols, slices, units, row_index, row_count, codes, scales);
  };
  bf16 ? go(mx4_quantize_kernel<true>) : go(mx4_quantize_kernel<false>);
  return hipGetLastError();
}

long long mx4_code_bytes(long long rows, int cols) {
  return (rows + kMx4Rows - 1) / kMx4Rows * mx4_slices(cols) * kMx4SliceBytes;
}
long long mx4_scale_bytes(long long rows, int cols) {
  return (rows + kMx4Rows - 1) / kMx4Rows * mx4_slices(cols) * kMx4SliceScales;
}

}  // namespace moepd

using namespace moepd;

namespace {

constexpr int64_t kMaxRows = (1LL << 31) - 32;

bool valid_size(int64_t rows, int32_t cols) {
  return rows >= 0 && rows <= kMaxRows && cols >= 1 && cols <= MOE_MX4_MAX_COLS;
}

}  // namespace

extern "C" {

int moe_mx4_size(int64_t rows, int32_t cols, int64_t* code_bytes, int64_t* scale_bytes) {
  if (!code_bytes || !scale_bytes || !valid_size(rows, cols)) return MOE_ERR_INVALID_ARG;
  *code_bytes = mx4_code_bytes(rows, cols);
  *scale_bytes = mx4_scale_bytes(rows, cols);
  return MOE_OK;
}

int moe_mx4_quantize(const void* x, int32_t x_dtype, int64_t x_stride, int64_t rows, int32_t cols,
                     const int32_t* row_index, const int32_t* row_count, uint8_t* codes, uint8_t* scales,
                     hipStream_t stream) {
  if (!stream || !valid_size(rows, cols)) return MOE_ERR_INVALID_ARG;
  if (x_dtype != MOE_DTYPE_F32 && x_dtype != MOE_DTYPE_BF16) return MOE_ERR_INVALID_ARG;
  if (x_stride == 0) x_stride = cols;
  if (x_stride < cols) return MOE_ERR_INVALID_ARG;
  if (rows == 0) return MOE_OK;
  if (!x || !codes || !scales || !aligned(codes, 16) || !aligned(scales, 16) ||
      !aligned(x, x_dtype == MOE_DTYPE_F32 ? 4 : 2) || !aligned(row_index, 4) || !aligned(row_count, 4))
    return MOE_ERR_INVALID_ARG;
  return launch_mx4_quantize(x, x_dtype == MOE_DTYPE_BF16, x_stride, rows, cols, row_index, row_count, codes, scales,
                             stream) == hipSuccess
             ? MOE_OK
             : MOE_ERR_HIP;
}

int moe_mx4_pack(const uint8_t* in_codes, const uint8_t* in_scales, int64_t rows, int32_t cols, uint8_t* codes,
                 uint8_t* scales, hipStream_t stream) {
  if (!stream || !valid_size(rows, cols) || cols % 32) return MOE_ERR_INVALID_ARG;
  if (rows == 0) return MOE_OK;
  if (!in_codes || !in_scales || !codes || !scales || !aligned(in_codes, 16) || !aligned(codes, 16) ||
      !aligned(scales, 16))
    return MOE_ERR_INVALID_ARG;
  const int slices = mx4_slices(cols);
  const long long units = (rows + kMx4Rows - 1) / kMx4Rows * slices;
  mx4_pack_kernel<<<dim3(unit_grid(units)), 256, 0, stream>>>(in_codes, in_scales, rows, cols / 32, slices, units, codes,
                                                              scales);
  return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_HIP;
}

int moe_mx4_dequantize(const uint8_t* codes, const uint8_t* scales, int64_t rows, int32_t cols, void* out,
                       int32_t out_dtype, int64_t out_stride, hipStream_t stream) {
  if (!stream || !valid_size(rows, cols)) return MOE_ERR_INVALID_ARG;
  if (out_dtype != MOE_DTYPE_F32 && out_dtype != MOE_DTYPE_BF16) return MOE_ERR_INVALID_ARG;
  if (out_stride == 0) out_stride = cols;
  if (out_stride < cols) return MOE_ERR_INVALID_ARG;
  if (rows == 0) return MOE_OK;
  const int esz = out_dtype == MOE_DTYPE_F32 ? 4 : 2;
  if (!codes || !scales || !out || !aligned(codes, 16) || !aligned(scales, 16) || !aligned(out, esz))
    return MOE_ERR_INVALID_ARG;
  const int slices = mx4_slices(cols);
  const long long units = (rows + kMx4Rows - 1) / kMx4Rows * slices;
  auto go = [&](auto k) {
    k<<<dim3(unit_grid(units)), 256, 0, stream>>>(codes, scales, rows, cols, slices, units, out, out_stride);
  };
  esz == 2 ? go(mx4_dequantize_kernel<true>) : go(mx4_dequantize_kernel<false>);
  return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_HIP;
}

}  // extern "C"
