// Token rows into expert order and, weighted, back, with their gradients and the gate's
// (include/moepd_rows.h).  All of it is one pass over rows: what bounds it is memory, and
// for small batches the launch.  A lane takes 8 neighbouring values of a row at a time (16
// bytes of bf16, 32 of float32), at any alignment; a row's last values go one by one.
#include "common.h"
#include "kernels.h"
#include "moepd_rows.h"
#include "swiglu.h"
#include "tiles.h"

#include <algorithm>
#include <type_traits>

namespace moepd {
namespace {

typedef uint32_t u32x4_at4 __attribute__((ext_vector_type(4), aligned(4)));

constexpr int kSmallTokens = 2048;           // batches that share a row among waves
constexpr int kRowVec = 8;                   // values of a lane and pass
constexpr int kRowPass = kWave * kRowVec;    // values of a wave and pass

// Batches of more than kSmallTokens go past the caches (STREAM), as wide rows that each move once
// should.  The rule counts tokens, not bytes, and rows that are still in the caches would rather stay: the
// same rows again and again, us, through the caches / past them, k = 8 with an eighth of the slots resident,
// bf16: 2049 tokens of 40 gather 2.0 / 2.0, combine 3.5 / 3.5, its gradient 8.3 / 9.0; 8192 of 64 3.1 / 3.1, 5.0 / 4.9,
// 21 / 20; 8192 of 512 4.0 / 3.4, 4.9 / 6.5, 21 / 20; 8192 of 7168 34 / 34, 34 / 45, 95 / 81 (from memory combine 50, its
// gradient 78 past them); 1000 of 32768 18 / 18, 20 / 26, 56 / 112.
template <bool STREAM, class V>
__device__ __forceinline__ V row_get(const uint8_t* p) {
  if constexpr (STREAM) return __builtin_nontemporal_load(reinterpret_cast<const V*>(p));
  else return *reinterpret_cast<const V*>(p);
}
template <bool STREAM, class V>
__device__ __forceinline__ void row_put(uint8_t* p, V v) {
  if constexpr (STREAM) __builtin_nontemporal_store(v, reinterpret_cast<V*>(p));
  else *reinterpret_cast<V*>(p) = v;
}

// 8 values from element `at` of a row of n on; those past the row are 0.
template <bool BF16, bool STREAM>
__device__ __forceinline__ void row_load(const uint8_t* row, int at, int n, float (&v)[8]) {
  if (at + 8 <= n) {
    if constexpr (BF16) {
      const u32x4_any q = row_get<STREAM, u32x4_any>(row + 2LL * at);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(q[i] << 16);
        v[2 * i + 1] = __uint_as_float(q[i] & 0xffff0000u);
      }
    } else {
      const u32x4_at4 a = row_get<STREAM, u32x4_at4>(row + 4LL * at);
      const u32x4_at4 b = row_get<STREAM, u32x4_at4>(row + 4LL * at + 16);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[i] = __uint_as_float(a[i]);
        v[4 + i] = __uint_as_float(b[i]);
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      v[i] = 0.f;
      if (at + i < n) {
        if constexpr (BF16) v[i] = bf16_to_f32(reinterpret_cast<const uint16_t*>(row)[at + i]);
        else v[i] = reinterpret_cast<const float*>(row)[at + i];
      }
    }
  }
}
template <bool BF16, bool STREAM>
__device__ __forceinline__ void row_store(uint8_t* row, int at, int n, const float (&v)[8]) {
  if (at + 8 <= n) {
    if constexpr (BF16) {
      row_put<STREAM>(row + 2LL * at, u32x4_any{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]),
                                                bf16_pair(v[6], v[7])});
    } else {
      row_put<STREAM>(row + 4LL * at, u32x4_at4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]),
                                                __float_as_uint(v[3])});
      row_put<STREAM>(row + 4LL * at + 16, u32x4_at4{__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]),
                                                     __float_as_uint(v[7])});
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (at + i < n) {
        if constexpr (BF16) reinterpret_cast<uint16_t*>(row)[at + i] = f32_to_bf16(v[i]);
        else reinterpret_cast<float*>(row)[at + i] = v[i];
      }
  }
}

// This wave's place among all: workgroups of four.
__device__ __forceinline__ long long wave_index() {
  return ((long long)blockIdx.y * gridDim.x + blockIdx.x) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
}

// ------------------------------------------------------------------ gather

// 65,532 rows of 2048 float32 from 16,383 tokens: 153 us, 4.4 TB/s of which the rows are four fifths.
// A row is copied as it is (by 16 bytes; the last ones by element), so bits of NaN survive.
template <int SIZE, bool STREAM>
__global__ __launch_bounds__(256) void rows_gather_kernel(const uint8_t* x, long long x_stride, int T,
                                                          const int32_t* token_of_row, const int32_t* row_count, int rows,
                                                          int hidden, uint8_t* out, long long out_stride, int parts) {
  const long long w = wave_index();
  const long long r = w / parts;
  const int part = (int)(w - r * parts), lane = threadIdx.x & 63;
  if (r >= (row_count ? min(max(*row_count, 0), rows) : rows)) return;
  const int t = token_of_row[r];
  const bool live = t >= 0 && t < T;
  const uint8_t* from = x + (live ? t : 0) * x_stride * SIZE;
  uint8_t* to = out + r * out_stride * SIZE;
  constexpr int EACH = 16 / SIZE, U = 4;
  const int whole = hidden / EACH;
  for (int v0 = part * (64 * U); v0 < whole; v0 += parts * (64 * U)) {
    u32x4_any q[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int v = v0 + 64 * i + lane;
      q[i] = u32x4_any{0, 0, 0, 0};
      if (live && v < whole) q[i] = *reinterpret_cast<const u32x4_any*>(from + 16LL * v);
    }
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int v = v0 + 64 * i + lane;
      if (v < whole) row_put<STREAM>(to + 16LL * v, q[i]);
    }
  }
  const int at = whole * EACH + lane;
  if (part == 0 && at < hidden) {
    if constexpr (SIZE == 2) reinterpret_cast<uint16_t*>(to)[at] = live ? reinterpret_cast<const uint16_t*>(from)[at] : 0;
    else reinterpret_cast<uint32_t*>(to)[at] = live ? reinterpret_cast<const uint32_t*>(from)[at] : 0u;
  }
}

// ------------------------------------------------------------------ combine

// The waves of a token share its row: a wave that takes more of it waits for memory once a
// pass, and one token's slots are few.  8192 tokens of k = 8, an eighth of the slots resident, 7168 bf16: one wave a
// token 74 us (four passes at a time, which takes 190 registers, 108), four 57, seven 50 (4.7 TB/s).  16383 tokens of
// four slots, 2048 float32: 132 us, 5.1 TB/s.
template <bool YB, bool OB, bool STREAM>
__global__ __launch_bounds__(256) void rows_combine_kernel(const uint8_t* y, long long y_stride, int rows, const float* w,
                                                           const int32_t* row_of_slot, int T, int k, int hidden,
                                                           uint8_t* out, long long out_stride, int parts) {
  const long long wi = wave_index();
  const long long t = wi / parts;
  if (t >= T) return;
  const int part = (int)(wi - t * parts), lane = threadIdx.x & 63;
  const int r_l = lane < k ? row_of_slot[t * k + lane] : -1;
  const float w_l = lane < k && w ? w[t * k + lane] : 1.f;
  const uint64_t resident = __ballot(r_l >= 0 && r_l < rows);
  uint8_t* o = out + t * out_stride * (OB ? 2 : 4);
  constexpr int GROUP = STREAM ? 2 : 4;  // rows in flight
  for (int at0 = part * kRowPass; at0 < hidden; at0 += parts * kRowPass) {
    const int at = at0 + kRowVec * lane;
    float acc[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) acc[i] = 0.f;
    uint64_t m = resident;
    while (m) {  // in slot order
      float v[GROUP][8], f[GROUP];
      int n = 0;
#pragma unroll
      for (int q = 0; q < GROUP; ++q) {
        f[q] = 0.f;
        if (m) {
          const int j = __builtin_ctzll(m);
          m &= m - 1;
          f[q] = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(w_l), j));
          row_load<YB, STREAM>(y + __builtin_amdgcn_readlane(r_l, j) * y_stride * (YB ? 2 : 4), at, hidden, v[q]);
          n = q + 1;
        }
      }
#pragma unroll
      for (int q = 0; q < GROUP; ++q)
        if (q < n)
#pragma unroll
          for (int i = 0; i < 8; ++i) acc[i] = __builtin_fmaf(f[q], v[q][i], acc[i]);
    }
    row_store<OB, STREAM>(o, at, hidden, acc);
  }
}

// ------------------------------------------------------------------ combine, backward

__device__ __forceinline__ float wave_sum(float v) {  // the same order in every run
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, kWave);
  return v;
}

// A wave takes every parts-th of its token's slots that have a row: with one wave a token, tokens of many
// resident slots set the pace (8192 tokens as above: 114 us, with four 78, 4.5 TB/s).
template <bool DB, bool YB, bool GB, bool STREAM>
__global__ __launch_bounds__(256) void rows_combine_backward_kernel(const uint8_t* dout, long long dout_stride,
                                                                    const uint8_t* y, long long y_stride, int rows,
                                                                    const float* w, const int32_t* row_of_slot, int T,
                                                                    int k, int hidden, uint8_t* dy, long long dy_stride,
                                                                    float* dw, int parts) {
  const long long wi = wave_index();
  const long long t = wi / parts;
  if (t >= T) return;
  const int part = (int)(wi - t * parts), lane = threadIdx.x & 63;
  const int r_l = lane < k ? row_of_slot[t * k + lane] : -1;
  const float w_l = lane < k && w ? w[t * k + lane] : 1.f;
  const bool has = r_l >= 0 && r_l < rows;
  uint64_t m = __ballot(has);
  if (dw && part == 0 && lane < k && !has) dw[t * k + lane] = 0.f;
  const uint8_t* d = dout + t * dout_stride * (DB ? 2 : 4);
  for (int i = 0; i < part; ++i) m &= m - 1;  // 0 stays 0
  while (m) {
    const int j = __builtin_ctzll(m);
    for (int i = 0; i < parts; ++i) m &= m - 1;
    const long long r = __builtin_amdgcn_readlane(r_l, j);
    const float f = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(w_l), j));
    const uint8_t* yr = y + r * y_stride * (YB ? 2 : 4);
    uint8_t* g = dy + r * dy_stride * (GB ? 2 : 4);
    float sum = 0.f;
    constexpr int U = STREAM ? 4 : 2;
    for (int at0 = 0; at0 < hidden; at0 += U * kRowPass) {
      float dv[U][8], yv[U][8];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int at = at0 + u * kRowPass + kRowVec * lane;
        row_load<DB, false>(d, at, hidden, dv[u]);
        if (dw) row_load<YB, STREAM>(yr, at, hidden, yv[u]);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int at = at0 + u * kRowPass + kRowVec * lane;
        float o[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          if (dw) sum = __builtin_fmaf(dv[u][i], yv[u][i], sum);
          o[i] = f * dv[u][i];
        }
        row_store<GB, STREAM>(g, at, hidden, o);
      }
    }
    if (dw) {
      sum = wave_sum(sum);
      if (lane == 0) dw[t * k + j] = sum;
    }
  }
}

// ------------------------------------------------------------------ gate

template <bool BF16>
__global__ __launch_bounds__(256) void rows_gate_backward_kernel(const int32_t* idx, const float* w, const float* dw, int T,
                                                                 int E, int k, uint8_t* dlogits, long long stride,
                                                                 bool accumulate) {
  const long long t = wave_index();
  if (t >= T) return;
  const int lane = threadIdx.x & 63;
  const int i_l = lane < k ? idx[t * k + lane] : -1;
  const float w_l = lane < k ? w[t * k + lane] : 0.f;
  const float d_l = lane < k ? dw[t * k + lane] : 0.f;
  float mean = 0.f;
  for (int j = 0; j < k; ++j)
    mean = __builtin_fmaf(__int_as_float(__builtin_amdgcn_readlane(__float_as_int(w_l), j)),
                          __int_as_float(__builtin_amdgcn_readlane(__float_as_int(d_l), j)), mean);
  const float g_l = w_l * (d_l - mean);
  uint8_t* o = dlogits + t * stride * (BF16 ? 2 : 4);
  for (int e = lane; e < E; e += kWave) {
    float v = 0.f;
    bool any = false;
    for (int j = 0; j < k; ++j) {
      const bool here = __builtin_amdgcn_readlane(i_l, j) == e;
      v += here ? __int_as_float(__builtin_amdgcn_readlane(__float_as_int(g_l), j)) : 0.f;
      any |= here;
    }
    if (accumulate && !any) continue;
    if constexpr (BF16) {
      uint16_t* p = reinterpret_cast<uint16_t*>(o) + e;
      *p = f32_to_bf16(accumulate ? bf16_to_f32(*p) + v : v);
    } else {
      float* p = reinterpret_cast<float*>(o) + e;
      *p = accumulate ? *p + v : v;
    }
  }
}

// ------------------------------------------------------------------ host side

bool type_ok(int32_t t) { return t == MOE_DTYPE_F32 || t == MOE_DTYPE_BF16; }
bool bf16(int32_t t) { return t == MOE_DTYPE_BF16; }
bool at_element(const void* p, int32_t t) { return (uintptr_t)p % (t == MOE_DTYPE_F32 ? 4 : 2) == 0; }
bool stride_of(int64_t* stride, int32_t width) {
  if (*stride == 0) *stride = width;
  return *stride >= width;
}
bool tokens_ok(int32_t T, int32_t k, int32_t hidden, int64_t rows, hipStream_t s) {
  return s && T >= 0 && T <= (1 << 24) && k >= 1 && k <= kMaxTopK && hidden >= 1 && hidden <= (1 << 20) && rows >= 0 &&
         rows <= (1LL << 31) - 512;
}
dim3 waves_grid(long long waves) { return grid_of((waves + 3) / 4, 256); }
int done() { return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_HIP; }

}  // namespace
}  // namespace moepd

using namespace moepd;

extern "C" {

int moe_rows_gather(const void* x, int32_t dtype, int64_t x_stride, int32_t T, const int32_t* token_of_row,
                    const int32_t* row_count, int64_t rows, int32_t hidden, void* out, int64_t out_stride,
                    hipStream_t stream) {
  if (!tokens_ok(T, 1, hidden, rows, stream) || !type_ok(dtype) || !stride_of(&x_stride, hidden) ||
      !stride_of(&out_stride, hidden) || !at_element(x, dtype) || !at_element(out, dtype) ||
      ((uintptr_t)token_of_row | (uintptr_t)row_count) % 4)
    return MOE_ERR_INVALID_ARG;
  if (rows == 0) return MOE_OK;
  if ((!x && T > 0) || !token_of_row || !out) return MOE_ERR_INVALID_ARG;
  const int size = bf16(dtype) ? 2 : 4;
  const int parts = std::max(1, (hidden * size / 16 + 255) / 256);
  const dim3 grid = waves_grid(rows * parts);
  auto go = [&](auto kernel) {
    kernel<<<grid, 256, 0, stream>>>((const uint8_t*)x, x_stride, T, token_of_row, row_count, (int)rows, hidden,
                                     (uint8_t*)out, out_stride, parts);
  };
  if (rows > kSmallTokens) bf16(dtype) ? go(rows_gather_kernel<2, true>) : go(rows_gather_kernel<4, true>);
  else bf16(dtype) ? go(rows_gather_kernel<2, false>) : go(rows_gather_kernel<4, false>);
  return done();
}

int moe_rows_combine(const void* y, int32_t y_dtype, int64_t y_stride, int64_t rows, const float* w,
                     const int32_t* row_of_slot, int32_t T, int32_t k, int32_t hidden, void* out, int32_t out_dtype,
                     int64_t out_stride, hipStream_t stream) {
  if (!tokens_ok(T, k, hidden, rows, stream) || !type_ok(y_dtype) || !type_ok(out_dtype) || !stride_of(&y_stride, hidden) ||
      !stride_of(&out_stride, hidden) || !at_element(y, y_dtype) || !at_element(out, out_dtype) ||
      ((uintptr_t)w | (uintptr_t)row_of_slot) % 4)
    return MOE_ERR_INVALID_ARG;
  if (T == 0) return MOE_OK;
  if ((!y && rows > 0) || !row_of_slot || !out) return MOE_ERR_INVALID_ARG;
  const bool large = T > kSmallTokens;
  const int parts = (hidden + kRowPass * (large ? 2 : 1) - 1) / (kRowPass * (large ? 2 : 1));
  const dim3 grid = waves_grid((long long)T * parts);
  auto go = [&](auto kernel) {
    kernel<<<grid, 256, 0, stream>>>((const uint8_t*)y, y_stride, (int)rows, w, row_of_slot, T, k, hidden, (uint8_t*)out,
                                     out_stride, parts);
  };
  auto by_out = [&](auto yb, auto ob) {
    constexpr bool Y = decltype(yb)::value, O = decltype(ob)::value;
    large ? go(rows_combine_kernel<Y, O, true>) : go(rows_combine_kernel<Y, O, false>);
  };
  auto by_y = [&](auto yb) { bf16(out_dtype) ? by_out(yb, std::true_type{}) : by_out(yb, std::false_type{}); };
  bf16(y_dtype) ? by_y(std::true_type{}) : by_y(std::false_type{});
  return done();
}

int moe_rows_combine_backward(const void* dout, int32_t dout_dtype, int64_t dout_stride, const void* y, int32_t y_dtype,
                              int64_t y_stride, int64_t rows, const float* w, const int32_t* row_of_slot, int32_t T,
                              int32_t k, int32_t hidden, void* dy, int32_t dy_dtype, int64_t dy_stride, float* dw,
                              hipStream_t stream) {
  if (!tokens_ok(T, k, hidden, rows, stream) || !type_ok(dout_dtype) || !type_ok(y_dtype) || !type_ok(dy_dtype) ||
      !stride_of(&dout_stride, hidden) || !stride_of(&y_stride, hidden) || !stride_of(&dy_stride, hidden) ||
      !at_element(dout, dout_dtype) || !at_element(y, y_dtype) || !at_element(dy, dy_dtype) ||
      ((uintptr_t)w | (uintptr_t)row_of_slot | (uintptr_t)dw) % 4)
    return MOE_ERR_INVALID_ARG;
  if (T == 0) return MOE_OK;
  if (!dout || !row_of_slot || (rows > 0 && (!dy || (dw && !y)))) return MOE_ERR_INVALID_ARG;
  const bool large = T > kSmallTokens;
  const int parts = large ? (k < 4 ? k : 4) : k;
  const dim3 grid = waves_grid((long long)T * parts);
  auto go = [&](auto kernel) {
    kernel<<<grid, 256, 0, stream>>>((const uint8_t*)dout, dout_stride, (const uint8_t*)y, y_stride, (int)rows, w,
                                     row_of_slot, T, k, hidden, (uint8_t*)dy, dy_stride, dw, parts);
  };
  auto by_dy = [&](auto d, auto yb) {
    constexpr bool D = decltype(d)::value, Y = decltype(yb)::value;
    if (large)
      bf16(dy_dtype) ? go(rows_combine_backward_kernel<D, Y, true, true>) : go(rows_combine_backward_kernel<D, Y, false, true>);
    else
      bf16(dy_dtype) ? go(rows_combine_backward_kernel<D, Y, true, false>) : go(rows_combine_backward_kernel<D, Y, false, false>);
  };
  auto by_y = [&](auto d) { bf16(y_dtype) ? by_dy(d, std::true_type{}) : by_dy(d, std::false_type{}); };
  bf16(dout_dtype) ? by_y(std::true_type{}) : by_y(std::false_type{});
  return done();
}

int moe_gate_backward(const int32_t* topk_idx, const float* topk_w, const float* dw, int32_t T, int32_t E, int32_t k,
                      void* dlogits, int32_t dlogits_dtype, int64_t dlogits_stride, int32_t accumulate,
                      hipStream_t stream) {
  if (!tokens_ok(T, k, 1, 0, stream) || E < 1 || E > kMaxExperts || k > E || !type_ok(dlogits_dtype) ||
      !stride_of(&dlogits_stride, E) || !at_element(dlogits, dlogits_dtype) ||
      ((uintptr_t)topk_idx | (uintptr_t)topk_w | (uintptr_t)dw) % 4)
    return MOE_ERR_INVALID_ARG;
  if (T == 0) return MOE_OK;
  if (!topk_idx || !topk_w || !dw || !dlogits) return MOE_ERR_INVALID_ARG;
  const dim3 grid = waves_grid(T);
  if (bf16(dlogits_dtype))
    rows_gate_backward_kernel<true><<<grid, 256, 0, stream>>>(topk_idx, topk_w, dw, T, E, k, (uint8_t*)dlogits,
                                                              dlogits_stride, accumulate != 0);
  else
    rows_gate_backward_kernel<false><<<grid, 256, 0, stream>>>(topk_idx, topk_w, dw, T, E, k, (uint8_t*)dlogits,
                                                               dlogits_stride, accumulate != 0);
  return done();
}

}  // extern "C"
