// The gated feed-forward block and its backward pass (include/moepd_ffn.h): tiles, launches and
// the C entry points.  The tile itself is in ffn_ring.h (bf16) and ffn_block_f32.h.
#include <algorithm>
#include <type_traits>

#include "common.h"
#include "ffn_ring.h"
#include "ffn_block_f32.h"
#include "kernels.h"
#include "moepd_ffn.h"
#include "tiles.h"

namespace moepd {
namespace {

// ------------------------------------------------------------------ rows times a group's weights

template <int SHARE>
__device__ __forceinline__ bool ffn_row_tile(const FfnArgs& g, int bm, int bn, FfnTile& t) {
  GroupTile w;
  if (!group_tile<false, SHARE>(g, (int)(blockIdx.y * gridDim.x + blockIdx.x), bm, w)) return false;
  t.group = w.group;
  t.m0 = w.m0;
  t.rows = w.m_end - w.m0;
  t.n0 = w.nt * bn;
  t.k0 = t.k_count = 0;
  return true;
}

// A tile of up to 160 rows, cut to the 32-row blocks that it holds; four waves side by side along the
// columns.  32 groups, H 7168, I 2048, gate/up: 128 rows each 350 us, 5.7 TB/s (the weights 5.4); 320 rows 571,
// 1050 TFLOP/s.  Two workgroups to a CU with 32-deep slices, whose rows are half a line, were 22 % slower at 257 rows.
template <int KIND, bool F32>
__device__ __forceinline__ void ffn_mid_tile(const FfnArgs& g, const FfnTile& t, u32x4* lds) {
  const int blocks = (t.rows + 31) / 32;
  if (blocks <= 1) ffn_tile<KIND, F32, 32, 256, 64, 1, 4, 3, 3>(g, t, g.c, lds);
  else if (blocks == 2) ffn_tile<KIND, F32, 64, 256, 64, 1, 4, 3, 3>(g, t, g.c, lds);
  else if (blocks == 3) ffn_tile<KIND, F32, 96, 256, 64, 1, 4, 3, 3>(g, t, g.c, lds);
  else if (blocks == 4) ffn_tile<KIND, F32, 128, 256, 64, 1, 4, 3, 3>(g, t, g.c, lds);
  else ffn_tile<KIND, F32, 160, 256, 64, 1, 4, 3, 3>(g, t, g.c, lds);
}
template <int KIND, bool F32>
__global__ __launch_bounds__(256) void ffn_block_mid(FfnArgs g) {
  __shared__ u32x4 lds[ffn_chunks(kFfnMidRows, 256, 64, 3, 3)];
  FfnTile t;
  if (ffn_row_tile(g, g.bm, KIND == kFfnGateUp ? 128 : 256, t)) ffn_mid_tile<KIND, F32>(g, t, lds);
}

// Groups of more rows (1024 in each of 32 groups, H 7168, I 2048: gate/up 1494 us, 1290 TFLOP/s): tiles of 256 by a 2 x 2 grid of waves, the rows' slices one ahead of the weights', and a
// rest of up to 160 rows in a tile cut to it.
template <int KIND, bool F32>
__global__ __launch_bounds__(256) void ffn_block_wide(FfnArgs g) {
  __shared__ u32x4 lds[ffn_chunks(kFfnWideRows, 256, 64, 3, 2)];
  static_assert(ffn_chunks(kFfnMidRows, 256, 64, 3, 3) <= ffn_chunks(kFfnWideRows, 256, 64, 3, 2), "the rest's ring");
  FfnTile t;
  if (!ffn_row_tile<kRowsFull>(g, kFfnWideRows, KIND == kFfnGateUp ? 128 : 256, t)) return;
  if (t.rows > kFfnMidRows) ffn_tile<KIND, F32, 256, 256, 64, 2, 2, 3, 2>(g, t, g.c, lds);
  else ffn_mid_tile<KIND, F32>(g, t, lds);
}

// Few rows: up to 8 by eight waves of two or three blocks in flight each, up to 32 by four of three.  One token, H
// 7168, I 2048: gate/up 12 us (4.7 TB/s of weights), down 7; 256 rows: gate/up 37, where a tile of 160 rows takes 81.
template <int KIND, bool F32, int RA>
__global__ __launch_bounds__(RA == 8 ? 512 : 256) void ffn_block_few(FfnArgs g) {
  constexpr int NB = ffn_few_columns(KIND, RA) == (KIND == kFfnGateUp ? 16 : 32) ? 1 : 2;
  constexpr int W = RA == 8 ? 8 : 4, S = RA == 8 && NB == 2 ? 2 : 3;
  __shared__ u32x4 lds[ffn_few_chunks(RA, NB, W, S)];
  FfnTile t;
  if (!ffn_row_tile(g, RA, ffn_few_columns(KIND, RA), t)) return;
  ffn_few_tile<KIND, F32, RA, NB, W, S>(g, t, lds);
}

// ------------------------------------------------------------------ gradients of the weights

// Workgroup b's tile: parts of the rows outermost, then groups; within a group blocks of four
// column tiles, row tile by row tile; runs of consecutive tiles dealt to the XCDs in turn.
__device__ __forceinline__ bool ffn_weight_tile(const FfnArgs& g, int bm, int bn, FfnTile& t, int& split) {
  const int b = (int)(blockIdx.y * gridDim.x + blockIdx.x);
  const int per = g.m_tiles * g.n_tiles, total = per * g.groups * g.splits;
  const int x = b & 7, slot = b >> 3, round = slot / g.run, base = round * 8 * g.run, j = slot - round * g.run;
  const int L = uniform(base + 8 * g.run <= total ? base + x * g.run + j : base + 8 * j + x);
  if (L >= total) return false;
  const int sg = L / per, at = L - sg * per;
  split = sg / g.groups;
  t.group = sg - split * g.groups;
  const int q = at / (4 * g.m_tiles), r = at - q * 4 * g.m_tiles;
  const int width = min(4, g.n_tiles - 4 * q);
  const int mi = r / width;
  t.m0 = mi * bm;
  t.rows = min(bm, g.m - t.m0);
  t.n0 = (4 * q + r - mi * width) * bn;
  int lo = 0, hi = g.rows;
  if (g.offsets) {
    lo = uniform(min(max(g.offsets[t.group], 0), g.rows));
    hi = uniform(max(lo, min(g.offsets[t.group + 1], g.rows)));
  }
  const int part = (hi - lo + g.splits - 1) / g.splits;
  const int each = (part + 63) / 64 * 64;
  t.k0 = min((long long)hi, lo + (long long)split * each);
  t.k_count = min(each, hi - t.k0);
  return true;
}

// Two workgroups share a CU.  What bounds them, for the few hundred rows of a group in training, is the results'
// way out, through LDS and to memory: w_gate_up's gradient of 32 groups, 4096 x 7168, a dozen passes in a row, 128 rows
// 405 to 425 us (4.7 to 4.9 TB/s), 257 610 to 650 (of drawn lengths, forty passes in a row, 698), 512 1050 (920 TFLOP/s);
// results past the caches 883 -> 717 at 257 rows, rounded before LDS 675 -> 625.  256 x 128
// tiles are 3 % slower (their rows of results are half as long), 128 x 128, three to a CU, 5.
// ADD: bf16 results that are added to what is there.
template <bool F32, bool ADD>
__global__ __launch_bounds__(256, 2) void ffn_block_weights(FfnArgs g) {
  __shared__ u32x4 lds[ffn_chunks(kFfnWeightRows, kFfnWeightCols, 32, 3, 3)];
  FfnTile t;
  int split;
  if (!ffn_weight_tile(g, kFfnWeightRows, kFfnWeightCols, t, split)) return;
  if (g.accumulate && t.k_count == 0) return;  // nothing to add
  uint8_t* c = g.c + ((long long)split * g.groups + t.group) * g.m * g.ldc;
  ffn_tile<kFfnWeightGrad, F32, kFfnWeightRows, kFfnWeightCols, 32, 2, 2, 3, 3, !F32 && !ADD>(g, t, c, lds);
}

// The parts' sums, in order, to the result: four values to a thread, eight parts in flight.
template <bool F32>
__global__ __launch_bounds__(256) void ffn_block_join(const float* parts, long long values, int splits, int accumulate,
                                                      uint8_t* out) {
  const long long at = ((long long)blockIdx.x * 256 + threadIdx.x) * 4;
  if (at >= values) return;
  typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
  const f32x4_ffn* p = reinterpret_cast<const f32x4_ffn*>(parts + at);
  f32x4_ffn v = {0.f, 0.f, 0.f, 0.f};
  constexpr int U = 8;
  for (int s = 0; s < splits; s += U) {
    f32x4_ffn q[U];
#pragma unroll
    for (int i = 0; i < U; ++i) q[i] = s + i < splits ? p[(s + i) * (values / 4)] : f32x4_ffn{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < U; ++i) v += q[i];
  }
  if constexpr (F32) {
    f32x4_ffn* o = reinterpret_cast<f32x4_ffn*>(out + at * 4);
    *o = accumulate ? *o + v : v;
  } else {
    u32x2* o = reinterpret_cast<u32x2*>(out + at * 2);
    if (accumulate) {
      const u32x2 w = *o;
      v += f32x4_ffn{__uint_as_float(w[0] << 16), __uint_as_float(w[0] & 0xffff0000u), __uint_as_float(w[1] << 16),
                     __uint_as_float(w[1] & 0xffff0000u)};
    }
    *o = u32x2{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3])};
  }
}

// ------------------------------------------------------------------ host side

constexpr long long kMostBlocks = (1LL << 31) - (1 << 16);

bool launched() { return hipGetLastError() == hipSuccess; }

int launch_rows(FfnArgs g, int kind, bool out_f32, bool f32, hipStream_t s) {
  if (f32) {
    g.n_tiles = (g.n + kFfnF32Cols - 1) / kFfnF32Cols;
    g.run = 32;
    const long long tiles = (g.rows / kFfnF32Rows + (long long)g.groups) * g.n_tiles;
    if (tiles > kMostBlocks) return MOE_ERR_INVALID_ARG;
    const dim3 grid = grid_of((tiles + 7) / 8 * 8, 256);
    switch (kind) {
      case kFfnGateUp: ffn_block_f32<kFfnGateUp><<<grid, 256, 0, s>>>(g); break;
      case kFfnDown: ffn_block_f32<kFfnDown><<<grid, 256, 0, s>>>(g); break;
      case kFfnDownGrad: ffn_block_f32<kFfnDownGrad><<<grid, 256, 0, s>>>(g); break;
      default: ffn_block_f32<kFfnGateUpGrad><<<grid, 256, 0, s>>>(g);
    }
    return launched() ? MOE_OK : MOE_ERR_HIP;
  }
  const FfnForm f = ffn_form(kind, g.rows, g.groups, g.n, g.k);
  if (f.count > kMostBlocks) return MOE_ERR_INVALID_ARG;
  g.bm = f.rows;
  g.n_tiles = f.n_tiles;
  g.run = f.run;
  const dim3 grid = grid_of((f.count + 7) / 8 * 8, f.threads());
  auto go = [&](auto kind_of, auto f32_of) {
    constexpr int KIND = decltype(kind_of)::value;
    constexpr bool F32 = decltype(f32_of)::value;
    switch (f.tiles) {
      case kFfnFew8: ffn_block_few<KIND, F32, 8><<<grid, f.threads(), 0, s>>>(g); break;
      case kFfnFew32: ffn_block_few<KIND, F32, 32><<<grid, f.threads(), 0, s>>>(g); break;
      case kFfnMid: ffn_block_mid<KIND, F32><<<grid, f.threads(), 0, s>>>(g); break;
      default: ffn_block_wide<KIND, F32><<<grid, f.threads(), 0, s>>>(g);
    }
  };
  using No = std::false_type;
  using Yes = std::true_type;
  switch (kind) {
    case kFfnGateUp: go(std::integral_constant<int, kFfnGateUp>{}, No{}); break;
    case kFfnDown:
      if (out_f32) go(std::integral_constant<int, kFfnDown>{}, Yes{});
      else go(std::integral_constant<int, kFfnDown>{}, No{});
      break;
    case kFfnDownGrad: go(std::integral_constant<int, kFfnDownGrad>{}, No{}); break;
    default:
      if (out_f32) go(std::integral_constant<int, kFfnGateUpGrad>{}, Yes{});
      else go(std::integral_constant<int, kFfnGateUpGrad>{}, No{});
  }
  return launched() ? MOE_OK : MOE_ERR_HIP;
}

constexpr int kMostWidth = 32768;
constexpr long long kMostStride = 1 << 20;

bool shape_ok(int64_t rows, int32_t groups, const int32_t* offsets, int32_t H, int32_t I, int32_t dtype, hipStream_t s) {
  if (!s || rows < 0 || rows > (1LL << 31) - 512) return false;
  if (groups < 1 || groups > 1024 || (!offsets && groups != 1) || (uintptr_t)offsets % 4) return false;
  if (H < 8 || H > kMostWidth || H % 8 || I < 8 || I > kMostWidth || I % 8 || (long long)H * I > (1 << 28)) return false;
  return dtype == MOE_DTYPE_F32 || dtype == MOE_DTYPE_BF16;
}

bool stride_ok(int64_t* stride, int width) {
  if (*stride == 0) *stride = width;
  return *stride >= width && *stride <= kMostStride && *stride % 8 == 0;
}

bool out_ok(int32_t out, int32_t dtype) { return out == MOE_DTYPE_F32 || (out == MOE_DTYPE_BF16 && dtype == MOE_DTYPE_BF16); }

template <class... P>
bool aligned16(const P*... p) {
  return ((0 | ... | (uintptr_t)p) % 16) == 0;
}

int size_of(int32_t dtype) { return dtype == MOE_DTYPE_F32 ? 4 : 2; }

long long weight_bytes(long long rows, int groups, int m, int n) {
  const int s = ffn_weight_parts(rows, groups, m, n);
  return s > 1 ? 4LL * s * groups * m * n : 0;
}
bool weight_shape_ok(int64_t rows, int32_t groups, int32_t m, int32_t n) {
  return rows >= 0 && rows <= (1LL << 31) - 512 && groups >= 1 && groups <= 1024 && m >= 8 && n >= 8 && m % 8 == 0 &&
         n % 8 == 0 && m <= 2 * kMostWidth && n <= 2 * kMostWidth && (long long)m * n <= (1 << 29);
}

}  // namespace
}  // namespace moepd

using namespace moepd;

extern "C" {

int moe_ffn_gate_up(const void* x, int64_t x_stride, int64_t rows, const void* w_gate_up, int32_t groups,
                    const int32_t* offsets, int32_t hidden, int32_t inter, int32_t dtype, void* gate_up, void* h,
                    hipStream_t stream) {
  if (!shape_ok(rows, groups, offsets, hidden, inter, dtype, stream) || !stride_ok(&x_stride, hidden))
    return MOE_ERR_INVALID_ARG;
  if (!aligned16(x, w_gate_up, gate_up, h)) return MOE_ERR_INVALID_ARG;
  if (rows == 0) return MOE_OK;
  if (!x || !w_gate_up || !h) return MOE_ERR_INVALID_ARG;
  const int sz = size_of(dtype);
  FfnArgs g{};
  g.a = (const uint8_t*)x;
  g.b = (const uint8_t*)w_gate_up;
  g.c = (uint8_t*)gate_up;
  g.h = (uint8_t*)h;
  g.lda = x_stride * sz;
  g.ldb = (long long)hidden * sz;
  g.b_group = 2LL * inter * hidden * sz;
  g.offsets = offsets;
  g.rows = (int)rows;
  g.groups = groups;
  g.n = inter;
  g.k = hidden;
  return launch_rows(g, kFfnGateUp, false, dtype == MOE_DTYPE_F32, stream);
}

int moe_ffn_down(const void* h, int64_t rows, const void* w_down, int32_t groups, const int32_t* offsets, int32_t hidden,
                 int32_t inter, int32_t dtype, void* y, int32_t y_dtype, int64_t y_stride, hipStream_t stream) {
  if (!shape_ok(rows, groups, offsets, hidden, inter, dtype, stream) || !stride_ok(&y_stride, hidden) ||
      !out_ok(y_dtype, dtype) || !aligned16(h, w_down, y))
    return MOE_ERR_INVALID_ARG;
  if (rows == 0) return MOE_OK;
  if (!h || !w_down || !y) return MOE_ERR_INVALID_ARG;
  const int sz = size_of(dtype);
  FfnArgs g{};
  g.a = (const uint8_t*)h;
  g.b = (const uint8_t*)w_down;
  g.c = (uint8_t*)y;
  g.lda = (long long)inter * sz;
  g.ldb = (long long)inter * sz;
  g.ldc = y_stride * size_of(y_dtype);
  g.b_group = (long long)inter * hidden * sz;
  g.offsets = offsets;
  g.rows = (int)rows;
  g.groups = groups;
  g.n = hidden;
  g.k = inter;
  return launch_rows(g, kFfnDown, y_dtype == MOE_DTYPE_F32, dtype == MOE_DTYPE_F32, stream);
}

int moe_ffn_down_backward(const void* dy, int64_t dy_stride, int64_t rows, const void* w_down, const void* gate_up,
                          int32_t groups, const int32_t* offsets, int32_t hidden, int32_t inter, int32_t dtype,
                          void* dgate_up, void* h, hipStream_t stream) {
  if (!shape_ok(rows, groups, offsets, hidden, inter, dtype, stream) || !stride_ok(&dy_stride, hidden) ||
      !aligned16(dy, w_down, gate_up, dgate_up, h))
    return MOE_ERR_INVALID_ARG;
  if (rows == 0) return MOE_OK;
  if (!dy || !w_down || !gate_up || !dgate_up) return MOE_ERR_INVALID_ARG;
  const int sz = size_of(dtype);
  FfnArgs g{};
  g.a = (const uint8_t*)dy;
  g.b = (const uint8_t*)w_down;
  g.c = (uint8_t*)dgate_up;
  g.h = (uint8_t*)h;
  g.gu = (const uint8_t*)gate_up;
  g.lda = dy_stride * sz;
  g.ldb = (long long)inter * sz;
  g.b_group = (long long)inter * hidden * sz;
  g.offsets = offsets;
  g.rows = (int)rows;
  g.groups = groups;
  g.n = inter;
  g.k = hidden;
  return launch_rows(g, kFfnDownGrad, false, dtype == MOE_DTYPE_F32, stream);
}

int moe_ffn_gate_up_backward(const void* dgate_up, int64_t rows, const void* w_gate_up, int32_t groups,
                             const int32_t* offsets, int32_t hidden, int32_t inter, int32_t dtype, void* dx,
                             int32_t dx_dtype, int64_t dx_stride, hipStream_t stream) {
  if (!shape_ok(rows, groups, offsets, hidden, inter, dtype, stream) || !stride_ok(&dx_stride, hidden) ||
      !out_ok(dx_dtype, dtype) || !aligned16(dgate_up, w_gate_up, dx))
    return MOE_ERR_INVALID_ARG;
  if (rows == 0) return MOE_OK;
  if (!dgate_up || !w_gate_up || !dx) return MOE_ERR_INVALID_ARG;
  const int sz = size_of(dtype);
  FfnArgs g{};
  g.a = (const uint8_t*)dgate_up;
  g.b = (const uint8_t*)w_gate_up;
  g.c = (uint8_t*)dx;
  g.lda = 2LL * inter * sz;
  g.ldb = (long long)hidden * sz;
  g.ldc = dx_stride * size_of(dx_dtype);
  g.b_group = 2LL * inter * hidden * sz;
  g.offsets = offsets;
  g.rows = (int)rows;
  g.groups = groups;
  g.n = hidden;
  g.k = 2 * inter;
  return launch_rows(g, kFfnGateUpGrad, dx_dtype == MOE_DTYPE_F32, dtype == MOE_DTYPE_F32, stream);
}

int moe_ffn_weight_workspace(int64_t rows, int32_t groups, int32_t m, int32_t n, int64_t* bytes) {
  if (!bytes || !weight_shape_ok(rows, groups, m, n)) return MOE_ERR_INVALID_ARG;
  *bytes = weight_bytes(rows, groups, m, n);
  return MOE_OK;
}

int moe_ffn_weight_grad(const void* a, int64_t a_stride, const void* b, int64_t b_stride, int64_t rows, int32_t groups,
                        const int32_t* offsets, int32_t m, int32_t n, int32_t dtype, void* dw, int32_t dw_dtype,
                        int32_t accumulate, void* workspace, int64_t workspace_bytes, hipStream_t stream) {
  if (!stream || !weight_shape_ok(rows, groups, m, n) || (!offsets && groups != 1) || (uintptr_t)offsets % 4 ||
      !stride_ok(&a_stride, m) || !stride_ok(&b_stride, n) || (dtype != MOE_DTYPE_F32 && dtype != MOE_DTYPE_BF16) ||
      !out_ok(dw_dtype, dtype) || !aligned16(a, b, dw) || !dw || (uintptr_t)workspace % 256)
    return MOE_ERR_INVALID_ARG;
  if (rows > 0 && (!a || !b)) return MOE_ERR_INVALID_ARG;
  const long long need = weight_bytes(rows, groups, m, n);
  if (need > 0 && !workspace) return MOE_ERR_INVALID_ARG;
  if (need > workspace_bytes) return MOE_ERR_CAPACITY;
  const int sz = size_of(dtype);
  const bool f32 = dw_dtype == MOE_DTYPE_F32;
  FfnArgs g{};
  g.a = (const uint8_t*)a;
  g.b = (const uint8_t*)b;
  g.lda = a_stride * sz;
  g.ldb = b_stride * sz;
  g.offsets = offsets;
  g.rows = (int)rows;
  g.groups = groups;
  g.m = m;
  g.n = n;
  g.splits = ffn_weight_parts(rows, groups, m, n);
  g.c = g.splits > 1 ? (uint8_t*)workspace : (uint8_t*)dw;
  g.accumulate = g.splits > 1 ? 0 : accumulate != 0;
  g.ldc = (long long)n * (g.splits > 1 ? 4 : size_of(dw_dtype));
  const int bm = dtype == MOE_DTYPE_F32 ? kFfnF32Rows : kFfnWeightRows;
  const int bn = dtype == MOE_DTYPE_F32 ? kFfnF32Cols : kFfnWeightCols;
  g.m_tiles = (m + bm - 1) / bm;
  g.n_tiles = (n + bn - 1) / bn;
  // An eighth of a group's tiles to each XCD, so that groups of any length weigh on all alike (32 groups of Zipf-skewed
  // lengths, 30001 rows, 2048 x 2048: 490 us with runs of 64, 378 so).  8243 rows, 32 groups, both gradients in turn:
  // 1117 us with at most 64 tiles to a run, 1054 with 112 and 56.
  g.run = std::min(std::max(g.m_tiles * g.n_tiles / 8, 4), 128);
  const long long tiles = (long long)g.m_tiles * g.n_tiles * groups * g.splits;
  if (tiles > kMostBlocks) return MOE_ERR_INVALID_ARG;
  const dim3 grid = grid_of((tiles + 7) / 8 * 8, 256);
  if (dtype == MOE_DTYPE_F32) ffn_block_f32_weights<<<grid, 256, 0, stream>>>(g);
  else if (f32 || g.splits > 1) ffn_block_weights<true, false><<<grid, 256, 0, stream>>>(g);
  else if (accumulate) ffn_block_weights<false, true><<<grid, 256, 0, stream>>>(g);
  else ffn_block_weights<false, false><<<grid, 256, 0, stream>>>(g);
  if (!launched()) return MOE_ERR_HIP;
  if (g.splits > 1) {
    const long long values = (long long)groups * m * n;
    const dim3 blocks((unsigned)((values / 4 + 255) / 256));
    if (f32) ffn_block_join<true><<<blocks, 256, 0, stream>>>((const float*)workspace, values, g.splits, accumulate != 0, (uint8_t*)dw);
    else ffn_block_join<false><<<blocks, 256, 0, stream>>>((const float*)workspace, values, g.splits, accumulate != 0, (uint8_t*)dw);
    if (!launched()) return MOE_ERR_HIP;
  }
  return MOE_OK;
}

}  // extern "C"
