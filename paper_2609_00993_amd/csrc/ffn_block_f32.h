// The gated feed-forward block's products in float32 on the vector ALUs: 64 x 64 results to a
// workgroup (gate/up: 64 of each), 4 x 4 to a thread, both operands through LDS in slices of 16
// of K whatever their layout.  The type for checks by differences, not for speed: what
// bounds it is the vector ALUs, four LDS reads to 16 (gate/up: five to 32) multiply-adds.
#pragma once

#include "ffn_ring.h"

namespace moepd {
namespace {

constexpr int kFfnF32Rows = 64, kFfnF32Cols = 64, kFfnF32Depth = 16;

template <int SHARE = kRowsInBlocks>
__device__ __forceinline__ bool ffn_row_tile(const FfnArgs& g, int bm, int bn, FfnTile& t);
__device__ __forceinline__ bool ffn_weight_tile(const FfnArgs& g, int bm, int bn, FfnTile& t, int& split);

template <int KIND>
__device__ __forceinline__ void ffn_f32_tile(const FfnArgs& g, const FfnTile& t, float* c) {
  constexpr int BM = kFfnF32Rows, BN = kFfnF32Cols, BK = kFfnF32Depth, NB = KIND == kFfnGateUp ? 2 : 1;
  constexpr bool A_COL = KIND == kFfnWeightGrad, B_COL = KIND >= kFfnDownGrad;
  __shared__ float as[BK][BM + 4], bs[NB][BK][BN + 4];
  const int tid = threadIdx.x, tm = tid >> 4, tn = tid & 15;
  const long long lda = g.lda / 4, ldb = g.ldb / 4, ldc = g.ldc / 4;
  const int K = KIND == kFfnWeightGrad ? t.k_count : g.k;
  const float* a = reinterpret_cast<const float*>(g.a) + (A_COL ? t.k0 * lda + t.m0 : t.m0 * lda);
  const float* b = reinterpret_cast<const float*>(g.b + (KIND == kFfnWeightGrad ? 0 : t.group * g.b_group));
  if (KIND == kFfnWeightGrad) b += t.k0 * ldb;
  float acc[NB][4][4];
#pragma unroll
  for (int j = 0; j < NB; ++j)
#pragma unroll
    for (int x = 0; x < 4; ++x)
#pragma unroll
      for (int y = 0; y < 4; ++y) acc[j][x][y] = 0.f;
  for (int k0 = 0; k0 < K; k0 += BK) {
    for (int i = tid; i < BM * BK; i += 256) {
      const int p = A_COL ? i % BM : i / BK, k = A_COL ? i / BM : i % BK;
      const bool in = p < t.rows && k0 + k < K;
      as[k][p] = in ? a[A_COL ? (k0 + k) * lda + p : p * lda + k0 + k] : 0.f;
    }
    for (int i = tid; i < NB * BN * BK; i += 256) {
      const int j = i / (BN * BK), r = i % (BN * BK);
      const int p = B_COL ? r % BN : r / BK, k = B_COL ? r / BN : r % BK;
      const long long col = t.n0 + p + (long long)j * g.n;
      const bool in = t.n0 + p < g.n && k0 + k < K;
      bs[j][k][p] = in ? b[B_COL ? (k0 + k) * ldb + col : col * ldb + k0 + k] : 0.f;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < BK; ++k) {
      float av[4];
#pragma unroll
      for (int x = 0; x < 4; ++x) av[x] = as[k][4 * tm + x];
#pragma unroll
      for (int j = 0; j < NB; ++j)
#pragma unroll
        for (int y = 0; y < 4; ++y) {
          const float bv = bs[j][k][4 * tn + y];
#pragma unroll
          for (int x = 0; x < 4; ++x) acc[j][x][y] = __builtin_fmaf(av[x], bv, acc[j][x][y]);
        }
    }
    __syncthreads();
  }
#pragma unroll
  for (int x = 0; x < 4; ++x) {
    if (4 * tm + x >= t.rows) continue;
    const long long row = t.m0 + 4 * tm + x;
#pragma unroll
    for (int y = 0; y < 4; ++y) {
      const int col = t.n0 + 4 * tn + y;
      if (col >= g.n) continue;
      const float v = acc[0][x][y];
      if constexpr (KIND == kFfnGateUp) {
        const float up = acc[NB - 1][x][y];
        if (c) {
          c[row * 2 * g.n + col] = v;
          c[row * 2 * g.n + g.n + col] = up;
        }
        reinterpret_cast<float*>(g.h)[row * g.n + col] = swiglu_of<true>(v, up);
      } else if constexpr (KIND == kFfnDownGrad) {
        const float* gu = reinterpret_cast<const float*>(g.gu) + row * 2 * g.n + col;
        const float gate = gu[0], up = gu[g.n];
        float dg, du;
        swiglu_grad(gate, up, v, dg, du);
        c[row * 2 * g.n + col] = dg;
        c[row * 2 * g.n + g.n + col] = du;
        if (g.h) reinterpret_cast<float*>(g.h)[row * g.n + col] = swiglu_of<true>(gate, up);
      } else {
        float* p = c + row * ldc + col;
        *p = KIND == kFfnWeightGrad && g.accumulate ? *p + v : v;
      }
    }
  }
}

template <int KIND>
__global__ __launch_bounds__(256) void ffn_block_f32(FfnArgs g) {
  FfnTile t;
  if (!ffn_row_tile(g, kFfnF32Rows, kFfnF32Cols, t)) return;
  ffn_f32_tile<KIND>(g, t, reinterpret_cast<float*>(g.c));
}

__global__ __launch_bounds__(256) void ffn_block_f32_weights(FfnArgs g) {
  FfnTile t;
  int split;
  if (!ffn_weight_tile(g, kFfnF32Rows, kFfnF32Cols, t, split)) return;
  if (g.accumulate && t.k_count == 0) return;
  ffn_f32_tile<kFfnWeightGrad>(g, t, reinterpret_cast<float*>(g.c + ((long long)split * g.groups + t.group) * g.m * g.ldc));
}

}  // namespace
}  // namespace moepd
