// Products of MX FP4 matrices, dense or with one weight matrix per run of rows
// (include/moepd_mx4.h), on v_mfma_scale_f32_32x32x64_f8f6f4: 32 x 32 outputs
// and 64 values of K per instruction, float32 accumulation, block scales
// applied by the matrix core.  The weights are the first operand, so lane l ends
// with one row of `a` (l % 32) and 16 of its columns, 8 q + 4 (l / 32) + (0..3).
#include <type_traits>

#include "kernels.h"
#include "moepd_mx4.h"
#include "mx4.h"
#include "pipeline.h"
#include "tiles.h"

namespace moepd {

typedef int32_t v8i32_mx4 __attribute__((ext_vector_type(8)));
typedef float f32x16_mx4 __attribute__((ext_vector_type(16)));
typedef float f32x4_mx4 __attribute__((ext_vector_type(4)));

namespace {

struct Mx4Tile {  // wave-uniform
  int group;
  int m0, m_end;  // rows
  int nt;         // column tile
};

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ long long uniform(long long v) {
  return (long long)(((uint64_t)(uint32_t)uniform((int)(v >> 32)) << 32) | (uint32_t)uniform((int)v));
}

// Inclusive sum over the wave's lanes (register moves across lanes; see common.h).
template <int CTRL, int ROW_MASK>
__device__ __forceinline__ int dpp_plus(int v) {
  return v + __builtin_amdgcn_update_dpp(0, v, CTRL, ROW_MASK, 0xF, false);
}
__device__ __forceinline__ int wave_scan(int v) {
  v = dpp_plus<0x111, 0xF>(v);  // row_shr:1
  v = dpp_plus<0x112, 0xF>(v);  // row_shr:2
  v = dpp_plus<0x114, 0xF>(v);  // row_shr:4
  v = dpp_plus<0x118, 0xF>(v);  // row_shr:8
  v = dpp_plus<0x142, 0xA>(v);  // row_bcast:15
  return dpp_plus<0x143, 0xC>(v);  // row_bcast:31
}

// The tile of workgroup b, if any, found by each wave from the offsets: lane i
// holds group i's rows, and a scan of the groups' counts of row tiles (of at most bm
// rows) places the tile; with more than 64 groups, 64 at a time.
//
// STRIPED (streaming tiles): groups in order, within a group of mt row tiles column
// tile 8 q + b % 8 for each q, with all its row tiles in a row: workgroup b runs on
// XCD b % 8, so the row tiles that read one weight panel share an L2, and every XCD
// streams an eighth of every group's weights.
//
// Otherwise (ring tiles): a group's rows are shared evenly among its row tiles; its
// tiles run over blocks of four column tiles, in each row tile by row tile; and runs of
// consecutive tiles are dealt to the XCDs in turn, so that an XCD's L2 serves each row
// block to four workgroups and each weight panel to as many as the run has row
// tiles.  The last runs, when they do not go round, are dealt tile by tile.  Runs of 64 tiles
// (16 row x 4 column tiles: what an XCD's CUs hold at a time) for groups of many rows,
// else 32, which leave less to the last round: 96,889 skewed rows (7168 x 2048)
// 1030 us with 64, 1096 with 32; 32,768 rows 391 / 430; 8192 rows, 256 to a group, 77 / 73.
template <bool STRIPED>
__device__ __forceinline__ bool mx4_tile(const Mx4Args& g, int b, int bm, Mx4Tile& t) {
  const int lane = lane_id();
  int l = 0, h = 0, mt = 0, incl = 0;  // of group g0 + lane
  auto count = [&](int g0) {
    l = h = 0;
    const int e = g0 + lane;
    if (!g.offsets) {
      h = lane == 0 ? g.rows : 0;
    } else if (e < g.groups) {
      const int a = g.offsets[e], z = g.offsets[e + 1];
      l = min(max(a, 0), g.rows);
      h = max(l, min(z, g.rows));
    }
    mt = (int)((unsigned)(h - l + bm - 1) / (unsigned)bm);
    incl = wave_scan(mt);
    return __builtin_amdgcn_readlane(incl, 63);
  };
  int m_here = count(0);
  int L = b;
  if constexpr (!STRIPED) {
    int m_total = m_here;
    if (g.groups > kWave) {
      for (int g0 = kWave; g0 < g.groups; g0 += kWave) m_total += count(g0);
      m_here = count(0);
    }
    const int total = m_total * g.n_tiles;
    const int x = b & 7, slot = b >> 3, round = slot / g.run, base = round * 8 * g.run, j = slot - round * g.run;
    L = base + 8 * g.run <= total ? base + x * g.run + j : base + 8 * j + x;
    if (L >= total) return false;
  }
  int want = (int)((unsigned)L / (unsigned)g.n_tiles);  // row tiles before this one
  int at = L - want * g.n_tiles, g0 = 0;
  while (want >= m_here) {
    want -= m_here;
    g0 += kWave;
    if (g0 >= g.groups) return false;
    m_here = count(g0);
  }
  const uint64_t past = __ballot(incl > want);
  if (!past) return false;
  const int src = __builtin_ctzll(past);
  const int mt_e = __builtin_amdgcn_readlane(mt, src);
  const int lo = __builtin_amdgcn_readlane(l, src), hi = __builtin_amdgcn_readlane(h, src);
  at += (want - (__builtin_amdgcn_readlane(incl, src) - mt_e)) * g.n_tiles;  // within the group
  t.group = uniform(g0 + src);
  if constexpr (STRIPED) {
    const int j = at >> 3, q = j / mt_e;
    t.nt = uniform(8 * q + (at & 7));
    t.m0 = uniform(lo + (j - q * mt_e) * bm);
    t.m_end = uniform(min(t.m0 + bm, hi));
  } else {
    const int q = at / (4 * mt_e), r = at - q * 4 * mt_e;
    const int width = min(4, g.n_tiles - 4 * q);
    const int mi = r / width;
    t.nt = uniform(4 * q + r - mi * width);
    const int per = (hi - lo + mt_e - 1) / mt_e;
    t.m0 = uniform(lo + mi * per);
    t.m_end = uniform(min(t.m0 + per, hi));
  }
  return true;
}

__device__ __forceinline__ v8i32_mx4 widen(const u32x4& a) {
  return v8i32_mx4{(int32_t)a[0], (int32_t)a[1], (int32_t)a[2], (int32_t)a[3], 0, 0, 0, 0};
}

// Step S (64 of a slice's 256 values): both operands' scale words hold the four
// steps' scales, of which the instruction picks byte S.
template <int S>
__device__ __forceinline__ f32x16_mx4 mx4_mfma(const u32x4& w, const u32x4& a, const f32x16_mx4& acc, uint32_t sw,
                                               uint32_t sa) {
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(widen(w), widen(a), acc, 4, 4, S, (int)sw, S, (int)sa);
}

// silu(g) * u.  With q = e^-|g|, silu is g / (1 + q), times q where g is negative: q never
// overflows, and 1 + q is between 1 and 2.  q as 2^(t + lo): the product's rounding error and
// log2 e's own, lo, would otherwise cost |g| ulp; with it, and the hardware's 2^x and
// reciprocal (1 ulp each), the result is within a few ulp.  Far below zero q and g q pass
// below the normal numbers (which the hardware's 2^x flushes), at -87 and -92, while u may
// bring the result back: there q carries a factor of 2^64 that 1 + q leaves out and u gives
// back, good down to gates of -131.  Past 256 q is 0 in any case.
__device__ __forceinline__ float mx4_silu_mul(float g, float u) {
#pragma clang fp contract(off)  // t + 64 must start from the rounded t, whose error lo holds
  constexpr float kLog2e = 1.44269504f, kLog2eLow = 1.92596303e-8f, kLn2 = 0.693147181f;
  const float a = fminf(__builtin_fabsf(g), 256.f);
  const float t = -a * kLog2e;
  const float lo = __builtin_fmaf(-a, kLog2eLow, __builtin_fmaf(-a, kLog2e, -t));
  const bool deep = g < -44.f;
  const float k = deep ? 0x1p-64f : 1.f;
  const float e = __builtin_amdgcn_exp2f(t + (deep ? 64.f : 0.f));
  const float q = __builtin_fmaf(e, lo * kLn2, e);
  return (g < 0.f ? g * q : g) * __builtin_amdgcn_rcpf(__builtin_fmaf(q, k, 1.f)) * (u * k);
}

// Two values to bf16, nearest even, packed.
__device__ __forceinline__ uint32_t mx4_bf16_pair(float a, float b) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, bf16x2));
}

// Store one 32 x 32 block: lane (r, h) holds v[4 q + t] = column col0 + 8 q + 4 h + t of `row`.
// The lanes of a row's two halves both call this (fp4 exchanges between them).
template <int OUT>
__device__ __forceinline__ void mx4_store(const Mx4Args& g, const float (&v)[16], long long row, bool live, int col0,
                                          int h) {
  if constexpr (OUT == kMx4Fp4) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const uint32_t b = __float_as_uint(v[i]) & 0x7fffffffu;
      m = b > m ? b : m;
    }
    const uint32_t o = (uint32_t)__shfl_xor((int)m, 32, kWave);
    m = o > m ? o : m;
    const uint32_t byte = mx4_scale_byte(m);
    const uint32_t w0 = mx4_codes8({v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7]}, byte);
    const uint32_t w1 = mx4_codes8({v[8], v[9], v[10], v[11], v[12], v[13], v[14], v[15]}, byte);
    // this half's codes of quarter q are 16 bits; a quarter's word is (half 0, half 1)
    const uint32_t p0 = (uint32_t)__shfl_xor((int)w0, 32, kWave), p1 = (uint32_t)__shfl_xor((int)w1, 32, kWave);
    if (live && h == 0) {
      const int blocks = (g.n + kMx4Slice - 1) / kMx4Slice * 8;
      const long long rb = row >> 5;
      const int r = (int)(row & 31), b = col0 >> 5;
      store16(static_cast<uint8_t*>(g.c) + ((rb * blocks + b) * 32 + r) * 16,
              u32x4{(w0 & 0xffffu) | (p0 << 16), (w0 >> 16) | (p0 & 0xffff0000u), (w1 & 0xffffu) | (p1 << 16),
                    (w1 >> 16) | (p1 & 0xffff0000u)});
      g.cs[(rb * (blocks / 8) + (b >> 3)) * kMx4SliceScales + ((b & 1) * 32 + r) * 4 + ((b & 7) >> 1)] = (uint8_t)byte;
    }
  } else {
    if (!live) return;
    const long long at = row * g.ldc + col0 + 4 * h;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int col = col0 + 4 * h + 8 * q;
      if (col + 4 <= g.n) {
        if constexpr (OUT == kMx4F32) {
          *reinterpret_cast<u32x4_any*>(static_cast<float*>(g.c) + at + 8 * q) =
              u32x4_any{__float_as_uint(v[4 * q]), __float_as_uint(v[4 * q + 1]), __float_as_uint(v[4 * q + 2]),
                        __float_as_uint(v[4 * q + 3])};
        } else {
          typedef uint32_t u32x2 __attribute__((ext_vector_type(2), aligned(2)));
          *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(g.c) + at + 8 * q) =
              u32x2{mx4_bf16_pair(v[4 * q], v[4 * q + 1]), mx4_bf16_pair(v[4 * q + 2], v[4 * q + 3])};
        }
      } else {
#pragma unroll
        for (int t = 0; t < 4; ++t)
          if (col + t < g.n) {
            if constexpr (OUT == kMx4F32) static_cast<float*>(g.c)[at + 8 * q + t] = v[4 * q + t];
            else static_cast<uint16_t*>(g.c)[at + 8 * q + t] = f32_to_bf16(v[4 * q + t]);
          }
      }
    }
  }
}

// A lane's place in a run of rows of a held matrix: its code bytes and scale bytes
// from the block of the run's first row, or past every resource where the row does
// not count (kMx4Nowhere: such loads give zeros and touch no memory).
struct Mx4Lane {
  int codes, scales;
};
__device__ __forceinline__ Mx4Lane mx4_lane(long long first, int row, bool counts, int slices, int h) {
  const int rr = (int)(first & 31) + row;
  const int b = rr >> 5, r = rr & 31;
  return counts ? Mx4Lane{b * slices * kMx4SliceBytes + h * 512 + r * 16, b * slices * kMx4SliceScales + (h * 32 + r) * 4}
                : Mx4Lane{kMx4Nowhere, kMx4Nowhere};
}
// The resource of `rows` rows from `first` on, which starts at the block of the first.
// At least one block (of which no lane reads anything where there is no row), so that
// every slice's offset lies within it.
struct Mx4Span {
  void* base;
  int bytes;
  __device__ __forceinline__ __amdgpu_buffer_rsrc_t rsrc(int bytes) const {
    return __builtin_amdgcn_make_buffer_rsrc(base, (short)0, bytes, kBufferRsrcWord3);
  }
};
__device__ __forceinline__ Mx4Span mx4_span(const uint8_t* p, long long first, int rows, int slices, int unit) {
  const int blocks = rows > 0 ? ((int)(first & 31) + rows + 31) >> 5 : 1;
  return Mx4Span{(void*)uniform((long long)p + (first >> 5) * slices * unit), uniform(blocks * slices * unit)};
}
__device__ __forceinline__ u32x4 mx4_load(const __amdgpu_buffer_rsrc_t& rsrc, int lane_off, int off) {
  typedef uint32_t raw4 __attribute__((vector_size(16)));
  const raw4 v = __builtin_amdgcn_raw_buffer_load_b128(rsrc, lane_off, off, 0);
  return u32x4{v[0], v[1], v[2], v[3]};
}

// ------------------------------------------------------------------ streaming tile

// Few rows per group: what bounds the product is the stream of weights.  A wave
// takes up to 32 MB rows and two panels of 32 weight rows (gate and up, or 64
// columns; one panel where there are few tiles), each slice of a panel 4 KB of
// consecutive memory straight into registers, two slices in flight.  The waves of
// a workgroup share a tile and deal its slices among them; their sums meet in
// LDS and are added in wave order.  131 rows over 32 groups, 4096 x 7168: 85 us, 5.8 TB/s
// of weights; one row, 7168 x 2048 (8 MB): 4.6 us, the launch, the tile's place, one HBM
// latency and the join.
template <int MB, int NB>
struct Mx4Slice4 {
  u32x4 w[NB][4], a[MB][4];
  uint32_t sw[NB], sa[MB];
};

template <int MB, int NB, bool GATED, int OUT>
__device__ __forceinline__ void mx4_stream_tile(const Mx4Args& g, const Mx4Tile& t, float* lds) {
  const int lane = threadIdx.x & 63, r = lane & 31, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
  const int KT = g.slices;
  constexpr int BN = GATED ? 32 : 32 * NB;
  const int n0 = t.nt * BN;
  const long long w_first = (long long)t.group * (GATED ? 2 : 1) * g.n + n0;
  const int m_rows = t.m_end - t.m0;
  const Mx4Span a_span = mx4_span(g.a, t.m0, m_rows, KT, kMx4SliceBytes);
  const Mx4Span as_span = mx4_span(g.as, t.m0, m_rows, KT, kMx4SliceScales);
  Mx4Lane al[MB], wl[NB];
  Mx4Span w_span[NB], ws_span[NB];
#pragma unroll
  for (int m = 0; m < MB; ++m) al[m] = mx4_lane(t.m0, 32 * m + r, 32 * m + r < m_rows, KT, h);
#pragma unroll
  for (int j = 0; j < NB; ++j) {
    const long long first = GATED ? w_first + (j ? g.n : 0) : w_first + 32 * j;
    const int left = g.n - n0 - (GATED ? 0 : 32 * j);  // weight rows from the panel's first on
    const int rows = left < 0 ? 0 : left < 32 ? left : 32;
    wl[j] = mx4_lane(first, r, r < rows, KT, h);
    w_span[j] = mx4_span(g.w, first, rows, KT, kMx4SliceBytes);
    ws_span[j] = mx4_span(g.ws, first, rows, KT, kMx4SliceScales);
  }

  // A slice past the last one is the beginning of an empty resource: zeros, and no branch.
  auto load = [&](Mx4Slice4<MB, NB>& s, int kt) {
    const bool in = kt < KT;
    const int at = uniform(in ? kt : 0);
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      s.sw[j] = __builtin_amdgcn_raw_buffer_load_b32(ws_span[j].rsrc(in ? ws_span[j].bytes : 0), wl[j].scales,
                                                     at * kMx4SliceScales, 0);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        s.w[j][i] = mx4_load(w_span[j].rsrc(in ? w_span[j].bytes : 0), wl[j].codes + i * kMx4StepBytes, at * kMx4SliceBytes);
    }
#pragma unroll
    for (int m = 0; m < MB; ++m) {
      s.sa[m] = __builtin_amdgcn_raw_buffer_load_b32(as_span.rsrc(in ? as_span.bytes : 0), al[m].scales,
                                                     at * kMx4SliceScales, 0);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        s.a[m][i] = mx4_load(a_span.rsrc(in ? a_span.bytes : 0), al[m].codes + i * kMx4StepBytes, at * kMx4SliceBytes);
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  f32x16_mx4 acc[MB][NB];
#pragma unroll
  for (int m = 0; m < MB; ++m)
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
      for (int q = 0; q < 16; ++q) acc[m][j][q] = 0.f;
  auto multiply = [&](const Mx4Slice4<MB, NB>& s) {
    weave_run<0, 4>([&](auto i) {
      constexpr int S = decltype(i)::value;
#pragma unroll
      for (int m = 0; m < MB; ++m)
#pragma unroll
        for (int j = 0; j < NB; ++j) acc[m][j] = mx4_mfma<S>(s.w[j][S], s.a[m][S], acc[m][j], s.sw[j], s.sa[m]);
    });
    __builtin_amdgcn_sched_barrier(0);
  };
  // This wave's slices: wave, wave + waves, ...
  if (KT <= waves) {
    Mx4Slice4<MB, NB> s;
    load(s, wave);
    multiply(s);
  } else {
    Mx4Slice4<MB, NB> s0, s1;
    int kt = wave;
    load(s0, kt);
    load(s1, kt + waves);
    for (; kt + 2 * waves < KT; kt += 2 * waves) {
      multiply(s0);
      load(s0, kt + 2 * waves);
      multiply(s1);
      load(s1, kt + 3 * waves);
    }
    multiply(s0);
    multiply(s1);
  }

  if (waves > 1) {
    f32x4_mx4* sums = reinterpret_cast<f32x4_mx4*>(lds);
#pragma unroll
    for (int m = 0; m < MB; ++m)
#pragma unroll
      for (int j = 0; j < NB; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          sums[((wave * MB + m) * NB + j) * 256 + q * 64 + lane] =
              f32x4_mx4{acc[m][j][4 * q], acc[m][j][4 * q + 1], acc[m][j][4 * q + 2], acc[m][j][4 * q + 3]};
    __syncthreads();
    if (wave) return;
#pragma unroll
    for (int m = 0; m < MB; ++m)
#pragma unroll
      for (int j = 0; j < NB; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          for (int w = 1; w < waves; ++w) {
            const f32x4_mx4 o = sums[((w * MB + m) * NB + j) * 256 + q * 64 + lane];
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[m][j][4 * q + i] += o[i];
          }
  }
#pragma unroll
  for (int m = 0; m < MB; ++m) {
    const int row = t.m0 + 32 * m + r;
    const bool live = row < t.m_end;
    float v[16];
    if constexpr (GATED) {
#pragma unroll
      for (int i = 0; i < 16; ++i) v[i] = mx4_silu_mul(acc[m][0][i], acc[m][NB - 1][i]);
      mx4_store<OUT>(g, v, row, live, n0, h);
    } else {
#pragma unroll
      for (int j = 0; j < NB; ++j) {
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = acc[m][j][i];
        mx4_store<OUT>(g, v, row, live, n0 + 32 * j, h);
      }
    }
  }
}

// Tiles of up to 32 MAXB rows: 32 where groups are expected to have few rows, since without
// the 64-row body the kernel takes registers for three waves to a SIMD instead of two.
template <int MAXB, int NB, bool GATED, int OUT>
__global__ __launch_bounds__(64 * kStreamWaves, MAXB == 2 ? 2 : NB == 2 ? 3 : 4) void mx4_stream_kernel(
    Mx4Args g) {
  extern __shared__ __align__(16) float lds[];
  Mx4Tile t;
  if (!mx4_tile<true>(g, (int)(blockIdx.y * gridDim.x + blockIdx.x), 32 * MAXB, t)) return;
  if (t.nt * (GATED ? 32 : 32 * NB) >= (OUT == kMx4Fp4 ? (g.n + kMx4Slice - 1) / kMx4Slice * kMx4Slice : g.n)) return;
  if constexpr (MAXB == 1) {
    mx4_stream_tile<1, NB, GATED, OUT>(g, t, lds);
  } else {
    if (t.m_end - t.m0 <= 32) mx4_stream_tile<1, NB, GATED, OUT>(g, t, lds);
    else mx4_stream_tile<2, NB, GATED, OUT>(g, t, lds);
  }
}

// 32 rows x COLS columns of results in LDS, on their way from the lanes that hold 4
// columns of a row to lanes that store 16 bytes side by side: a wave's store then
// covers whole 64-byte pieces of its rows, where straight from the registers it would
// touch 32 rows with 16 (bf16) or 32 bytes each, and the L2's request rate bounded the
// epilogue (it took 16,000 cycles of a 128 x 256 bf16 tile's 53,000).  Rows are 16 bytes
// apart beyond their width, so that neither side conflicts on banks.
template <int OUT, int COLS>
struct Mx4Patch {
  static constexpr int esz = OUT == kMx4F32 ? 4 : 2;
  static constexpr int pitch = COLS * esz + 16;
  static constexpr int bytes = OUT == kMx4Fp4 ? 0 : 32 * pitch;
  typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

  static __device__ __forceinline__ void put(uint8_t* part, const float (&v)[16], int col, int r, int h) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      uint8_t* p = part + r * pitch + (col + 8 * q + 4 * h) * esz;
      if constexpr (OUT == kMx4F32)
        *reinterpret_cast<f32x4_mx4*>(p) = f32x4_mx4{v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]};
      else
        *reinterpret_cast<u32x2*>(p) = u32x2{mx4_bf16_pair(v[4 * q], v[4 * q + 1]), mx4_bf16_pair(v[4 * q + 2], v[4 * q + 3])};
    }
  }

  // The first `rows` rows, from row `row` and column `col0` on, in the order in which
  // the wave wrote them (its LDS operations complete in order).
  static __device__ __forceinline__ void store(const Mx4Args& g, const uint8_t* part, int row, int rows, int col0,
                                               int lane) {
    __builtin_amdgcn_wave_barrier();
    constexpr int per_row = COLS * esz / 16, at_once = 64 / per_row, each = 16 / esz;
    const int col = col0 + lane % per_row * each;
#pragma unroll
    for (int i = 0; i < 32 / at_once; ++i) {
      const int rr = i * at_once + lane / per_row;
      const u32x4 q = *reinterpret_cast<const u32x4*>(part + rr * pitch + lane % per_row * 16);
      if (rr >= rows) continue;
      uint8_t* o = static_cast<uint8_t*>(g.c) + ((long long)(row + rr) * g.ldc + col) * esz;
      if (col + each <= g.n) {
        // past the caches' keeping: 8192 rows x 7168 bf16 100 -> 87 us, 96,889 rows float32 1164 -> 1088 us
        __builtin_nontemporal_store(u32x4_any(q), reinterpret_cast<u32x4_any*>(o));
      } else {
#pragma unroll
        for (int e = 0; e < each; ++e)
          if (col + e < g.n) {
            if constexpr (OUT == kMx4F32) reinterpret_cast<uint32_t*>(o)[e] = q[e];
            else reinterpret_cast<uint16_t*>(o)[e] = (uint16_t)(q[e / 2] >> (16 * (e & 1)));
          }
      }
    }
    __builtin_amdgcn_wave_barrier();
  }
};

// ------------------------------------------------------------------ ring tile

// Many rows per group: four waves side by side along the weights.  Each wave
// takes all 32 MB rows of the tile and two panels of 32 weight rows (gate and
// up, or 64 columns).  No two waves use the same weights, so these go straight
// into registers; the rows of `a`, which all four read, travel by DMA into a
// ring of SA slots of one slice (256 values) each, where one operand of one MFMA is
// 1 KB in a row.  With 128 rows that is, for the 256 cycles of a step's 8 MFMAs per
// SIMD, 16 KB of LDS reads (half the LDS's rate) and 12 KB from L2.  8192 x 8192 x
// 8192: 250 us, 4.4 PFLOP/s, where MFMAs on random codes alone, from registers, hold
// 6.0 to 6.5 (9.7 on zeros: the power limit).  With K 2048 a tile's start and end take
// as long as its slices, and float32 results 12 bytes of HBM writes a cycle and CU:
// 96,889 rows, 7168 x 2048, 980 us, 2.9 PFLOP/s and 2.8 TB/s of results.
//
// A slice is four steps of 64 values.  Step s multiplies while the next step's
// operands come from LDS; the registers of its weights are then free, and the
// weights of step s two slices on are requested into them during step s + 1 (those of
// step 3, and the scales, during the next slice's step 0).  The slice's barrier
// stands before step 3, when every wave holds the last operands of the slice: its
// slot is free for slice kt + SA, and slice kt + 1, which each wave has waited for,
// is complete.  Requests past the last slice go to an empty resource: they move
// no memory, and every slice has the same instructions, so the counted waits are exact
// throughout.
template <int MB, int SA, bool GATED, int OUT>
__device__ __forceinline__ void mx4_ring_tile(const Mx4Args& g, const Mx4Tile& t, u32x4* lds) {
  constexpr int kSlot = MB * 256;  // 16-byte units
  static_assert(SA >= 3, "the wait below counts whole slices between a slot's request and its use");
  const int lane = threadIdx.x & 63, r = lane & 31, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int KT = g.slices;
  const int n0 = t.nt * (GATED ? 128 : 256) + wave * (GATED ? 32 : 64);
  const int group = t.group;
  const int m0 = t.m0;
  const int m_rows = t.m_end - t.m0;
  const Mx4Span a_span = mx4_span(g.a, m0, m_rows, KT, kMx4SliceBytes);
  const Mx4Span as_span = mx4_span(g.as, m0, m_rows, KT, kMx4SliceScales);
  Mx4Span w_span[2], ws_span[2];
  // Row block b is MB - 1 blocks at most past the first; only the last one may be cut short.
  Mx4Lane full = mx4_lane(m0, r, true, KT, h), cut = mx4_lane(m0, r, 32 * (MB - 1) + r < m_rows, KT, h);
  full.codes += wave * kMx4StepBytes;  // of a slice of `a`, this wave moves step `wave`
  cut.codes += wave * kMx4StepBytes;
  Mx4Lane wl[2];
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const long long first = (long long)group * (GATED ? 2 : 1) * g.n + n0 + (GATED ? j * g.n : 32 * j);
    const int left = g.n - n0 - (GATED ? 0 : 32 * j);
    const int rows = left < 0 ? 0 : left < 32 ? left : 32;
    wl[j] = mx4_lane(first, r, r < rows, KT, h);
    w_span[j] = mx4_span(g.w, first, rows, KT, kMx4SliceBytes);
    ws_span[j] = mx4_span(g.ws, first, rows, KT, kMx4SliceScales);
  }

  u32x4 wf[2][2][4];  // [slice parity][panel][step]
  uint32_t sw[2][2], sa[2][MB];
  u32x4 af[2][MB];  // [step parity]
  f32x16_mx4 acc[MB][2];

  // What the requests of `a` and the loads of weights and scales name now: a slice's place, and
  // all of a resource; past the last slice its beginning, and nothing of it.  (All of it in
  // scalar registers: the lane offsets, which the resource's length checks, stay the same.)
  int a_slice, w_slice;
  bool a_in, w_in;
  auto aim_a = [&](int kt) {
    a_in = kt < KT;
    a_slice = uniform(a_in ? kt : 0);
  };
  auto aim_w = [&](int kt) {
    w_in = kt < KT;
    w_slice = uniform(w_in ? kt : 0);
  };
  auto request_a = [&](int b, int slot) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(a_span.rsrc(a_in ? a_span.bytes : 0),
                                             MOEPD_LPTR(lds + slot * kSlot + (b * 4 + wave) * 64), 16,
                                             (b == MB - 1 ? cut.codes : full.codes) + b * KT * kMx4SliceBytes,
                                             a_slice * kMx4SliceBytes, 0, 0);
  };
  auto load_w = [&](int j, int s, int p) {
    wf[p][j][s] = mx4_load(w_span[j].rsrc(w_in ? w_span[j].bytes : 0), wl[j].codes + s * kMx4StepBytes, w_slice * kMx4SliceBytes);
  };
  auto load_sw = [&](int j, int p) {
    sw[p][j] = __builtin_amdgcn_raw_buffer_load_b32(ws_span[j].rsrc(w_in ? ws_span[j].bytes : 0), wl[j].scales,
                                                    w_slice * kMx4SliceScales, 0);
  };
  auto load_sa = [&](int b, int p) {
    sa[p][b] = __builtin_amdgcn_raw_buffer_load_b32(as_span.rsrc(w_in ? as_span.bytes : 0),
                                                    (b == MB - 1 ? cut.scales : full.scales) + b * KT * kMx4SliceScales,
                                                    w_slice * kMx4SliceScales, 0);
  };

  // In program order: the waits count requests.
#pragma unroll
  for (int st = 0; st < SA; ++st) {
    aim_a(st);
#pragma unroll
    for (int b = 0; b < MB; ++b) request_a(b, st);
    __builtin_amdgcn_sched_barrier(0);
  }
  aim_w(0);
#pragma unroll
  for (int j = 0; j < 2; ++j) load_sw(j, 0);
#pragma unroll
  for (int b = 0; b < MB; ++b) load_sa(b, 0);
#pragma unroll
  for (int s = 0; s < 4; ++s)
#pragma unroll
    for (int j = 0; j < 2; ++j) load_w(j, s, 0);
  __builtin_amdgcn_sched_barrier(0);
  aim_w(1);
#pragma unroll
  for (int s = 0; s < 3; ++s)
#pragma unroll
    for (int j = 0; j < 2; ++j) load_w(j, s, 1);
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int m = 0; m < MB; ++m)
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int q = 0; q < 16; ++q) acc[m][j][q] = 0.f;

  constexpr int kPrologue = (SA - 1) * MB + 16 + MB;
  wait_vmcnt_lgkm0<(kPrologue < 63 ? kPrologue : 63)>();
  bare_barrier();
#pragma unroll
  for (int b = 0; b < MB; ++b) af[0][b] = lds[b * 256 + lane];

  int slot = 0;
  auto slice = [&](auto parity, int kt) {
    constexpr int P = decltype(parity)::value, Q = P ^ 1;
    const u32x4* here = lds + slot * kSlot + lane;
    const int next = slot + 1 == SA ? 0 : slot + 1;
    const u32x4* there = lds + next * kSlot + lane;
    auto mul = [&](auto step) {
      constexpr int S = decltype(step)::value;
      return [&](auto i) {
        constexpr int m = decltype(i)::value / 2, j = decltype(i)::value % 2;
        acc[m][j] = mx4_mfma<S>(wf[P][j][S], af[S & 1][m], acc[m][j], sw[P][j], sa[P][m]);
      };
    };
    using C0 = std::integral_constant<int, 0>;
    using C1 = std::integral_constant<int, 1>;
    using C2 = std::integral_constant<int, 2>;
    using C3 = std::integral_constant<int, 3>;
    aim_w(kt + 1);  // as the last slice left it: not carried over, where it would take a vector register
    weave<2 * MB, MB, 4 + MB>(mul(C0{}), [&](auto b) { af[1][b] = here[(b * 4 + 1) * 64]; },
                              [&](auto i) {
                                if constexpr (i < 2) load_w(i, 3, Q);
                                else if constexpr (i < 4) load_sw(i - 2, Q);
                                else load_sa(i - 4, Q);
                              });
    aim_w(kt + 2);
    weave<2 * MB, MB, 2>(mul(C1{}), [&](auto b) { af[0][b] = here[(b * 4 + 2) * 64]; },
                         [&](auto j) { load_w(j, 0, P); });
    weave<2 * MB, MB, 2>(mul(C2{}), [&](auto b) { af[1][b] = here[(b * 4 + 3) * 64]; },
                         [&](auto j) { load_w(j, 1, P); });
    // requests younger than slice kt + 1 of `a`: all of SA - 2 slices and this one's so far
    constexpr int kYounger = (SA - 2) * (10 + 2 * MB) + 8 + MB;
    wait_vmcnt_lgkm0<(kYounger < 63 ? kYounger : 63)>();
    bare_barrier();
    aim_a(kt + SA);
    weave<2 * MB, MB, 2 + MB>(mul(C3{}), [&](auto b) { af[0][b] = there[b * 256]; },
                              [&](auto i) {
                                if constexpr (i < 2) load_w(i, 2, P);
                                else request_a(i - 2, slot);
                              });
    slot = next;
  };
  int kt = 0;
  for (; kt + 1 < KT; kt += 2) {
    slice(std::integral_constant<int, 0>{}, kt);
    slice(std::integral_constant<int, 1>{}, kt + 1);
  }
  if (kt < KT) slice(std::integral_constant<int, 0>{}, kt);

  // The ring is free once every wave has left its last slice (whose requests past the
  // end still write zeros to it): the waves pass their results through it, each in a part
  // of its own, to store whole lines.
  wait_vmcnt_lgkm0<0>();
  bare_barrier();
  constexpr int COLS = GATED ? 32 : 64;
  uint8_t* part = reinterpret_cast<uint8_t*>(lds) + wave * Mx4Patch<OUT, COLS>::bytes;
#pragma unroll
  for (int m = 0; m < MB; ++m) {
    float v[16];
    if constexpr (GATED) {
#pragma unroll
      for (int i = 0; i < 16; ++i) v[i] = mx4_silu_mul(acc[m][0][i], acc[m][1][i]);
      if constexpr (OUT == kMx4Fp4) mx4_store<OUT>(g, v, m0 + 32 * m + r, 32 * m + r < m_rows, n0, h);
      else Mx4Patch<OUT, COLS>::put(part, v, 0, r, h);
    } else {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = acc[m][j][i];
        Mx4Patch<OUT, COLS>::put(part, v, 32 * j, r, h);
      }
    }
    if constexpr (OUT != kMx4Fp4) Mx4Patch<OUT, COLS>::store(g, part, m0 + 32 * m, m_rows - 32 * m, n0, lane);
  }
}

// Tiles of up to 128 rows, cut to the 32-row blocks that they hold.  Two workgroups
// share a CU: one's start and end, which take as long as eight slices, run beside the
// other's slices (256-row tiles, one to a CU, took 150 us where these take 103: 8192 rows
// over 32 groups, 7168 x 2048).
template <bool GATED, int OUT>
__global__ __launch_bounds__(256, 2) void mx4_ring_kernel(Mx4Args g) {
  constexpr int ring = kRingSlots * kRingBlocks * 256, parts = 4 * Mx4Patch<OUT, GATED ? 32 : 64>::bytes / 16;
  __shared__ u32x4 lds[ring > parts ? ring : parts];
  Mx4Tile t;
  if (!mx4_tile<false>(g, (int)(blockIdx.y * gridDim.x + blockIdx.x), 32 * kRingBlocks, t)) return;
  const int blocks = (t.m_end - t.m0 + 31) / 32;
  if (blocks <= 0) return;  // fewer rows than tiles: an even share of none
  weave_run<1, kRingBlocks + 1>([&](auto mb) {
    constexpr int MB = decltype(mb)::value;
    if (blocks == MB) mx4_ring_tile<MB, kRingSlots, GATED, OUT>(g, t, lds);
  });
}

}  // namespace

hipError_t launch_mx4_gemm(Mx4Args g, bool gated, int out, long long expect, hipStream_t s) {
  const long long width = out == kMx4Fp4 ? (g.n + kMx4Slice - 1) / kMx4Slice * kMx4Slice : g.n;
  const Mx4Form f = mx4_form(gated, width, g.rows, g.groups, g.slices, expect < 1 ? 1 : expect < g.rows ? expect : g.rows);
  if (!f.fits()) return hipErrorInvalidValue;
  g.n_tiles = f.n_tiles;
  g.run = f.run;
  auto launch = [&](auto kernel) {
    kernel<<<grid_of(f.groups, f.threads()), f.threads(), f.lds(), s>>>(g);
    return hipGetLastError();
  };
  auto go = [&](auto gate, auto kind) {
    constexpr bool GATED = decltype(gate)::value;
    constexpr int OUT = decltype(kind)::value;
    if (f.ring) return launch(mx4_ring_kernel<GATED, OUT>);
    if constexpr (!GATED) {
      if (f.panels == 1) return f.blocks == 2 ? launch(mx4_stream_kernel<2, 1, false, OUT>) : launch(mx4_stream_kernel<1, 1, false, OUT>);
    }
    return f.blocks == 2 ? launch(mx4_stream_kernel<2, 2, GATED, OUT>) : launch(mx4_stream_kernel<1, 2, GATED, OUT>);
  };
  using Plain = std::false_type;
  using Gated = std::true_type;
  using F32 = std::integral_constant<int, kMx4F32>;
  using Bf16 = std::integral_constant<int, kMx4Bf16>;
  using Fp4 = std::integral_constant<int, kMx4Fp4>;
  if (gated) return out == kMx4Fp4 ? go(Gated{}, Fp4{}) : out == kMx4Bf16 ? go(Gated{}, Bf16{}) : go(Gated{}, F32{});
  return out == kMx4Bf16 ? go(Plain{}, Bf16{}) : go(Plain{}, F32{});
}

}  // namespace moepd

using namespace moepd;

namespace {

bool aligned(const void* p, size_t a) { return (uintptr_t)p % a == 0; }

int product(const uint8_t* a, const uint8_t* a_scales, int64_t rows, const uint8_t* w, const uint8_t* w_scales,
            int32_t groups, const int32_t* offsets, int32_t n, int32_t k, void* out, uint8_t* out_scales,
            int32_t out_dtype, int64_t out_stride, bool gated, hipStream_t stream) {
  if (!stream || rows < 0 || rows > (1LL << 31) - 32 || n < 1 || n > MOE_MX4_MAX_COLS || k < 1 || k > MOE_MX4_MAX_COLS ||
      groups < 1 || groups > MOE_MX4_MAX_GROUPS || (!offsets && groups != 1))
    return MOE_ERR_INVALID_ARG;
  const bool fp4 = gated && out_dtype == MOE_DTYPE_FP4;
  if (!fp4 && out_dtype != MOE_DTYPE_F32 && out_dtype != MOE_DTYPE_BF16) return MOE_ERR_INVALID_ARG;
  if (fp4 ? (n % 32 != 0 || out_stride != 0) : out_scales != nullptr) return MOE_ERR_INVALID_ARG;
  if (out_stride == 0) out_stride = n;
  if (out_stride < n) return MOE_ERR_INVALID_ARG;
  if (rows == 0) return MOE_OK;
  const int esz = out_dtype == MOE_DTYPE_F32 ? 4 : 2;
  if (!a || !a_scales || !w || !w_scales || !out || (fp4 && !out_scales)) return MOE_ERR_INVALID_ARG;
  if (!aligned(a, 16) || !aligned(a_scales, 16) || !aligned(w, 16) || !aligned(w_scales, 16) || !aligned(offsets, 4) ||
      !aligned(out, fp4 ? 16 : esz) || !aligned(out_scales, 16))
    return MOE_ERR_INVALID_ARG;
  Mx4Args g{};
  g.a = a;
  g.as = a_scales;
  g.w = w;
  g.ws = w_scales;
  g.c = out;
  g.cs = out_scales;
  g.offsets = offsets;
  g.rows = (int)rows;
  g.ldc = out_stride;
  g.groups = groups;
  g.n = n;
  g.slices = mx4_slices(k);
  const int kind = fp4 ? kMx4Fp4 : out_dtype == MOE_DTYPE_BF16 ? kMx4Bf16 : kMx4F32;
  const hipError_t st = launch_mx4_gemm(g, gated, kind, rows, stream);
  return st == hipSuccess ? MOE_OK : st == hipErrorInvalidValue ? MOE_ERR_INVALID_ARG : MOE_ERR_HIP;
}

}  // namespace

extern "C" {

int moe_mx4_gemm(const uint8_t* a, const uint8_t* a_scales, int64_t rows, const uint8_t* w, const uint8_t* w_scales,
                 int32_t groups, const int32_t* offsets, int32_t n, int32_t k, void* out, int32_t out_dtype,
                 int64_t out_stride, hipStream_t stream) {
  return product(a, a_scales, rows, w, w_scales, groups, offsets, n, k, out, nullptr, out_dtype, out_stride, false,
                 stream);
}

int moe_mx4_gemm_swiglu(const uint8_t* a, const uint8_t* a_scales, int64_t rows, const uint8_t* w,
                        const uint8_t* w_scales, int32_t groups, const int32_t* offsets, int32_t n, int32_t k,
                        void* out, uint8_t* out_scales, int32_t out_dtype, int64_t out_stride, hipStream_t stream) {
  return product(a, a_scales, rows, w, w_scales, groups, offsets, n, k, out, out_scales, out_dtype, out_stride, true,
                 stream);
}

}  // extern "C"
