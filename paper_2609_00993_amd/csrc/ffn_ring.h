// One tile of a bf16 product on the matrix cores, for the gated feed-forward block
// and its backward pass: c[m][n] = sum_k a[m][k] b[n][k], each operand in memory either
// by rows (k runs along a row) or by columns (row k holds the values of all m or n).
//
//   gate/up       a = x by rows,         b = w_gate_up by rows, gate and up rows together
//   down          a = h by rows,         b = w_down by rows
//   down grad     a = dy by rows,        b = w_down by columns (k = H)
//   gate/up grad  a = dgate_up by rows,  b = w_gate_up by columns (k = 2I)
//   weights' grad a, b by columns (k = the group's rows)
//
// A slice is BK (32 or 64) of K.  Slices travel HBM -> LDS by 16-byte DMA into rings, and the
// 32x32x16 MFMA's operands (lane l: row l % 32, 8 values of k from 8 (l / 32) on) are read
// from there: by rows with one ds_read_b128, whose 16-byte chunks are swizzled by the row
// (swz in pipeline.h); by columns with two ds_read_b64_tr_b16, each of which gives a
// group of 16 lanes the transpose of 4 rows x 16 columns, so no operand is ever transposed
// in memory.  There, 64-byte pieces of row k are swizzled by k % 4, so that the 32 lanes
// served together take 4 rows x 64 bytes from all 64 banks.  The DMA applies either
// swizzle on the global side.
//
// Rows and values of k past the operands' ends come as zeros from the buffer resource's
// bounds, with no memory request; columns past n may come as anything in the buffers and
// feed results that are not stored.
//
// The ring, its waits, and the order of each step's instructions are those of the
// grouped GEMMs in ffn_bf16.hip (gemm_ring_body): see there.
#pragma once

#include "ffn_form.h"
#include "group_tile.h"
#include "pipeline.h"
#include "swiglu.h"

namespace moepd {

typedef __bf16 bf16x8_ffn __attribute__((ext_vector_type(8)));
typedef short i16x4_ffn __attribute__((ext_vector_type(4)));
typedef short i16x8_ffn __attribute__((ext_vector_type(8)));
typedef float f32x16_ffn __attribute__((ext_vector_type(16)));
typedef float f32x4_ffn __attribute__((ext_vector_type(4)));

struct FfnArgs {
  const uint8_t* a;
  const uint8_t* b;
  uint8_t* c;         // result; gate/up: gate_up or null; down grad: dgate_up
  uint8_t* h;         // gate/up: h; down grad: h or null
  const uint8_t* gu;  // down grad: the kept gate_up
  long long lda, ldb, ldc;  // bytes from row to row
  long long b_group;        // bytes from one group's weights to the next
  const int32_t* offsets;   // null: one group of all rows
  int rows;
  int groups;
  int n;           // columns of the result (gate/up, down grad: I)
  int k;           // by rows: values of a row
  int m;           // weights' grad: rows of the result
  int n_tiles;     // column tiles; set by the launcher
  int m_tiles;     // weights' grad: row tiles; set by the launcher
  int bm;          // rows of a tile at most; set by the launcher
  int run;         // consecutive tiles that go to one XCD; set by the launcher
  int splits;      // weights' grad: parts of a group's rows, each with a result of its own
  int accumulate;  // weights' grad: add to c
};

struct FfnTile {  // wave-uniform
  int group;
  int m0, rows;     // first row of the result in this group's part of it, and how many (at most the tile's)
  int n0;
  int k0, k_count;  // weights' grad: rows of a and b
};

__device__ __forceinline__ bf16x8_ffn as_bf16x8_ffn(const u32x4& u) { return __builtin_bit_cast(bf16x8_ffn, u); }

constexpr int kFfnNowhere = 1 << 30;  // past every resource: bytes of an operand panel stay below it

// Four rows x 16 columns per 16 lanes, transposed: lane i gives row i / 4, columns 4 (i % 4)
// .. + 3, and gets column i of the four rows.  The pointer is restrict so that the read
// carries an alias scope: without one the compiler, which sees no difference between the
// ring's slots, waits for every DMA in flight before each read (the counted waits and
// barriers of the ring order them).
typedef __attribute__((address_space(3))) i16x4_ffn* ffn_lds_ptr;
__device__ __forceinline__ i16x4_ffn ffn_read_tr(ffn_lds_ptr __restrict__ at) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16(at);
}

// One operand's part of a slice in LDS: P rows of BK values, or BK rows of P values.
// Moved by SHARE waves.
template <bool COL, int P, int BK, int SHARE = 4>
struct FfnPanel {
  static constexpr int CPR = COL ? P / 8 : BK / 8;  // 16-byte chunks of an LDS row
  static constexpr int RPI = 64 / CPR;              // LDS rows of one DMA instruction (1 KB)
  static constexpr int CH = P * BK / 8;             // chunks of a slice
  static constexpr int INS = (CH / 64 + SHARE - 1) / SHARE;  // DMA instructions of a wave and slice
  static_assert(CH % 64 == 0 && (!COL || P == 64 || P == 128 || P == 256), "whole instructions");
  // By columns: the 64-byte pieces of row k are swizzled by this (a row of 128 bytes has two).
  static __device__ __forceinline__ int twist(int k) { return P == 64 ? (k >> 1) & 1 : k & 3; }

  uint8_t* base;  // by rows: of the panel's first row; by columns: of row 0, at the panel's first column
  long long ld;
  int bytes;      // by rows: of the resource
  int left;       // by columns: rows of k from row 0 on
  int width;      // by columns: bytes of a row that count
  int tail;       // by rows: bit i: this lane's chunk of instruction i is past K in the last slice
  int off[INS];   // this lane's byte of instruction i

  // The waves take the slice's instructions in turn; where these do not go round, the last ones
  // are issued twice (the same bytes to the same place), so that every wave counts alike.
  static __device__ __forceinline__ int instruction(int i, int wave) {
    const int n = SHARE * i + wave;
    if constexpr (CH / 64 % SHARE == 0) return n;
    return n < CH / 64 ? n : n - CH / 64 % SHARE;
  }
  // row_of(r): the panel's row r in the resource that starts at `first`.
  template <class F>
  __device__ __forceinline__ void by_rows(const uint8_t* first, long long stride, int nbytes, int k, int wave, int lane,
                                          F&& row_of) {
    base = (uint8_t*)uniform((long long)first);
    ld = stride;
    bytes = uniform(nbytes);
    tail = 0;
    const int last = (k - 1) / BK * BK;
#pragma unroll
    for (int i = 0; i < INS; ++i) {
      const int r = instruction(i, wave) * RPI + lane / CPR;
      const int chunk = (lane % CPR) ^ swz<BK>(r);
      off[i] = row_of(r) * (int)stride + chunk * 16;
      tail |= (last + 8 * chunk >= k ? 1 : 0) << i;
    }
  }
  __device__ __forceinline__ void by_columns(const uint8_t* first, long long stride, int rows, int columns, int wave,
                                             int lane) {
    base = (uint8_t*)uniform((long long)first);
    ld = stride;
    left = uniform(rows);
    width = uniform(columns * 2);
#pragma unroll
    for (int i = 0; i < INS; ++i) {
      const int r = instruction(i, wave) * RPI + lane / CPR;
      off[i] = r * (int)stride + ((lane % CPR) ^ (4 * twist(r))) * 16;
    }
  }
  __device__ __forceinline__ void issue(int i, int kt, bool last, u32x4* slot, int wave) const {
    u32x4* dst = slot + instruction(i, wave) * 64;
    if constexpr (COL) {
      // a resource of the slice's rows: past them, and past the last one's columns, zeros
      const int n = (min(left - kt * BK, BK) - 1) * (int)ld + width;
      const __amdgpu_buffer_rsrc_t rsrc =
          __builtin_amdgcn_make_buffer_rsrc(base + (long long)kt * BK * ld, (short)0, n, kBufferRsrcWord3);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, MOEPD_LPTR(dst), 16, off[i], 0, 0, 0);
    } else {
      const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc(base, (short)0, bytes, kBufferRsrcWord3);
      const int past = ((tail & -(int)last) >> i) & 1;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, MOEPD_LPTR(dst), 16, off[i] | past * kFfnNowhere, kt * (2 * BK), 0, 0);
    }
  }
  // The MFMA operand of 32 rows from row `p` (a multiple of 32) on, substep `sub` (16 of k).
  static __device__ __forceinline__ bf16x8_ffn read(const u32x4* slot, int p, int sub, int lane) {
    if constexpr (COL) {
      const int g = lane >> 4, i = lane & 15;
      const uint8_t* at = reinterpret_cast<const uint8_t*>(slot) + (8 * (g >> 1) + (i >> 2)) * (P * 2) +
                          ((p / 32) ^ twist(i >> 2)) * 64 + 32 * (g & 1) + 8 * (i & 3) + sub * (16 * P * 2);
      const i16x4_ffn lo = ffn_read_tr((ffn_lds_ptr)(at));
      const i16x4_ffn hi = ffn_read_tr((ffn_lds_ptr)(at + 4 * P * 2));
      return __builtin_bit_cast(bf16x8_ffn, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    } else {
      const int r = p + (lane & (P < 32 ? P - 1 : 31));
      return as_bf16x8_ffn(slot[r * CPR + ((2 * sub + (lane >> 5)) ^ swz<BK>(r))]);
    }
  }
};

// Eight values of a row, from column `col` on, to bf16 or float32.
__device__ __forceinline__ u32x4 ffn_bf16x8(const float (&v)[8]) {
  return u32x4{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7])};
}
__device__ __forceinline__ void ffn_unpack8(const u32x4& q, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(q[i] << 16);
    v[2 * i + 1] = __uint_as_float(q[i] & 0xffff0000u);
  }
}

__device__ __forceinline__ void ffn_store16(uint8_t* p, const u32x4& v) {
  __builtin_nontemporal_store(v, reinterpret_cast<u32x4*>(p));
}

// What 8 neighbouring results of one row become: load() what has to be read for them (issued ahead of
// their way through LDS), store() the rest.
template <int KIND, bool F32>
struct FfnStore {
  struct Old {
    u32x4 q[KIND == kFfnDownGrad || (KIND == kFfnWeightGrad && F32) ? 2 : 1];
  };
  static __device__ __forceinline__ void load(const FfnArgs& g, const FfnTile& t, uint8_t* c, int row, int col, Old& o) {
    if constexpr (KIND == kFfnDownGrad) {
      const uint8_t* p = g.gu + (long long)(t.m0 + row) * 4 * g.n + 2 * col;
      o.q[0] = load16(p);
      o.q[1] = load16(p + 2 * g.n);
    } else if constexpr (KIND == kFfnWeightGrad) {
      if (g.accumulate) {
        const uint8_t* p = c + (long long)(t.m0 + row) * g.ldc + (F32 ? 4 : 2) * col;
        o.q[0] = load16(p);
        if constexpr (F32) o.q[1] = load16(p + 16);
      }
    }
  }
  static __device__ __forceinline__ void store(const FfnArgs& g, const FfnTile& t, uint8_t* c, int row, int col, const Old& o,
                                               float (&v)[8], const float (&up)[8]) {
    const long long r = t.m0 + row;
    if constexpr (KIND == kFfnGateUp) {
      if (c) {
        uint8_t* p = c + r * 4 * g.n + 2 * col;
        store16(p, ffn_bf16x8(v));
        store16(p + 2 * g.n, ffn_bf16x8(up));
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = swiglu_of<true>(v[i], up[i]);
      store16(g.h + r * 2 * g.n + 2 * col, ffn_bf16x8(v));
    } else if constexpr (KIND == kFfnDownGrad) {
      float gate[8], u[8], du[8], h[8];
      ffn_unpack8(o.q[0], gate);
      ffn_unpack8(o.q[1], u);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        h[i] = swiglu_of<true>(gate[i], u[i]);
        swiglu_grad(gate[i], u[i], v[i], v[i], du[i]);
      }
      uint8_t* p = c + r * 4 * g.n + 2 * col;
      store16(p, ffn_bf16x8(v));
      store16(p + 2 * g.n, ffn_bf16x8(du));
      if (g.h) store16(g.h + r * 2 * g.n + 2 * col, ffn_bf16x8(h));
    } else {
      uint8_t* p = c + r * g.ldc + (F32 ? 4 : 2) * col;
      if constexpr (KIND == kFfnWeightGrad) {
        if (g.accumulate) {
          if constexpr (F32) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] += __uint_as_float(o.q[i / 4][i % 4]);
          } else {
            float old[8];
            ffn_unpack8(o.q[0], old);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] += old[i];
          }
        }
      }
      if constexpr (F32) {
        ffn_store16(p, u32x4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])});
        ffn_store16(p + 16, u32x4{__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7])});
      } else {
        ffn_store16(p, ffn_bf16x8(v));
      }
    }
  }
};

// LDS of a tile, in 16-byte chunks: SA slots of the BM x BK panel, SB of the BR x BK one.
constexpr int ffn_chunks(int bm, int br, int bk, int sa, int sb) { return (sa * bm + sb * br) * (bk / 8); }

// A tile of BM rows and BR columns (gate/up: BR / 2 of each), by a WM x WN grid of waves.
template <int KIND, bool F32, int BM, int BR, int BK, int WM, int WN, int SA, int SB,
          bool HALF = !F32 && KIND != kFfnGateUp && KIND != kFfnDownGrad>
__device__ __forceinline__ void ffn_tile(const FfnArgs& g, const FfnTile& t, uint8_t* c, u32x4* lds) {
  constexpr bool GATED = KIND == kFfnGateUp, A_COL = KIND == kFfnWeightGrad, B_COL = KIND >= kFfnDownGrad;
  constexpr int NB = GATED ? 2 : 1, BN = BR / NB;
  constexpr int WTM = BM / WM, WTN = BN / WN, FM = WTM / 32, FN = WTN / 32, FB = FN * NB;
  constexpr int SUB = BK / 16, NRD = FM + FB, NMF = FM * FB;
  using PA = FfnPanel<A_COL, BM, BK>;
  using PB = FfnPanel<B_COL, BR, BK>;
  constexpr int A_INS = PA::INS, B_INS = PB::INS, NPS = A_INS + B_INS;
  constexpr int LEAD = SA - SB;
  static_assert(WM * WN == 4 && FM * 32 == WTM && FN * 32 == WTN, "four waves of whole blocks");
  static_assert(LEAD == 0 || (LEAD == 1 && SB == 2), "activation lead: two weight slots only");
  static_assert(NPS * (SB - 1) < 64 && 2 * A_INS + B_INS < 64, "wait range");
  constexpr int PART_N = LEAD == 1 ? A_INS : NPS, NPART = LEAD == 1 ? SUB - 1 : SUB;
  constexpr int END_PARTS = NPART - (SUB - 1), PART0 = END_PARTS * PART_N / NPART;
  u32x4* const ring_a = lds;
  u32x4* const ring_b = lds + SA * PA::CH;

  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave / WN, wn = wave % WN;
  const int K = KIND == kFfnWeightGrad ? t.k_count : g.k;
  const int KT = (K + BK - 1) / BK;

  PA pa;
  PB pb;
  if constexpr (A_COL)
    pa.by_columns(g.a + (long long)t.k0 * g.lda + 2 * t.m0, g.lda, t.k_count, g.m - t.m0, wave, lane);
  else
    pa.by_rows(g.a + (long long)t.m0 * g.lda, g.lda, (t.rows - 1) * (int)g.lda + 2 * K, K, wave, lane,
               [](int r) { return r; });
  if constexpr (KIND == kFfnWeightGrad)
    pb.by_columns(g.b + (long long)t.k0 * g.ldb + 2 * t.n0, g.ldb, t.k_count, g.n - t.n0, wave, lane);
  else if constexpr (B_COL)
    pb.by_columns(g.b + t.group * g.b_group + 2 * t.n0, g.ldb, K, g.n - t.n0, wave, lane);
  else
    pb.by_rows(g.b + t.group * g.b_group, g.ldb, (GATED ? 2 : 1) * g.n * (int)g.ldb, K, wave, lane, [&](int r) {
      // columns past n read the last one
      return GATED && r >= BN ? g.n + min(t.n0 + r - BN, g.n - 1) : min(t.n0 + r, g.n - 1);
    });

  // Where weights by rows are a multiple of 4 KB apart, they all start on one memory channel, and
  // tiles that read the same k at a time press on a few: the tiles of a column tile start at
  // their own slice, and go round.
  int rot = 0;
  if constexpr (!B_COL) {
    if (g.ldb % 4096 == 0) rot = uniform((int)((unsigned)(t.group * g.n_tiles + t.n0 / BN) * 2u % (unsigned)KT));
  }
  auto slice_at = [&](int kt) { return B_COL || kt + rot < KT ? kt + rot : kt + rot - KT; };
  auto issue_a1 = [&](int i, int kt, int slot) {
    const int at = slice_at(kt);
    pa.issue(i, at, at == KT - 1, ring_a + slot * PA::CH, wave);
  };
  auto issue_b1 = [&](int i, int kt, int slot) {
    const int at = slice_at(kt);
    pb.issue(i, at, at == KT - 1, ring_b + slot * PB::CH, wave);
  };
  auto issue_a = [&](int kt, int slot) {
#pragma unroll
    for (int i = 0; i < A_INS; ++i) issue_a1(i, kt, slot);
  };
  auto issue_b = [&](int kt, int slot) {
#pragma unroll
    for (int i = 0; i < B_INS; ++i) issue_b1(i, kt, slot);
  };
  auto issue_part1 = [&](int i, int kt, int slot) {
    if (LEAD == 1 || i < A_INS) issue_a1(i, kt, slot);
    else issue_b1(i - A_INS, kt, slot);
  };
  bf16x8_ffn fa[2][FM], fb[2][FB];
  auto read_frag = [&](int i, int aslot, int bslot, int sub, bf16x8_ffn (&a)[FM], bf16x8_ffn (&b)[FB]) {
    if (i < FM) {
      a[i] = PA::read(ring_a + aslot * PA::CH, wm * WTM + i * 32, sub, lane);
    } else {
      const int j = i - FM;
      b[j] = PB::read(ring_b + bslot * PB::CH, j / FN * BN + wn * WTN + j % FN * 32, sub, lane);
    }
  };
  // The b fragment goes first: lane l ends with row l % 32 of a block and, in registers 4 q ..
  // 4 q + 3, its columns 8 q + 4 (l / 32) + 0 .. 3.
  f32x16_ffn acc[FM][FB];
  auto mfma = [&](int i, const bf16x8_ffn (&a)[FM], const bf16x8_ffn (&b)[FB]) {
    const int fm = i / FB, j = i % FB;
    acc[fm][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(b[j], a[fm], acc[fm][j], 0, 0, 0);
  };
  auto no_op = [](auto) {};
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FB; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;

  if (KT > 0) {
    if constexpr (LEAD == 1) issue_a(0, 0);
#pragma unroll
    for (int st = 0; st < SB; ++st) {
      if (st >= KT) break;
      if (LEAD == 0) issue_a(st, st);
      issue_b(st, st);
      if (LEAD == 1 && st + 1 < KT) issue_a(st + 1, st + 1);
    }
    if constexpr (LEAD == 0) {
      wait_rings_lgkm0<A_INS, B_INS, SA - 1, SB - 1>(KT - 1);
    } else {
      if (KT > 2) wait_vmcnt_lgkm0<2 * A_INS + B_INS>();
      else if (KT == 2) wait_vmcnt_lgkm0<A_INS + B_INS>();
      else wait_vmcnt_lgkm0<0>();
    }
    bare_barrier();
#pragma unroll
    for (int i = 0; i < NRD; ++i) read_frag(i, 0, 0, 0, fa[0], fb[0]);

    // One slice.  MODE 0: a later slice goes into this one's slot after the barrier; 1: none
    // is left; 2: the last.  PEND: parts of the group begun at the last slice's end remain.
    auto slice = [&](auto mode, auto pend, int kt, int aslot, int bslot) {
      constexpr int MODE = decltype(mode)::value;
      constexpr bool PEND = decltype(pend)::value;
      int pkt, pslot;
      if constexpr (LEAD == 1) {
        pkt = kt + 2;
        pslot = aslot + 2 >= SA ? aslot + 2 - SA : aslot + 2;
      } else {
        pkt = kt - 1 + SB;
        pslot = bslot == 0 ? SB - 1 : bslot - 1;
      }
      weave_run<0, SUB>([&](auto subc) {
        constexpr int sub = decltype(subc)::value;
        constexpr int cur = sub & 1, nxt = cur ^ 1;
        auto mul = [&](auto i) { mfma(i, fa[cur], fb[cur]); };
        if constexpr (sub + 1 < SUB) {
          auto rd = [&](auto i) { read_frag(i, aslot, bslot, sub + 1, fa[nxt], fb[nxt]); };
          constexpr int P = END_PARTS + sub;
          constexpr int D0 = PEND ? PART_N * P / NPART : 0, D1 = PEND ? PART_N * (P + 1) / NPART : 0;
          weave<NMF, NRD, D1 - D0>(mul, rd, [&](auto i) { issue_part1(D0 + i, pkt, pslot); });
        } else if constexpr (MODE < 2) {
          if constexpr (LEAD == 1) {
            if (kt + 2 < KT) wait_vmcnt_lgkm0<A_INS>();
            else wait_vmcnt_lgkm0<0>();
          } else if constexpr (MODE == 0) {
            wait_vmcnt_lgkm0<A_INS*(SA - 2) + B_INS * (SB - 2)>();
          } else {
            wait_rings_lgkm0<A_INS, B_INS, SA - 2, SB - 2>(KT - 2 - kt);
          }
          bare_barrier();
          int nb = bslot + 1, na = aslot + 1;
          if (nb == SB) nb = 0;
          if (na == SA) na = 0;
          auto rd = [&](auto i) { read_frag(i, na, nb, 0, fa[nxt], fb[nxt]); };
          constexpr int ND = MODE != 0 ? 0 : LEAD == 1 ? B_INS : PART0;
          weave<NMF, NRD, ND>(mul, rd, [&](auto i) {
            if constexpr (LEAD == 1) issue_b1(i, kt + SB, bslot);
            else issue_part1(i, kt + SB, bslot);
          });
        } else {
          weave<NMF, 0, 0>(mul, no_op, no_op);
        }
      });
    };
    int kt = 0, aslot = 0, bslot = 0;
    auto advance = [&] {
      if (++bslot == SB) bslot = 0;
      if (++aslot == SA) aslot = 0;
    };
    using M0 = std::integral_constant<int, 0>;
    using M1 = std::integral_constant<int, 1>;
    using NoPend = std::false_type;
    using Pend = std::true_type;
    if (KT > SB) {
      slice(M0{}, NoPend{}, kt, aslot, bslot);
      advance();
      for (++kt; kt < KT - SB; ++kt) {
        slice(M0{}, Pend{}, kt, aslot, bslot);
        advance();
      }
      if constexpr (LEAD == 0) {
        slice(M1{}, Pend{}, kt, aslot, bslot);
        advance();
        ++kt;
      }
    }
    for (; kt < KT - 1; ++kt) {
      slice(M1{}, NoPend{}, kt, aslot, bslot);
      advance();
    }
    slice(std::integral_constant<int, 2>{}, NoPend{}, kt, aslot, bslot);
    wait_vmcnt_lgkm0<63>();
    bare_barrier();
  }

  // Results go out through LDS, 32 rows of the wave's columns at a time (within a wave LDS
  // operations complete in order): written as the accumulators lie, rows 16 bytes apart
  // beyond their width, read back 8 columns of a row to a lane, so that memory sees whole
  // lines.  Where nothing else is done to them they are rounded on the way in (HALF), which
  // halves what passes through LDS: it, not the MFMAs, bounds the weights' gradients of short groups (257
  // rows, 4096 x 7168 of 32 groups: 675 us without, 625 with).
  constexpr int LPR = WTN / 8, RPP = 64 / LPR, PASSES = 32 / RPP;
  const int rr0 = lane / LPR, col = lane % LPR * 8, n_at = t.n0 + wn * WTN + col;
  if constexpr (HALF) {
    typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
    constexpr int PITCH = WTN * 2 + 16, PATCH = 32 * PITCH;  // bytes
    static_assert(4 * PATCH <= 16 * ffn_chunks(BM, BR, BK, SA, SB) && !GATED, "patches within the ring");
    uint8_t* patch = reinterpret_cast<uint8_t*>(lds) + wave * PATCH;
#pragma unroll
    for (int fm = 0; fm < FM; ++fm) {
#pragma unroll
      for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          *reinterpret_cast<u32x2*>(patch + (lane & 31) * PITCH + 2 * (j * 32 + 8 * q + 4 * (lane >> 5))) =
              u32x2{bf16_pair(acc[fm][j][4 * q], acc[fm][j][4 * q + 1]), bf16_pair(acc[fm][j][4 * q + 2], acc[fm][j][4 * q + 3])};
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int p = 0; p < PASSES; ++p) {
        const int rr = p * RPP + rr0, row = wm * WTM + fm * 32 + rr;
        const u32x4 v = load16(patch + rr * PITCH + 2 * col);
        if (row < t.rows && n_at < g.n) ffn_store16(c + (long long)(t.m0 + row) * g.ldc + 2 * n_at, v);
      }
      __builtin_amdgcn_wave_barrier();
    }
  } else {
    constexpr int PITCH = WTN + 4, PATCH = 32 * PITCH;  // floats; gate/up: one of each
    static_assert(4 * NB * PATCH <= 4 * ffn_chunks(BM, BR, BK, SA, SB), "patches within the ring");
    float* patch = reinterpret_cast<float*>(lds) + wave * (NB * PATCH);
    using Out = FfnStore<KIND, F32>;
#pragma unroll
    for (int fm = 0; fm < FM; ++fm) {
      typename Out::Old old[PASSES];
      const int row0 = wm * WTM + fm * 32;
#pragma unroll
      for (int p = 0; p < PASSES; ++p) {
        const int row = row0 + p * RPP + rr0;
        if (row < t.rows && n_at < g.n) Out::load(g, t, c, row, n_at, old[p]);
      }
#pragma unroll
      for (int j = 0; j < FB; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          *reinterpret_cast<f32x4_ffn*>(patch + j / FN * PATCH + (lane & 31) * PITCH + j % FN * 32 + 8 * q + 4 * (lane >> 5)) =
              f32x4_ffn{acc[fm][j][4 * q], acc[fm][j][4 * q + 1], acc[fm][j][4 * q + 2], acc[fm][j][4 * q + 3]};
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int p = 0; p < PASSES; ++p) {
        const int rr = p * RPP + rr0, row = row0 + rr;
        float v[8], up[8];
        auto take = [&](float (&to)[8], const float* from) {
          const f32x4_ffn lo = *reinterpret_cast<const f32x4_ffn*>(from), hi = *reinterpret_cast<const f32x4_ffn*>(from + 4);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            to[i] = lo[i];
            to[4 + i] = hi[i];
          }
        };
        take(v, patch + rr * PITCH + col);
        if constexpr (GATED) take(up, patch + PATCH + rr * PITCH + col);
        if (row < t.rows && n_at < g.n) Out::store(g, t, c, row, n_at, old[p], v, up);
      }
      __builtin_amdgcn_wave_barrier();
    }
  }
}

// A tile of up to 32 rows and 32 NB columns (gate/up: 16 NB of each) for few rows, where the stream of
// weights is what bounds a product: the W waves of a workgroup deal the tile's blocks of 64 of K
// among them, each with a ring of S blocks of its own (no barrier: a wave waits for its own
// transfers alone), and their sums meet in LDS and are added in wave order.  Up to 8 rows take an
// 8-row panel (RA), whose rows the MFMA's 32 read over and over: what the others give is not stored.
constexpr int ffn_few_chunks(int ra, int nb, int w, int s) { return w * s * (ra + 32 * nb) * 8; }
template <int KIND, bool F32, int RA, int NB, int W, int S>
__device__ __forceinline__ void ffn_few_tile(const FfnArgs& g, const FfnTile& t, u32x4* lds) {
  constexpr bool GATED = KIND == kFfnGateUp, B_COL = KIND >= kFfnDownGrad;
  static_assert(KIND != kFfnWeightGrad && (!B_COL || NB == 2), "panels");
  constexpr int BN = GATED ? 16 * NB : 32 * NB;
  using PA = FfnPanel<false, RA, 64, 1>;
  using PB = FfnPanel<B_COL, 32 * NB, 64, 1>;
  constexpr int NP = PA::INS + PB::INS, SLOT = PA::CH + PB::CH;
  static_assert(NP * S < 64, "wait range");
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  u32x4* ring = lds + wave * (S * SLOT);
  const int KT = (g.k + 63) / 64, count = (KT - wave + W - 1) / W;  // this wave's blocks: wave, wave + W, ...

  PA pa;
  PB pb;
  pa.by_rows(g.a + (long long)t.m0 * g.lda, g.lda, (t.rows - 1) * (int)g.lda + 2 * g.k, g.k, 0, lane,
             [](int r) { return r; });
  if constexpr (B_COL)
    pb.by_columns(g.b + t.group * g.b_group + 2 * t.n0, g.ldb, g.k, g.n - t.n0, 0, lane);
  else
    pb.by_rows(g.b + t.group * g.b_group, g.ldb, (GATED ? 2 : 1) * g.n * (int)g.ldb, g.k, 0, lane, [&](int r) {
      return GATED && r >= BN ? g.n + min(t.n0 + r - BN, g.n - 1) : min(t.n0 + r, g.n - 1);
    });
  auto issue = [&](int i, int slot) {
    const int kt = wave + i * W;
#pragma unroll
    for (int q = 0; q < PA::INS; ++q) pa.issue(q, kt, kt == KT - 1, ring + slot * SLOT, 0);
#pragma unroll
    for (int q = 0; q < PB::INS; ++q) pb.issue(q, kt, kt == KT - 1, ring + slot * SLOT + PA::CH, 0);
  };
  f32x16_ffn acc[NB];
#pragma unroll
  for (int j = 0; j < NB; ++j)
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[j][r] = 0.f;
#pragma unroll
  for (int q = 0; q < S; ++q)
    if (q < count) issue(q, q);
  int slot = 0;
  for (int i = 0; i < count; ++i) {
    wait_rings_lgkm0<NP, 0, S - 1, 0>(count - 1 - i);  // block i has landed
    __atomic_signal_fence(__ATOMIC_SEQ_CST);           // the reads stay behind the wait
    const u32x4* at = ring + slot * SLOT;
    bf16x8_ffn fa[4], fb[4][NB];
#pragma unroll
    for (int sub = 0; sub < 4; ++sub) {
      fa[sub] = PA::read(at, 0, sub, lane);
#pragma unroll
      for (int j = 0; j < NB; ++j) fb[sub][j] = PB::read(at + PA::CH, 32 * j, sub, lane);
    }
    __atomic_signal_fence(__ATOMIC_SEQ_CST);  // and ahead of the next
    wait_vmcnt_lgkm0<63>();                   // it is in registers: its slot is free
    __atomic_signal_fence(__ATOMIC_SEQ_CST);
    if (i + S < count) issue(i + S, slot);
#pragma unroll
    for (int sub = 0; sub < 4; ++sub)
#pragma unroll
      for (int j = 0; j < NB; ++j)
        acc[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fb[sub][j], fa[sub], acc[j], 0, 0, 0);
    if (++slot == S) slot = 0;
  }

  // Each wave's sums to a patch of its own ring; then every thread adds 8 columns of a row.
  constexpr int PITCH = 32 * NB + 4;
  static_assert(32 * PITCH * 4 <= S * SLOT * 16, "a patch within the wave's ring");
  float* patch = reinterpret_cast<float*>(ring);
#pragma unroll
  for (int j = 0; j < NB; ++j)
#pragma unroll
    for (int q = 0; q < 4; ++q)
      *reinterpret_cast<f32x4_ffn*>(patch + (lane & 31) * PITCH + 32 * j + 8 * q + 4 * (lane >> 5)) =
          f32x4_ffn{acc[j][4 * q], acc[j][4 * q + 1], acc[j][4 * q + 2], acc[j][4 * q + 3]};
  __syncthreads();
  constexpr int LPR = BN / 8;
  using Out = FfnStore<KIND, F32>;
  for (int at = threadIdx.x; at < t.rows * LPR; at += 64 * W) {
    const int row = at / LPR, col = at % LPR * 8;
    if (t.n0 + col >= g.n) continue;
    typename Out::Old old;
    Out::load(g, t, g.c, row, t.n0 + col, old);
    float v[8], up[8];
    auto take = [&](float (&to)[8], int c) {
#pragma unroll
      for (int i = 0; i < 8; ++i) to[i] = 0.f;
#pragma unroll
      for (int w = 0; w < W; ++w) {
        const float* from = reinterpret_cast<const float*>(lds + w * (S * SLOT)) + row * PITCH + c;
        const f32x4_ffn lo = *reinterpret_cast<const f32x4_ffn*>(from), hi = *reinterpret_cast<const f32x4_ffn*>(from + 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          to[i] += lo[i];
          to[4 + i] += hi[i];
        }
      }
    };
    take(v, col);
    if constexpr (GATED) take(up, BN + col);
    Out::store(g, t, g.c, row, t.n0 + col, old, v, up);
  }
}

}  // namespace moepd
