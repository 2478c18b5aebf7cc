// Tiles of a product whose rows lie in groups (an expert's rows), found by each
// workgroup from the groups' offsets on the device: no launch before the product and no
// prefix in memory.  G is an argument struct with offsets (null: one group of all rows),
// rows, groups, n_tiles and run.
#pragma once

#include "common.h"

namespace moepd {

struct GroupTile {  // wave-uniform
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

// How a group's rows are shared among its row tiles.
enum RowShare : int { kRowsEven = 0, kRowsInBlocks = 1, kRowsFull = 2 };

// The tile of workgroup b, if any, found by each wave from the offsets: lane i
// holds group i's rows, and a scan of the groups' counts of row tiles (of at most bm
// rows) places the tile; with more than 64 groups, 64 at a time.
//
// STRIPED (streaming tiles): groups in order, within a group of mt row tiles column
// tile 8 q + b % 8 for each q, with all its row tiles in a row: workgroup b runs on
// XCD b % 8, so the row tiles that read one weight panel share an L2, and every XCD
// streams an eighth of every group's weights.
//
// Otherwise (ring tiles): a group's rows are shared evenly among its row tiles (kRowsInBlocks: its
// blocks of 32 rows are, for tiles cut to them; kRowsFull: full tiles and a rest,
// of which a small one takes half of the last full tile's with it); its
// tiles run over blocks of four column tiles, in each row tile by row tile; and runs of
// consecutive tiles are dealt to the XCDs in turn, so that an XCD's L2 serves each row
// block to four workgroups and each weight panel to as many as the run has row
// tiles.  The last runs, when they do not go round, are dealt tile by tile.  Runs of 64 tiles
// (16 row x 4 column tiles: what an XCD's CUs hold at a time) for groups of many rows,
// else 32, which leave less to the last round: 96,889 skewed rows (7168 x 2048)
// 1030 us with 64, 1096 with 32; 32,768 rows 391 / 430; 8192 rows, 256 to a group, 77 / 73.
template <bool STRIPED, int SHARE = kRowsEven, class G>
__device__ __forceinline__ bool group_tile(const G& g, int b, int bm, GroupTile& t) {
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
    if constexpr (SHARE == kRowsFull) {
      const int full = bm / 32, rest = (hi - lo + 31) / 32 - full * (mt_e - 1);  // of the last tile, in blocks
      const int last = rest <= full / 4 && mt_e > 1 ? full * (mt_e - 2) + (full + rest + 1) / 2 : full * (mt_e - 1);
      t.m0 = uniform(lo + 32 * (mi < mt_e - 1 ? full * mi : last));
      t.m_end = uniform(min(lo + 32 * (mi + 1 < mt_e - 1 ? full * (mi + 1) : mi + 1 == mt_e - 1 ? last : full * mt_e), hi));
    } else if constexpr (SHARE == kRowsInBlocks) {
      const int nb = (hi - lo + 31) / 32;
      t.m0 = uniform(lo + (int)((long long)nb * mi / mt_e) * 32);
      t.m_end = uniform(min(lo + (int)((long long)nb * (mi + 1) / mt_e) * 32, hi));
    } else {
      const int per = (hi - lo + mt_e - 1) / mt_e;
      t.m0 = uniform(lo + mi * per);
      t.m_end = uniform(min(t.m0 + per, hi));
    }
  }
  return true;
}

}  // namespace moepd
