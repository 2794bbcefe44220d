// Rows in ragged groups: group e of N owns rows offsets[e] .. offsets[e + 1] - 1 of an
// S-row array (the layer's expert_offsets, or the token offsets of the requests of a
// batch).  A launch cuts every group into tiles of TM rows; the offsets are on the device,
// so the host launches the most tiles there can be and each wave finds its own.
#pragma once

#include "ace_internal.h"

namespace ace {

struct RaggedTile {
  int group;  // 0 .. N - 1, or -1: rows of no group (before the first, behind the last)
  int row0, rows;
  bool valid;
};

// Tiles of S rows in N groups and the two gaps around them: a group of r rows has at most
// r / TM full ones and one short one.
inline long long ragged_max_tiles(long long S, long long N, int tm) {
  return S / tm + (N + 2 < S ? N + 2 : S);
}

// Tile `tile` in group order, the same in every lane of the calling wave (all 64 lanes
// call).  The gaps come as groups of their own before the first and behind the last when
// `gaps` is set.  Offsets are clamped to 0 .. S, so whatever they hold, rows outside the
// array are never named.  Lane l counts the tiles of `per` consecutive groups, one wave
// scan places them: one round of loads and one scan, against a launch of its own for a tile
// list.
__device__ __forceinline__ RaggedTile ragged_tile(const int32_t *offsets, int N, int S, int tm_log2, int tile,
                                                  bool gaps) {
  const int lane = threadIdx.x & 63;
  const int tm = 1 << tm_log2;
  const int per = (N + 2 + 63) >> 6;
  // boundary i of the N + 2 groups: 0, offsets[0], .., offsets[N], S
  auto bound = [&](int i) { return i <= 0 ? 0 : i > N + 1 ? S : min(max(offsets[i - 1], 0), S); };
  auto tiles = [&](int p, int lo, int hi) {
    if (p > N + 1 || hi <= lo || ((p == 0 || p == N + 1) && !gaps)) return 0;
    return static_cast<int>((static_cast<uint32_t>(hi - lo) + static_cast<uint32_t>(tm) - 1u) >> tm_log2);
  };
  const int p0 = lane * per;
  int cnt = 0, lo = bound(p0);
  for (int j = 0; j < per; ++j) {
    const int hi = bound(p0 + j + 1);
    cnt += tiles(p0 + j, lo, hi);
    lo = hi;
  }
  int inc = cnt;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int v = __shfl_up(inc, o);
    if (lane >= o) inc += v;
  }
  const unsigned long long own = __ballot(inc - cnt <= tile && tile < inc);
  RaggedTile t{-1, 0, 0, false};
  if (own == 0) return t;
  const int src = __ffsll(static_cast<long long>(own)) - 1;
  const int first = __builtin_amdgcn_readlane(inc - cnt, src);
  int q = tile - first, p = src * per;
  lo = bound(p);
  for (int j = 0; j < per; ++j, ++p) {
    const int hi = bound(p + 1), n = tiles(p, lo, hi);
    if (q < n) {
      t.group = p == 0 || p == N + 1 ? -1 : p - 1;
      t.row0 = lo + (q << tm_log2);
      t.rows = min(tm, hi - t.row0);
      t.valid = true;
      break;
    }
    q -= n;
    lo = hi;
  }
  t.group = __builtin_amdgcn_readfirstlane(t.group);
  t.row0 = __builtin_amdgcn_readfirstlane(t.row0);
  t.rows = __builtin_amdgcn_readfirstlane(t.rows);
  return t;
}

// A launch takes fewer than 2^32 threads in x: grids of more blocks than a row of 2^20 are
// several rows, the last row's excess past the end.
constexpr int kRaggedGridRow = 20;
constexpr long long kRaggedMaxBlocks = (1ll << 31) - (1ll << kRaggedGridRow);  // block numbers are ints
inline dim3 ragged_grid(long long blocks) {
  if (blocks <= 1ll << kRaggedGridRow) return dim3(static_cast<unsigned>(blocks));
  return dim3(1u << kRaggedGridRow, static_cast<unsigned>((blocks + (1ll << kRaggedGridRow) - 1) >> kRaggedGridRow));
}
__device__ __forceinline__ int ragged_block() {
  return static_cast<int>((blockIdx.y << kRaggedGridRow) + blockIdx.x);
}

}  // namespace ace
