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
  bool only;  // the group's only tile
  int slot;   // of a tile that is not: its number among those
};

// Tiles of S rows in N groups and the two gaps around them: a group of r rows has at most
// r / TM full ones and one short one.
inline long long ragged_max_tiles(long long S, long long N, int tm) {
  return S / tm + (N + 2 < S ? N + 2 : S);
}

// The tiles of all groups in group order, held by one wave (all 64 lanes take part in every
// call).  The gaps come as groups of their own before the first and behind the last when
// `gaps` is set; with `each`, a group without rows has one tile of none.  Offsets are clamped to 0 .. S, so whatever they hold, rows outside the
// array are never named.  Lane l counts the tiles of `per` consecutive groups, one wave
// scan places them: `per` + 2 loads and one scan, against a launch of its own for a tile
// list.  Every load is made, at a place that is there, and what it does not count for dropped, so that a lane's loads
// go out together: a trip to the cache for four of them, and again to find a tile where `per` is over 1.
struct RaggedTiles {
  const int32_t *offsets;
  int N, S, tm, per, cnt, inc, total;
  int shared, shared_inc;  // tiles of groups of more than one, counted alike
  int first, last;         // boundaries of this lane's groups
  bool gaps, each;

  // boundary i of the N + 2 groups: 0, offsets[0], .., offsets[N], S
  __device__ __forceinline__ int bound(int i) const {
    const int v = min(max(offsets[min(max(i - 1, 0), N)], 0), S);
    return i <= 0 ? 0 : i > N + 1 ? S : v;
  }
  __device__ __forceinline__ int tiles(int p, int lo, int hi) const {
    if (p > N + 1 || ((p == 0 || p == N + 1) && !gaps)) return 0;
    if (hi <= lo) return each && p > 0 && p <= N;
    return static_cast<int>((static_cast<uint32_t>(hi - lo) + tm - 1u) / static_cast<uint32_t>(tm));
  }

  __device__ __forceinline__ RaggedTiles(const int32_t *offsets_, int N_, int S_, int tm_, bool gaps_,
                                         bool each_ = false)
      : offsets(offsets_), N(N_), S(S_), tm(tm_), per((N_ + 2 + 63) >> 6), cnt(0), shared(0), gaps(gaps_), each(each_) {
    const int lane = threadIdx.x & 63;
    const int p0 = lane * per;
    int lo = bound(p0);
#pragma unroll 4
    for (int j = 0; j < per; ++j) {
      const int hi = bound(p0 + j + 1);
      const int n = tiles(p0 + j, lo, hi);
      cnt += n;
      shared += n > 1 ? n : 0;
      lo = hi;
    }
    first = bound(p0);
    last = lo;
    inc = cnt;
    shared_inc = shared;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int v = __shfl_up(inc, o), w = __shfl_up(shared_inc, o);
      if (lane >= o) {
        inc += v;
        shared_inc += w;
      }
    }
    // ascending offsets make no more than this; others could ask for thousands of passes over the array
    total = min(__builtin_amdgcn_readlane(inc, 63), S / tm + N + 2);
  }

  // tiles[i]: how many tiles of heights[i] rows there are, without the list of any
  template <int H>
  static __device__ __forceinline__ void count(const int32_t *offsets, int N, int S, const int (&heights)[H],
                                               int (&tiles)[H], bool gaps) {
#pragma unroll
    for (int i = 0; i < H; ++i) tiles[i] = 0;
    for (int p = static_cast<int>(threadIdx.x & 63); p < N + 2; p += 64) {
      const int lo = p == 0 ? 0 : min(max(offsets[p - 1], 0), S), hi = p > N ? S : min(max(offsets[p], 0), S);
      if (hi <= lo || ((p == 0 || p == N + 1) && !gaps)) continue;
#pragma unroll
      for (int i = 0; i < H; ++i)
        tiles[i] += static_cast<int>((static_cast<uint32_t>(hi - lo) + heights[i] - 1u) / static_cast<uint32_t>(heights[i]));
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1)
#pragma unroll
      for (int i = 0; i < H; ++i) tiles[i] += __shfl_xor(tiles[i], o);
#pragma unroll
    for (int i = 0; i < H; ++i) tiles[i] = __builtin_amdgcn_readfirstlane(tiles[i]);
  }

  // tile `tile`, each lane its own
  __device__ __forceinline__ RaggedTile find(int tile) const {
    RaggedTile t{-1, 0, 0, false, false, 0};
    // the lane that counts the tile: the first whose inclusive sum exceeds it
    int src = 0;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1)
      if (__shfl(inc, src + o - 1) <= tile) src += o;
    int q = tile - __shfl(inc - cnt, src), slot = __shfl(shared_inc - shared, src);
    if (tile < 0 || tile >= total || q < 0) return t;
    const int p0 = src * per;
    int from = __shfl(first, src), to = __shfl(last, src), n = 0;
    if (per == 1) {  // the lane's only group, without another load
      n = tiles(p0, from, to);
      if (q >= n) return t;
      t.group = p0;
    }
    int lo = from;
#pragma unroll 4
    for (int j = 0; per > 1 && j < per; ++j) {
      const int hi = bound(p0 + j + 1), m = tiles(p0 + j, lo, hi);
      if (n == 0) {  // not found yet
        if (q < m) {
          t.group = p0 + j;
          from = lo;
          to = hi;
          n = m;
        } else {
          q -= m;
          slot += m > 1 ? m : 0;
        }
      }
      lo = hi;
    }
    if (n == 0) return t;
    t.group = t.group == 0 || t.group == N + 1 ? -1 : t.group - 1;
    // the group's 16-row blocks spread evenly over its tiles: a short tile would stream the group's
    // operands for a few rows
    const uint32_t blocks = (static_cast<uint32_t>(max(to - from, 0)) + 15u) >> 4, each = blocks / n, more = blocks % n;
    const uint32_t b0 = q * each + min(static_cast<uint32_t>(q), more);
    t.row0 = from + static_cast<int>(b0 << 4);
    t.rows = min(static_cast<int>((each + (q < static_cast<int>(more))) << 4), max(to - t.row0, 0));
    t.valid = true;
    t.only = n == 1;
    t.slot = slot + q;
    return t;
  }

  // the same for a wave-uniform tile, in scalar registers
  __device__ __forceinline__ RaggedTile find_uniform(int tile) const {
    RaggedTile t = find(tile);
    t.group = __builtin_amdgcn_readfirstlane(t.group);
    t.row0 = __builtin_amdgcn_readfirstlane(t.row0);
    t.rows = __builtin_amdgcn_readfirstlane(t.rows);
    t.valid = __builtin_amdgcn_readfirstlane(t.valid);
    return t;
  }
};

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
