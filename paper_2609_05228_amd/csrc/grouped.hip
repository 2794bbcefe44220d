// Matrix products grouped by expert with ragged sizes, and their gradients.  Rows of x
// [S, K] lie in group order (group e: rows offsets[e] .. offsets[e + 1] - 1), group e has
// the weights w[e] [M, K] (nn.Linear layout):
//   forward          y[r]  = w[e] x[r]                      reduced over K
//   rows' gradient   dx[r] = w[e]^T dy[r]                   reduced over M
//   weights' one     dw[e] = sum over rows r of e: dy[r] x[r]^T   reduced over the group's rows
// One tile body serves the three (grouped_tile.h): w lies k-major in the forward and k down in the
// rows' gradient, dy and x k down in the weights' one.
#include "grouped_tile.h"

namespace ace {

namespace {

// Tiles of x's or dy's rows by columns, the whole work of a workgroup
template <typename T, bool GX, bool LINES, int MB, int NB, int WR, int WC, int DA, int DB>
__device__ __forceinline__ void grouped_rows(const GroupedArgs &g, const RaggedTiles &tiles, uint8_t *smem) {
  constexpr int BN = 16 * NB;
  const int cols = GX ? g.K : g.M, klen = GX ? g.M : g.K;
  const int nN = (cols + BN - 1) / BN, per = nN * g.splits;
  const Share share(static_cast<long long>(tiles.total) * per);
  using S = DenseTile<T, false, GX, MB, NB, WR, WC, DA, DB>;
  auto ref = [&](const Item &it, int) {
    const int c0 = it.tile * BN;
    const Part k = part_of<S::A::BK>(it.group < 0 ? 0 : klen, it.split, g.splits);
    typename S::Ref t;
    t.a.p[0] = static_cast<const T *>(g.rows) + static_cast<size_t>(it.row0) * klen + k.k0;
    const T *w = static_cast<const T *>(g.other) + static_cast<size_t>(max(it.group, 0)) * g.M * g.K;
    t.b.p[0] = GX ? w + static_cast<size_t>(k.k0) * g.K + c0 : w + static_cast<size_t>(c0) * g.K + k.k0;
    t.out = static_cast<T *>(g.out) + static_cast<size_t>(it.row0) * cols + c0;
    t.part = g.splits > 1 ? g.part + (static_cast<size_t>(it.split) * g.S + it.row0) * cols + c0 : nullptr;
    t.rows = it.rows;
    t.cols = min(BN, cols - c0);
    t.klen = k.len;
    t.rot = max(it.group, 0);
    t.once = it.once;
    return t;
  };
  long long done = 0;
  for (int n; (n = share.count(done)) > 0; done += n) {
    const long long i = share.item(done);
    const RaggedTile t = tiles.find(static_cast<int>(i / per));
    const int q = static_cast<int>(i % per);
    __syncthreads();  // every wave is done with the rings
    grouped_items<S>(Item{t.group, t.row0, t.rows, q % nN, t.only, q / nN}, n, klen, g.K, smem, ref,
                     StoreTile<T, LINES, S>{static_cast<size_t>(cols)});
  }
}

// Forward (GX = false) and rows' gradient (GX = true) in tiles of 16 MB rows of one group x 16 NB columns
template <typename T, bool GX, bool LINES, int MB, int NB, int WR, int WC, int DA, int DB>
__global__ __launch_bounds__(WR *WC * 64) void grouped_rows_kernel(GroupedArgs g) {
  __shared__ __align__(16) uint8_t smem[(DA * MB + DB * NB) * 2 * kUnitBytes];
  const RaggedTiles tiles(g.offsets, g.N, g.S, 16 * MB, g.fill);
  grouped_rows<T, GX, LINES, MB, NB, WR, WC, DA, DB>(g, tiles, smem);
}

// The same with the tile shape taken here, from the groups' sizes that only the device knows: a
// group's last row tile costs about a full one, so which height wastes least goes by them.
// Rounds of a CU times the time of a stage, in units of 50 ns as measured with every CU busy (all of them some 6% less
// since the second wave of a SIMD copies between its products).  Four tile bodies
// in one kernel spill 39 vector registers in the rows' gradient and 2 in the forward.
template <bool GX, bool LINES> __global__ __launch_bounds__(512) void grouped_shapes_kernel(GroupedArgs g) {
  __shared__ __align__(16) uint8_t smem[160 * 1024];
  const int cols = GX ? g.K : g.M;
  const int heights[3] = {192, 256, 320};
  int tiles[3];
  RaggedTiles::count(g.offsets, g.N, g.S, heights, tiles, g.fill);
  const int slots = static_cast<int>(gridDim.x);
  auto cost = [&](int h, int width, int stage) {
    const long long items = static_cast<long long>(tiles[h]) * ((cols + width - 1) / width);
    return (items + slots - 1) / slots * stage;
  };
  const long long c192 = cost(0, 192, 28), c192w = cost(0, 256, 35), c256 = cost(1, 256, 42), c320 = cost(2, 192, 41);
  const long long best = min(min(c192, c192w), min(c256, c320));
  if (best == c256)
    grouped_rows<bf16_t, GX, LINES, 16, 16, 4, 2, 2, 3>(g, RaggedTiles(g.offsets, g.N, g.S, 256, g.fill), smem);
  else if (best == c320)
    grouped_rows<bf16_t, GX, LINES, 20, 12, 4, 2, 2, 3>(g, RaggedTiles(g.offsets, g.N, g.S, 320, g.fill), smem);
  else if (best == c192)
    grouped_rows<bf16_t, GX, LINES, 12, 12, 4, 2, 3, 3>(g, RaggedTiles(g.offsets, g.N, g.S, 192, g.fill), smem);
  else
    grouped_rows<bf16_t, GX, LINES, 12, 16, 4, 2, 2, 3>(g, RaggedTiles(g.offsets, g.N, g.S, 192, g.fill), smem);
}

// Weights' gradient: tile = 16 MB rows x 16 NB columns of one group's dw.  MATS = 2: of both matrices of a gated
// block, whose sums share x (rows2, out2 of GroupedArgs; the second matrix's partial sums lie behind the first's).
template <typename T, bool LINES, int MATS, int MB, int NB, int WR, int WC, int DA, int DB>
__global__ __launch_bounds__(WR *WC * 64) void grouped_weights_kernel(GroupedArgs g) {
  constexpr int BM = 16 * MB, BN = 16 * NB;
  __shared__ __align__(16) uint8_t smem[(DA * MB + DB * NB) * 2 * kUnitBytes];
  const int nM = (g.M + BM - 1) / BM, nN = (g.K + BN - 1) / BN, one = nM * nN, per = MATS * one;
  const RaggedTiles tiles(g.offsets, g.N, g.S, g.chunk, false, true);
  // The tiles' work goes by their group's rows, so a workgroup takes every gridDim-th of all tiles (a run of them for each
  // XCD, as in Share, leaves the XCD of the largest group the last by far: both gradients of 256 groups of 512 x 2048
  // with 16384 rows, a fifth of them in one, 365 us and 308 so).  Side by side on an XCD are consecutive ones, which share
  // a group's rows; those that do not fill a round go to the XCDs in turn.
  const int grid = static_cast<int>(gridDim.x), block = static_cast<int>(blockIdx.x), self = (block & 7) * (grid >> 3) + (block >> 3);
  const long long all = static_cast<long long>(tiles.total) * per, rounds = all / grid, mine = rounds + (block < all % grid);
  using S = DenseTile<T, true, true, MB, NB, WR, WC, DA, DB>;
  auto ref = [&](const Item &it, int) {
    const int mat = MATS == 1 ? 0 : it.tile >= one, tile = MATS == 1 ? it.tile : it.tile - mat * one;
    const int m0 = tile / nN * BM, c0 = tile % nN * BN;
    const size_t at = static_cast<size_t>(m0) * g.K + c0, size = static_cast<size_t>(g.M) * g.K;
    typename S::Ref t;
    t.a.p[0] = static_cast<const T *>(mat ? g.rows2 : g.rows) + static_cast<size_t>(it.row0) * g.M + m0;
    t.b.p[0] = static_cast<const T *>(g.other) + static_cast<size_t>(it.row0) * g.K + c0;
    t.out = static_cast<T *>(mat ? g.out2 : g.out) + static_cast<size_t>(it.group) * size + at;
    t.part = it.split >= 0 ? g.part + static_cast<size_t>(mat * g.splits + it.split) * size + at : nullptr;
    t.rows = min(BM, g.M - m0);
    t.cols = min(BN, g.K - c0);
    t.klen = it.rows;
    t.rot = 0;
    t.once = false;
    return t;
  };
  for (long long done = 0; done < mine; done += kItems) {
    const int n = static_cast<int>(min(mine - done, static_cast<long long>(kItems)));
    const long long j = min(done + (threadIdx.x & 63), mine - 1), i = j * grid + (j < rounds ? self : block);
    const RaggedTile t = tiles.find(static_cast<int>(i / per));
    // offsets that do not ascend can make more parts than there is room for: those go to the last
    const int slot = t.only ? -1 : min(max(t.slot, 0), g.splits - 1);
    __syncthreads();  // every wave is done with the rings
    grouped_items<S>(Item{max(t.group, 0), t.row0, t.rows, static_cast<int>(i % per), 0, slot}, n, g.M, g.K, smem, ref,
                     StoreTile<T, LINES, S>{static_cast<size_t>(g.K)});
  }
}

// dw of the groups of more than `chunk` rows: their parts' sum in order, 16 bytes of dw a thread.  Workgroups
// (x, y, z): the y-th such group, if there is one, of matrix z.
template <typename T> __global__ __launch_bounds__(256) void grouped_weights_join_kernel(GroupedArgs g) {
  constexpr int E = kChunkElems<T>;
  const int lane = threadIdx.x & 63, mat = static_cast<int>(blockIdx.z);
  int nth = static_cast<int>(blockIdx.y), slot = 0, group = -1, parts = 0;
  for (int e0 = 0; e0 < g.N && group < 0; e0 += 64) {
    const int e = e0 + lane;
    int n = 0;
    if (e < g.N) {
      const int lo = min(max(g.offsets[e], 0), g.S), hi = min(max(g.offsets[e + 1], 0), g.S);
      if (hi > lo) n = static_cast<int>((static_cast<uint32_t>(hi - lo) + g.chunk - 1u) / static_cast<uint32_t>(g.chunk));
    }
    unsigned long long many = __ballot(n > 1);
    while (many) {  // wave-uniform
      const int l = __ffsll(static_cast<long long>(many)) - 1, m = __builtin_amdgcn_readlane(n, l);
      if (nth-- == 0) {
        group = e0 + l;
        parts = m;
        break;
      }
      slot += m;
      many &= many - 1;
    }
  }
  if (group < 0) return;
  const size_t size = static_cast<size_t>(g.M) * g.K;
  for (size_t i = (static_cast<size_t>(blockIdx.x) * 256 + threadIdx.x) * E; i < size;
       i += static_cast<size_t>(gridDim.x) * 256 * E) {
    float v[E];
#pragma unroll
    for (int j = 0; j < E; ++j) v[j] = 0.f;
    for (int s = 0; s < parts; ++s) {
      const float *p = g.part + static_cast<size_t>(mat * g.splits + min(max(slot + s, 0), g.splits - 1)) * size + i;
#pragma unroll
      for (int j = 0; j < E; j += 4) {
        const f32x4_t u = *reinterpret_cast<const f32x4_t *>(p + j);
#pragma unroll
        for (int k = 0; k < 4; ++k) v[j + k] += u[k];
      }
    }
    T *o = static_cast<T *>(mat ? g.out2 : g.out) + static_cast<size_t>(group) * size + i;
    if constexpr (E == 8)
      *reinterpret_cast<uint4 *>(o) =
          uint4{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
    else
      *reinterpret_cast<f32x4_t *>(o) = f32x4_t{v[0], v[1], v[2], v[3]};
  }
}

// out = the parts' sum in order, for the rows of the groups (16 bytes of out a thread); the others get zeros
// with `fill`, or stay
template <typename T> __global__ __launch_bounds__(256) void grouped_join_kernel(GroupedArgs g, size_t total, int cols) {
  constexpr int E = kChunkElems<T>;
  const int r0 = min(max(g.offsets[0], 0), g.S);
  const size_t first = static_cast<size_t>(r0) * cols;
  const size_t last = static_cast<size_t>(min(max(g.offsets[g.N], r0), g.S)) * cols;
  for (size_t i = (static_cast<size_t>(blockIdx.x) * 256 + threadIdx.x) * E; i < total;
       i += static_cast<size_t>(gridDim.x) * 256 * E) {
    float v[E];
#pragma unroll
    for (int j = 0; j < E; ++j) v[j] = 0.f;
    if (i >= first && i < last) {
#pragma unroll 4
      for (int s = 0; s < g.splits; ++s) {
        const float *p = g.part + s * total + i;
#pragma unroll
        for (int j = 0; j < E; j += 4) {
          const f32x4_t u = *reinterpret_cast<const f32x4_t *>(p + j);
#pragma unroll
          for (int k = 0; k < 4; ++k) v[j + k] += u[k];
        }
      }
    } else if (!g.fill) {
      continue;
    }
    T *o = static_cast<T *>(g.out) + i;
    if constexpr (E == 8)
      *reinterpret_cast<uint4 *>(o) =
          uint4{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
    else
      *reinterpret_cast<f32x4_t *>(o) = f32x4_t{v[0], v[1], v[2], v[3]};
  }
}

using Tile64 = TileShape<4, 4, 2, 2, 4, 4>;     // bf16: few tiles, deep rings
using Tile64x128 = TileShape<4, 8, 2, 2, 3, 3>;  // bf16: a few rows a group
using Tile128 = TileShape<8, 8, 2, 2, 2, 3>;     // bf16
using Tile256 = TileShape<16, 16, 4, 2, 2, 2>;   // bf16, weights' gradient
using TileF32 = TileShape<2, 4, 2, 2, 3, 3>;     // fp32
using TileF32Weights = TileShape<4, 4, 2, 2, 3, 3>;

enum class Kind { k64, k64x128, k128, kLarge, kF32 };

struct Plan {
  Kind kind;
  int splits;         // parts of the reduction (weights' gradient: room for so many parts of groups)
  size_t part_elems;  // of one part
  int chunk;          // weights' gradient: most rows of a part
};

// Which kernel for the forward and the rows' gradient.  us on 128 groups of 768 x 2048 (forward):
//   rows a group               2    16    48    96   128   256  1024
//   128 x 128 (two a CU)      67    74    77    86   117   169   531
//   large (best of its four)  65    76    79    86    92   127   407
// and 16 groups of 1024 x 1024 with 1, 16, 128 and 512 rows: 64 x 64 12.8, 14.2, -, -; 128 x 128 15.2, 16.4, 20, 25;
// large 17, 18, 23, 31.  Few rows a group, where its weights' way from memory bounds all of them: 64 x 128 tiles with
// deeper rings, 128 groups of 2048 x 768 with 2, 16, 32 rows 63, 70, 72.6 against 68, 71, 73.7 with 128 x 128;
// with 48 rows of the table's 84 against 73.
// So: 64 x 64 tiles while they are at most a round, 64 x 128 up to 32 rows a group, the large shapes past 80 for work
// of at least a round of 128 x 128 tiles.
Plan plan_rows(const GroupedArgs &g, bool grad, bool bf16) {
  const int cols = grad ? g.K : g.M, klen = grad ? g.M : g.K;
  const size_t elems = static_cast<size_t>(g.S) * cols;
  if (!bf16) {
    const long long items = about_tiles(g.S, g.N, TileF32::TM) * tiles_of(cols, TileF32::TN);
    return {Kind::kF32, pick_splits(items, kCUs * TileF32::PER_CU, tiles_of(klen, 32), elems, 0.6), elems};
  }
  const long long small = about_tiles(g.S, g.N, Tile64::TM) * tiles_of(cols, Tile64::TN);
  if (small <= kCUs * Tile64::PER_CU)
    return {Kind::k64, pick_splits(small, kCUs * Tile64::PER_CU, tiles_of(klen, 64), elems, 0.45), elems};
  if (g.S <= 32ll * g.N) return {Kind::k64x128, 1, elems};
  const long long items = about_tiles(g.S, g.N, Tile128::TM) * tiles_of(cols, Tile128::TN);
  const bool large = g.S > 80ll * g.N && items >= kCUs * Tile128::PER_CU;
  return {large ? Kind::kLarge : Kind::k128, 1, elems};
}

// ... and for the weights' gradient.  128 groups of 768 x 2048 and 128 rows: 256 x 256 tiles 105 us, 128 x 128 134
// (the former spill 12 registers and wait for each tile's stores).
// A group of more than p.chunk rows is summed in parts of at most that many, which a second launch adds: a few
// long groups would otherwise be a few workgroups' work.  Parts are four times the mean group (2048 rows at least),
// so that their sums take no more room than dw itself (bf16); or fewer rows where all tiles together
// would leave CUs idle, as far as the time of their stages pays for the launch and the traffic (us; 74 groups of
// 464 x 256, the largest a quarter of 39997 rows: 122 us whole, 54 in parts).
Plan plan_weights(const GroupedArgs &g, bool bf16) {
  const size_t elems = static_cast<size_t>(g.M) * g.K;
  const long long mean = (static_cast<long long>(g.S) + g.N - 1) / g.N;
  const int mats = g.out2 ? 2 : 1;
  auto tiles = [&](int t) { return mats * tiles_of(g.M, t) * tiles_of(g.K, t); };
  Plan p{Kind::kF32, 0, elems};
  long long one = tiles(64), slots = kCUs * TileF32Weights::PER_CU;
  double stage = 1.2;  // of 64 rows, us
  if (bf16) {
    if (g.N * tiles(64) <= kCUs * Tile64::PER_CU) {
      p.kind = Kind::k64;
      slots = kCUs * Tile64::PER_CU;
      stage = 0.45;
    } else if (g.N * tiles(256) >= kCUs) {
      p.kind = Kind::kLarge;
      one = tiles(256);
      slots = kCUs;
      stage = 2.1;
    } else {
      p.kind = Kind::k128;
      one = tiles(128);
      slots = kCUs * Tile128::PER_CU;
    }
  }
  long long chunk = std::max(4 * mean, 2048ll);
  if (g.N * one < slots) {
    double least = static_cast<double>(mean) / 64 * stage;
    for (long long c = mean / 2; c >= 128 && tiles_of(g.S, static_cast<int>(c)) * one <= slots; c /= 2) {
      const double t = static_cast<double>(c) / 64 * stage + 4.5 + 2e-6 * mats * (g.S / c) * static_cast<double>(elems);
      if (t < least) {
        least = t;
        chunk = c;
      }
    }
  }
  p.chunk = static_cast<int>(std::min<long long>((chunk + 63) / 64 * 64, 1 << 30));
  p.splits = g.S <= p.chunk ? 0 : static_cast<int>(2ll * g.S / p.chunk);
  return p;
}

// whether every row of the result is whole 128-byte lines (see put16)
bool whole_lines(const GroupedArgs &g, int cols, int es) {
  return cols * es % 128 == 0 && reinterpret_cast<uintptr_t>(g.out) % 128 == 0;
}

template <typename T, bool GX, class Sh> void launch_rows_shape(const GroupedArgs &g, int cols, hipStream_t s) {
  const long long items = ragged_max_tiles(g.S, g.N, Sh::TM) * tiles_of(cols, Sh::TN) * g.splits;
  auto launch = [&](auto kernel) { kernel<<<grouped_grid(items, Sh::PER_CU), Sh::THREADS, 0, s>>>(g); };
  if (whole_lines(g, cols, sizeof(T)))
    launch(grouped_rows_kernel<T, GX, true, Sh::MB, Sh::NB, Sh::WR, Sh::WC, Sh::DA, Sh::DB>);
  else
    launch(grouped_rows_kernel<T, GX, false, Sh::MB, Sh::NB, Sh::WR, Sh::WC, Sh::DA, Sh::DB>);
}

template <typename T, class Sh> void launch_weights_shape(const GroupedArgs &g, hipStream_t s) {
  const int mats = g.out2 ? 2 : 1;
  const long long items = (g.N + g.splits) * tiles_of(g.M, Sh::TM) * tiles_of(g.K, Sh::TN) * mats;
  auto launch = [&](auto kernel) { kernel<<<grouped_grid(items, Sh::PER_CU), Sh::THREADS, 0, s>>>(g); };
  const bool lines = whole_lines(g, g.K, sizeof(T)) && reinterpret_cast<uintptr_t>(g.out2) % 128 == 0;
  if (mats == 1 && lines)
    launch(grouped_weights_kernel<T, true, 1, Sh::MB, Sh::NB, Sh::WR, Sh::WC, Sh::DA, Sh::DB>);
  else if (mats == 1)
    launch(grouped_weights_kernel<T, false, 1, Sh::MB, Sh::NB, Sh::WR, Sh::WC, Sh::DA, Sh::DB>);
  else if (lines)
    launch(grouped_weights_kernel<T, true, 2, Sh::MB, Sh::NB, Sh::WR, Sh::WC, Sh::DA, Sh::DB>);
  else
    launch(grouped_weights_kernel<T, false, 2, Sh::MB, Sh::NB, Sh::WR, Sh::WC, Sh::DA, Sh::DB>);
}

template <bool GX> hipError_t launch_rows(GroupedArgs g, bool bf16, hipStream_t s) {
  const int cols = GX ? g.K : g.M;
  const Plan p = plan_rows(g, GX, bf16);
  g.splits = p.splits;
  switch (p.kind) {
    case Kind::k64: launch_rows_shape<bf16_t, GX, Tile64>(g, cols, s); break;
    case Kind::k64x128: launch_rows_shape<bf16_t, GX, Tile64x128>(g, cols, s); break;
    case Kind::k128: launch_rows_shape<bf16_t, GX, Tile128>(g, cols, s); break;
    case Kind::kLarge:
      if (whole_lines(g, cols, 2))
        grouped_shapes_kernel<GX, true><<<kCUs, 512, 0, s>>>(g);
      else
        grouped_shapes_kernel<GX, false><<<kCUs, 512, 0, s>>>(g);
      break;
    case Kind::kF32: launch_rows_shape<float, GX, TileF32>(g, cols, s); break;
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.splits == 1) return e;
  return launch_grouped_join(g, cols, bf16, s);
}

}  // namespace

size_t grouped_workspace_bytes(const GroupedArgs &g, bool weights, bool grad, bool bf16) {
  if (g.S <= 0 && !weights) return 0;
  const Plan p = weights ? plan_weights(g, bf16) : plan_rows(g, grad, bf16);
  return p.splits > 1 ? p.splits * p.part_elems * (g.out2 ? 2 : 1) * sizeof(float) : 0;
}

hipError_t launch_grouped_join(const GroupedArgs &g, int cols, bool bf16, hipStream_t s) {
  const size_t total = static_cast<size_t>(g.S) * cols;
  const size_t blocks = (total / (bf16 ? 8 : 4) + 255) / 256;
  const unsigned grid = static_cast<unsigned>(std::min<size_t>(std::max<size_t>(blocks, 1), 8 * kCUs));
  if (bf16)
    grouped_join_kernel<bf16_t><<<grid, 256, 0, s>>>(g, total, cols);
  else
    grouped_join_kernel<float><<<grid, 256, 0, s>>>(g, total, cols);
  return hipGetLastError();
}

hipError_t launch_grouped_rows(const GroupedArgs &g, bool grad, bool bf16, hipStream_t stream) {
  if (g.S <= 0) return hipSuccess;
  return grad ? launch_rows<true>(g, bf16, stream) : launch_rows<false>(g, bf16, stream);
}

hipError_t launch_grouped_weights(const GroupedArgs &args, bool bf16, hipStream_t stream) {
  GroupedArgs g = args;
  const Plan p = plan_weights(g, bf16);
  g.splits = p.splits;
  g.chunk = p.chunk;
  switch (p.kind) {
    case Kind::k64: launch_weights_shape<bf16_t, Tile64>(g, stream); break;
    case Kind::kLarge: launch_weights_shape<bf16_t, Tile256>(g, stream); break;
    case Kind::kF32: launch_weights_shape<float, TileF32Weights>(g, stream); break;
    default: launch_weights_shape<bf16_t, Tile128>(g, stream); break;
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.splits == 0) return e;
  // at most S / chunk groups have more rows than that
  const size_t blocks = (p.part_elems / (bf16 ? 8 : 4) + 255) / 256;
  const dim3 grid(static_cast<unsigned>(std::min<size_t>(blocks, 64)), static_cast<unsigned>(std::min(g.N, g.S / g.chunk)),
                  g.out2 ? 2 : 1);
  if (bf16)
    grouped_weights_join_kernel<bf16_t><<<grid, 256, 0, stream>>>(g);
  else
    grouped_weights_join_kernel<float><<<grid, 256, 0, stream>>>(g);
  return hipGetLastError();
}

}  // namespace ace
