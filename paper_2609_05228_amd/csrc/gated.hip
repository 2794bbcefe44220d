// The gated feed-forward block of the experts, grouped by expert with ragged sizes, and its gradient:
//   g[r] = w_gate[e] x[r],  u[r] = w_up[e] x[r],  a[r] = act(g[r]) * u[r]      for the rows r of group e
//   dg = da * u * act'(g),  du = da * act(g)
//   dx[r] = w_gate[e]^T dg[r] + w_up[e]^T du[r]
//   dw_gate[e] = sum over the rows r of e: dg[r] x[r]^T, dw_up alike with du
// act is SiLU, g / (1 + e^-g), or GELU, g Phi(g) with the normal distribution's Phi.
//
// Both projections are one tile (grouped_tile.h): its 16-column blocks alternate between
// the two matrices, so a lane's accumulators hold g and u of the same four features and the
// activation and the product happen in registers: x is read once, and g and u leave the chip only where they are kept,
// or where too few tiles fill the CUs and the reduction is in parts, whose fp32 sums of both go through the workspace to a
// second launch (gated_join_kernel).  The gradient takes dg and du either from the kept g and u, or in the
// epilogue of the same product computed again; both are rounded to the tensors' type there,
// since the two products behind them run on matrix cores of that type.  dx is one
// product with a reduction of two segments (dg with w_gate, then du with w_up), summed in the same
// accumulators and rounded once; both gradients of the weights are one launch, where the tiles of a group
// share its rows of x in an XCD's L2.
//
// What bounds it, on 128 groups of 768 x 2048 in bf16: the weights' way from and to memory.  The projections of 8 rows take
// 13.6 us (3.6 TB/s of what the call needs), of 32768 with g and u kept 252 us (4.3 TB/s at 0.82 PFLOP/s); the
// gradient of 16384 from kept projections 430 us (4.2 TB/s: 24 dg and du, 170 dx, 210 to 240 the weights').
#include "gated_tile.h"

namespace ace {

namespace {

// Both projections in tiles of 16 MB rows of one group x 8 NB features: the whole work of a workgroup.  KS > 1 (shapes of
// one wave): its KS waves split the reduction of each tile.
template <typename T, bool LINES, int MB, int NB, int WR, int WC, int DA, int DB, int KS = 1>
__device__ __forceinline__ void gated_rows(const GatedArgs &g, const RaggedTiles &tiles, uint8_t *smem) {
  using S = DenseTile<T, false, false, MB, NB, WR, WC, DA, DB, 2>;
  static_assert(sizeof(T) == 4 || S::NW % 4 == 0, "a wave holds whole pairs of feature blocks");
  constexpr int BF = 8 * NB;
  const int nN = (g.M + BF - 1) / BF, per = nN * g.splits;
  const Share share(static_cast<long long>(tiles.total) * per);
  auto ref = [&](const Item &it, int) {
    const int f0 = it.tile * BF;
    const int klen = it.group < 0 ? 0 : g.K;
    const Part k = KS > 1 ? part_of<S::A::BK>(klen, __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), KS)
                          : part_of<S::A::BK>(klen, it.split, g.splits);
    const size_t w = (static_cast<size_t>(max(it.group, 0)) * g.M + f0) * g.K + k.k0;
    GatedRef<S> t;
    t.a.p[0] = static_cast<const T *>(g.x) + static_cast<size_t>(it.row0) * g.K + k.k0;
    t.b.p[0] = static_cast<const T *>(g.w_gate) + w;
    t.b.p[1] = static_cast<const T *>(g.w_up) + w;
    t.at = static_cast<size_t>(it.row0) * g.M + f0;
    t.out = nullptr;
    t.part = g.splits > 1 ? g.part + 2 * static_cast<size_t>(it.split) * g.S * g.M + t.at : nullptr;
    t.rows = it.rows;
    t.cols = min(BF, g.M - f0);
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
    const Item item{t.group, t.row0, t.rows, q % nN, t.only, q / nN};
    __syncthreads();  // every wave is done with the rings
    if constexpr (KS > 1) {
      const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
      grouped_items<S>(item, n, g.K, g.K, smem + wave * S::LDS, ref,
                       JoinStore<S, KS, GatedStore<T, LINES, S>>{{g}, smem + KS * S::LDS, 0});
    } else {
      grouped_items<S>(item, n, g.K, g.K, smem, ref, GatedStore<T, LINES, S>{g});
    }
  }
}

// Few rows: tiles of 16, the reduction over the workgroup's four waves
constexpr int kSplitWaves = 4;
template <bool LINES> __global__ __launch_bounds__(64 * kSplitWaves) void gated_few_kernel(GatedArgs g) {
  using S = DenseTile<bf16_t, false, false, 1, 4, 1, 1, 3, 3, 2>;
  using J = JoinStore<S, kSplitWaves, GatedStore<bf16_t, LINES, S>>;
  __shared__ __align__(16) uint8_t smem[kSplitWaves * S::LDS + J::LDS];
  gated_rows<bf16_t, LINES, 1, 4, 1, 1, 3, 3, kSplitWaves>(g, RaggedTiles(g.offsets, g.N, g.S, 16, g.fill), smem);
}

template <typename T, bool LINES, int MB, int NB, int WR, int WC, int DA, int DB>
__global__ __launch_bounds__(WR *WC * 64) void gated_rows_kernel(GatedArgs g) {
  __shared__ __align__(16) uint8_t smem[(DA * MB + DB * NB) * 2 * kUnitBytes];
  gated_rows<T, LINES, MB, NB, WR, WC, DA, DB>(g, RaggedTiles(g.offsets, g.N, g.S, 16 * MB, g.fill), smem);
}

// The same with the tile's height taken here, from the groups' sizes that only the device knows: a group's last row tile
// costs about a full one.  Rounds of a CU times the time of a stage in units of 50 ns, measured on 128 groups of 768 x
// 2048 with 128 and 256 rows (the weights' way from memory in it): 192 rows 1.5 us, 256 1.8, 320 2.5.  32768 rows with g
// and u kept: 286, 312 and 264 us; 16384 rows without: 155, 165 and 176.
template <bool LINES> __global__ __launch_bounds__(512) void gated_shapes_kernel(GatedArgs g) {
  __shared__ __align__(16) uint8_t smem[160 * 1024];
  const int heights[3] = {192, 256, 320};
  int tiles[3];
  RaggedTiles::count(g.offsets, g.N, g.S, heights, tiles, g.fill);
  const int slots = static_cast<int>(gridDim.x);
  auto cost = [&](int h, int stage) {
    const long long items = static_cast<long long>(tiles[h]) * ((g.M + 127) / 128);
    return (items + slots - 1) / slots * stage;
  };
  const long long c192 = cost(0, 30), c256 = cost(1, 36), c320 = cost(2, 50);
  if (c192 <= min(c256, c320))
    gated_rows<bf16_t, LINES, 12, 16, 4, 2, 2, 3>(g, RaggedTiles(g.offsets, g.N, g.S, 192, g.fill), smem);
  else if (c256 <= c320)
    gated_rows<bf16_t, LINES, 16, 16, 4, 2, 2, 3>(g, RaggedTiles(g.offsets, g.N, g.S, 256, g.fill), smem);
  else
    gated_rows<bf16_t, LINES, 20, 16, 4, 2, 2, 2>(g, RaggedTiles(g.offsets, g.N, g.S, 320, g.fill), smem);
}

// What the epilogue does, from the fp32 parts of g and u (summed in order) or the kept g and u: 4 features a thread.  Bound
// by memory: dg and du of 16384 rows of 768 in bf16 24 us, 5.2 TB/s.
// Rows of no group: zeros into a, g and u with `fill`, else they stay (dg and du of them are never read).
template <typename T, int ACT> __global__ __launch_bounds__(256) void gated_join_kernel(GatedArgs g) {
  const size_t total = static_cast<size_t>(g.S) * g.M;
  const int r0 = min(max(g.offsets[0], 0), g.S);
  const size_t first = static_cast<size_t>(r0) * g.M, last = static_cast<size_t>(min(max(g.offsets[g.N], r0), g.S)) * g.M;
  for (size_t i = (static_cast<size_t>(blockIdx.x) * 256 + threadIdx.x) * 4; i < total;
       i += static_cast<size_t>(gridDim.x) * 256 * 4) {
    f32x4_t vg{0.f, 0.f, 0.f, 0.f}, vu = vg;
    if (i >= first && i < last) {
      if (g.splits > 1) {
#pragma unroll 4
        for (int s = 0; s < g.splits; ++s) {
          const float *p = g.part + 2 * s * total + i;
          const f32x4_t a = *reinterpret_cast<const f32x4_t *>(p), b = *reinterpret_cast<const f32x4_t *>(p + total);
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            vg[q] += a[q];
            vu[q] += b[q];
          }
        }
      } else {
        load4(static_cast<const T *>(g.g) + i, vg);
        load4(static_cast<const T *>(g.u) + i, vu);
      }
    } else if (!g.fill) {
      continue;
    }
    f32x4_t f, slope;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      float d;
      f[q] = Activation<T, ACT>::template both<true>(vg[q], d);
      slope[q] = d;
    }
    if (g.da) {
      f32x4_t da, dg, du;
      load4(static_cast<const T *>(g.da) + i, da);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        dg[q] = da[q] * vu[q] * slope[q];
        du[q] = da[q] * f[q];
      }
      store4(static_cast<T *>(g.dg) + i, dg);
      store4(static_cast<T *>(g.du) + i, du);
      continue;
    }
    if (g.g) {
      store4(static_cast<T *>(g.g) + i, vg);
      store4(static_cast<T *>(g.u) + i, vu);
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) f[q] *= vu[q];
    store4(static_cast<T *>(g.a) + i, f);
  }
}

// dx: tiles of 16 MB rows x 16 NB columns, reduced over the features of the gate, then of the up projection
template <typename T, bool LINES, int MB, int NB, int WR, int WC, int DA, int DB>
__global__ __launch_bounds__(WR *WC * 64) void gated_grad_x_kernel(GatedArgs g) {
  using S = DenseTile<T, false, true, MB, NB, WR, WC, DA, DB, 1, 2>;
  constexpr int BN = 16 * NB;
  __shared__ __align__(16) uint8_t smem[(DA * MB + DB * NB) * 2 * kUnitBytes];
  const RaggedTiles tiles(g.offsets, g.N, g.S, 16 * MB, g.fill);
  const int nN = (g.K + BN - 1) / BN, per = nN * g.splits;
  const Share share(static_cast<long long>(tiles.total) * per);
  auto ref = [&](const Item &it, int seg) {
    const int c0 = it.tile * BN;
    const Part k = part_of<S::A::BK>(it.group < 0 ? 0 : g.M, it.split, g.splits);
    typename S::Ref t;
    t.a.p[0] = static_cast<const T *>(seg ? g.du : g.dg) + static_cast<size_t>(it.row0) * g.M + k.k0;
    t.b.p[0] = static_cast<const T *>(seg ? g.w_up : g.w_gate) +
               (static_cast<size_t>(max(it.group, 0)) * g.M + k.k0) * g.K + c0;
    t.out = static_cast<T *>(g.dx) + static_cast<size_t>(it.row0) * g.K + c0;
    t.part = g.splits > 1 ? g.part + (static_cast<size_t>(it.split) * g.S + it.row0) * g.K + c0 : nullptr;
    t.rows = it.rows;
    t.cols = min(BN, g.K - c0);
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
    grouped_items<S>(Item{t.group, t.row0, t.rows, q % nN, t.only, q / nN}, n, g.M, g.K, smem, ref,
                     StoreTile<T, LINES, S>{static_cast<size_t>(g.K)});
  }
}

using Gated64 = TileShape<4, 4, 4, 1, 4, 4>;     // bf16: few tiles, deep rings
using GradX64 = TileShape<4, 4, 2, 2, 4, 4>;
using Gated64x128 = TileShape<4, 8, 2, 2, 3, 3>;  // bf16: a few rows a group
using Gated128 = TileShape<8, 8, 2, 2, 2, 3>;     // bf16
using GradX256 = TileShape<16, 16, 4, 2, 2, 3>;   // bf16
using GatedF32 = TileShape<2, 4, 2, 2, 3, 3>;      // fp32
using GatedF32Many = TileShape<2, 4, 2, 2, 2, 2>;  // fp32: more than a round

enum class Kind { kFew, k64, k64x128, k128, kLarge, kF32, kF32Many };
struct Plan {
  Kind kind;
  int splits;
};

// bf16: 64 x 64 tiles while they are at most a round, 64 x 128 up to 32 rows a group, then 128 x 128, and the large shapes
// past 40 rows a group where they fill most CUs (projections of 128 groups of 768 x 2048, kernel times with 32, 48, 96
// and 128 rows: 64 x 128 131, 142, 204, 233 us; 128 x 128 132, 135, 147, 205; large 129, 131, 134, 140; one group of 2048 x
// 2048 with 2048 rows, 128 large tiles: 128 x 128 44, large 51; 16 groups of 1024 x 1024 with 4096, about 192: 41.5 and
// 32.8).
// Kernel and parts of the reduction for S rows in N groups by `cols` columns (both projections' features, or dx's), over
// klen, with `elems` sums in a part.  fp32: the matrix cores bound all but the smallest, so past a round of the CUs six
// workgroups a CU with rings of two stages, else four with three (kernel times of the projections: 2069 rows in 32 groups of
// 512 x 1024 70.7 us against 75.7, 8192 rows in 16 190 against 201, 64 rows in 8 of 512 x 256 11.5 against 10.4).
Plan plan_rows(long long S, long long N, int cols, long long klen, size_t elems, bool bf16) {
  if (!bf16) {
    const long long items = about_tiles(S, N, GatedF32::TM) * tiles_of(cols, GatedF32::TN);
    if (items > kCUs * GatedF32::PER_CU) return {Kind::kF32Many, 1};
    return {Kind::kF32, pick_splits(items, kCUs * GatedF32::PER_CU, tiles_of(klen, 32), elems, 0.6)};
  }
  const long long small = about_tiles(S, N, Gated64::TM) * tiles_of(cols, Gated64::TN);
  if (small <= kCUs * Gated64::PER_CU)
    return {Kind::k64, pick_splits(small, kCUs * Gated64::PER_CU, tiles_of(klen, 64), elems, 0.45)};
  if (S <= 32 * N) return {Kind::k64x128, 1};
  const bool large = S > 40 * N && about_tiles(S, N, 256) * tiles_of(cols, 256) >= kCUs * 5 / 8;
  return {large ? Kind::kLarge : Kind::k128, 1};
}
Plan plan_gated(const GatedArgs &g, bool bf16) {
  // a few rows a group: tiles of 16 with the reduction over the waves of a workgroup, against larger ones with parts of the
  // reduction and a launch that adds them (kernel times on 128 groups of 768 x 2048: 8 rows 13.7 us against 21.4, 256 rows
  // 113 against 119, 1024 rows 126 against 123; one group of 4096 x 4096: 16 rows 18.1 against 21.4, 64 rows of half of
  // it 23 against 20.4)
  if (bf16 && (g.S <= 4ll * g.N || (g.S <= 16ll * g.N && about_tiles(g.S, g.N, 16) * tiles_of(g.M, 32) <= 2 * kCUs)))
    return {Kind::kFew, 1};
  return plan_rows(g.S, g.N, 2 * g.M, g.K, 2 * static_cast<size_t>(g.S) * g.M, bf16);
}
Plan plan_grad_x(const GatedArgs &g, bool bf16) {
  return plan_rows(g.S, g.N, g.K, 2ll * g.M, static_cast<size_t>(g.S) * g.K, bf16);
}

bool lines(const void *p) { return reinterpret_cast<uintptr_t>(p) % 128 == 0; }

// whether rows of all that the projections' kernel writes are whole 128-byte lines (see put16)
bool gated_lines(const GatedArgs &g, size_t es) {
  return g.M * es % 128 == 0 && lines(g.a) && lines(g.g) && lines(g.u) && lines(g.dg) && lines(g.du);
}

template <typename T, class Sh> void launch_gated_shape(const GatedArgs &g, hipStream_t s) {
  const long long items = ragged_max_tiles(g.S, g.N, Sh::TM) * tiles_of(g.M, Sh::TN / 2) * g.splits;
  auto launch = [&](auto kernel) { kernel<<<grouped_grid(items, Sh::PER_CU), Sh::THREADS, 0, s>>>(g); };
  if (gated_lines(g, sizeof(T)))
    launch(gated_rows_kernel<T, true, Sh::MB, Sh::NB, Sh::WR, Sh::WC, Sh::DA, Sh::DB>);
  else
    launch(gated_rows_kernel<T, false, Sh::MB, Sh::NB, Sh::WR, Sh::WC, Sh::DA, Sh::DB>);
}

template <typename T, class Sh> void launch_grad_x_shape(const GatedArgs &g, hipStream_t s) {
  const long long items = ragged_max_tiles(g.S, g.N, Sh::TM) * tiles_of(g.K, Sh::TN) * g.splits;
  auto launch = [&](auto kernel) { kernel<<<grouped_grid(items, Sh::PER_CU), Sh::THREADS, 0, s>>>(g); };
  if (g.K * sizeof(T) % 128 == 0 && lines(g.dx))
    launch(gated_grad_x_kernel<T, true, Sh::MB, Sh::NB, Sh::WR, Sh::WC, Sh::DA, Sh::DB>);
  else
    launch(gated_grad_x_kernel<T, false, Sh::MB, Sh::NB, Sh::WR, Sh::WC, Sh::DA, Sh::DB>);
}

}  // namespace

hipError_t launch_gated_join(const GatedArgs &g, bool bf16, hipStream_t s) {
  const size_t blocks = (static_cast<size_t>(g.S) * g.M / 4 + 255) / 256;
  const unsigned grid = static_cast<unsigned>(std::min<size_t>(std::max<size_t>(blocks, 1), 8 * kCUs));
  auto launch = [&](auto kernel) { kernel<<<grid, 256, 0, s>>>(g); };
  if (bf16)
    g.act == kActSilu ? launch(gated_join_kernel<bf16_t, kActSilu>) : launch(gated_join_kernel<bf16_t, kActGelu>);
  else
    g.act == kActSilu ? launch(gated_join_kernel<float, kActSilu>) : launch(gated_join_kernel<float, kActGelu>);
  return hipGetLastError();
}

size_t gated_part_bytes(const GatedArgs &g, bool bf16) {
  const int n = g.S > 0 ? plan_gated(g, bf16).splits : 1;
  return n > 1 ? 2 * n * static_cast<size_t>(g.S) * g.M * sizeof(float) : 0;
}

size_t gated_grad_x_part_bytes(const GatedArgs &g, bool bf16) {
  const int n = g.S > 0 ? plan_grad_x(g, bf16).splits : 1;
  return n > 1 ? n * static_cast<size_t>(g.S) * g.K * sizeof(float) : 0;
}

hipError_t launch_gated(GatedArgs g, bool bf16, hipStream_t s) {
  if (g.S <= 0) return hipSuccess;
  const Plan p = plan_gated(g, bf16);
  g.splits = p.splits;
  switch (p.kind) {
    case Kind::kFew: {
      const unsigned grid = grouped_grid(ragged_max_tiles(g.S, g.N, 16) * tiles_of(g.M, 32), 1);
      if (gated_lines(g, 2))
        gated_few_kernel<true><<<grid, 64 * kSplitWaves, 0, s>>>(g);
      else
        gated_few_kernel<false><<<grid, 64 * kSplitWaves, 0, s>>>(g);
      break;
    }
    case Kind::k64: launch_gated_shape<bf16_t, Gated64>(g, s); break;
    case Kind::k64x128: launch_gated_shape<bf16_t, Gated64x128>(g, s); break;
    case Kind::k128: launch_gated_shape<bf16_t, Gated128>(g, s); break;
    case Kind::kLarge:
      if (gated_lines(g, 2))
        gated_shapes_kernel<true><<<kCUs, 512, 0, s>>>(g);
      else
        gated_shapes_kernel<false><<<kCUs, 512, 0, s>>>(g);
      break;
    case Kind::kF32: launch_gated_shape<float, GatedF32>(g, s); break;
    case Kind::kF32Many: launch_gated_shape<float, GatedF32Many>(g, s); break;
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.splits == 1) return e;
  return launch_gated_join(g, bf16, s);
}

hipError_t launch_gated_slopes(GatedArgs g, bool bf16, hipStream_t s) {
  if (g.S <= 0) return hipSuccess;
  g.splits = 1;
  return launch_gated_join(g, bf16, s);
}

hipError_t launch_gated_grad_x(GatedArgs g, bool bf16, hipStream_t s) {
  if (g.S <= 0) return hipSuccess;
  const Plan p = plan_grad_x(g, bf16);
  g.splits = p.splits;
  switch (p.kind) {
    case Kind::kFew:
    case Kind::k64: launch_grad_x_shape<bf16_t, GradX64>(g, s); break;
    case Kind::k64x128: launch_grad_x_shape<bf16_t, Gated64x128>(g, s); break;
    case Kind::k128: launch_grad_x_shape<bf16_t, Gated128>(g, s); break;
    case Kind::kLarge: launch_grad_x_shape<bf16_t, GradX256>(g, s); break;
    case Kind::kF32: launch_grad_x_shape<float, GatedF32>(g, s); break;
    case Kind::kF32Many: launch_grad_x_shape<float, GatedF32Many>(g, s); break;
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.splits == 1) return e;
  GroupedArgs j{};
  j.out = g.dx;
  j.offsets = g.offsets;
  j.S = g.S;
  j.N = g.N;
  j.fill = g.fill;
  j.splits = p.splits;
  j.part = g.part;
  return launch_grouped_join(j, g.K, bf16, s);
}

}  // namespace ace
