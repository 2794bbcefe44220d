// Microscaled 4-bit floating point (the format: mx4_tile.h): numbers into it and back, and products grouped by
// expert with weights in it.
//   quantise: e = floor(log2 of the block's largest) - 2, at least -127; numbers / 2^e go to the nearest of 0, .5, 1, 1.5,
//             2, 3, 4, 6 with their sign (ties to the even code, beyond 6 to 6); a block that holds a NaN or an
//             infinity stands for NaN
//   y[r] = w[e] x[r], and a[r] = act(w_gate[e] x[r]) * (w_up[e] x[r]), for the rows r of group e, x in bf16 or in 4 bits
#include "gated_tile.h"
#include "mx4_tile.h"

namespace ace {

namespace {

// largest absolute bits over the 4 lanes of a block
__device__ __forceinline__ uint32_t quad_max(uint32_t v) {
  v = max(v, static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(static_cast<int>(v), 0xB1, 0xf, 0xf, true)));  // lanes 1, 0, 3, 2
  return max(v, static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(static_cast<int>(v), 0x4E, 0xf, 0xf, true)));  // 2, 3, 0, 1
}

// 8 numbers of a lane
__device__ __forceinline__ void load8(const float *p, float (&v)[8]) {
  const f32x4_t a = reinterpret_cast<const f32x4_t *>(p)[0], b = reinterpret_cast<const f32x4_t *>(p)[1];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[i] = a[i];
    v[4 + i] = b[i];
  }
}
__device__ __forceinline__ void load8(const bf16_t *p, float (&v)[8]) {
  const uint4 b = *reinterpret_cast<const uint4 *>(p);
  const uint32_t w[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(w[i] << 16);
    v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}

// A part is 128 numbers of a row (the last may be short), taken by 16 lanes, 8 numbers each: 4 lanes a block, their four
// scales one dword.  WHOLE: rows are whole parts, so a part's place needs no division.  Bound by memory: 98304 rows of
// 2048 in bf16 94 us there and 86 back (4.3 and 5.9 TB/s; the results' non-temporal stores leave the caches clean for
// whoever comes next: 128 us there after a way back without them).  In fp32 a lane's result is two pieces of 16 bytes, each
// store half lines, and the hint pays all the same: 260 us back and 181 there, 242 and 222 without it.  Two or four parts a lane under way: slower (98, 96
// and 94, 99).
template <bool WHOLE> struct Mx4Part {
  size_t x;  // where the lane's numbers start; their codes at half of it
  bool in;
  __device__ __forceinline__ Mx4Part(const Mx4Convert &a, uint32_t i) {
    const uint32_t l16 = threadIdx.x & 15;
    if (WHOLE) {
      in = true;
      x = static_cast<size_t>(i) * 128 + 8 * l16;
    } else {
      const uint32_t row = i / a.parts, k = (i - row * a.parts) * 128 + 8 * l16;
      in = k < static_cast<uint32_t>(a.K);
      x = static_cast<size_t>(row) * a.K + k;
    }
  }
};

template <typename T, bool WHOLE> __global__ __launch_bounds__(256) void mx4_quantize_kernel(Mx4Convert a) {
  const uint32_t l16 = threadIdx.x & 15, step = gridDim.x * 16;
  for (uint32_t i = blockIdx.x * 16 + (threadIdx.x >> 4); i < a.total; i += step) {
    const Mx4Part<WHOLE> p(a, i);
    float v[8] = {};
    if (p.in) load8(static_cast<const T *>(a.x) + p.x, v);
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(v[j]) & 0x7fffffffu);
    const uint32_t e = quad_max(top) >> 23;
    const uint32_t s = e == 255 ? 255 : e < 2 ? 0 : e - 2;
    const float scale = __uint_as_float(s << 23);  // its exponent is all that the conversion takes
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[0], v[1], scale, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[2], v[3], scale, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[4], v[5], scale, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[6], v[7], scale, 3);
    if (s == 255) c = 0;
    if (p.in) *reinterpret_cast<uint32_t *>(a.codes + p.x / 2) = c;
    // lanes 0, 4, 8, 12 of the 16 hold the blocks' scales
    uint32_t four = p.in ? s << (8 * (l16 >> 2)) : 0;
    four |= static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(static_cast<int>(four), 0x124, 0xf, 0xf, true));  // row_ror:4
    four |= static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(static_cast<int>(four), 0x128, 0xf, 0xf, true));  // row_ror:8
    if (l16 == 0) reinterpret_cast<uint32_t *>(a.scales)[i] = four;
  }
}

template <typename T, bool WHOLE> __global__ __launch_bounds__(256) void mx4_dequantize_kernel(Mx4Convert a) {
  const uint32_t l16 = threadIdx.x & 15, step = gridDim.x * 16;
  for (uint32_t i = blockIdx.x * 16 + (threadIdx.x >> 4); i < a.total; i += step) {
    const Mx4Part<WHOLE> p(a, i);
    if (!p.in) continue;
    const uint32_t c = *reinterpret_cast<const uint32_t *>(a.codes + p.x / 2);
    const float scale = __uint_as_float(static_cast<uint32_t>(a.scales[static_cast<size_t>(i) * 4 + (l16 >> 2)]) << 23);
    T *o = static_cast<T *>(const_cast<void *>(a.x)) + p.x;
    if constexpr (sizeof(T) == 2) {
      put16<WHOLE>(o, __builtin_bit_cast(uint4, mx4_to_bf16(c, scale)));
    } else {
      typedef float f32x2_v __attribute__((ext_vector_type(2)));
      const f32x2_v v0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, scale, 0);
      const f32x2_v v1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, scale, 1);
      const f32x2_v v2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, scale, 2);
      const f32x2_v v3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, scale, 3);
      put16<WHOLE>(o, __builtin_bit_cast(uint4, f32x4_t{v0[0], v0[1], v1[0], v1[1]}));
      put16<WHOLE>(o + 4, __builtin_bit_cast(uint4, f32x4_t{v2[0], v2[1], v3[0], v3[1]}));
    }
  }
}

// Tiles of 16 MB rows of one group x 16 NB columns (gated, MATS = 2: 8 NB features of both projections), the whole work
// of a workgroup.  KS > 1 (shapes of one wave): its KS waves split the reduction of each tile.
template <class S, bool LINES, int MATS, int KS = 1>
__device__ __forceinline__ void mx4_rows(const Mx4Args &m, uint8_t *smem) {
  static_assert(MATS == 1 || S::NW % 4 == 0, "gated: a wave holds whole pairs of feature blocks");
  constexpr bool ROWS4 = S::ROWS4;
  constexpr int BF = 16 * S::NB / MATS;
  const GatedArgs &g = m.g;
  const RaggedTiles tiles(g.offsets, g.N, g.S, 16 * S::MB, g.fill);
  const int nN = (g.M + BF - 1) / BF, per = nN * g.splits;
  const Share share(static_cast<long long>(tiles.total) * per);
  const uint32_t code_row = static_cast<uint32_t>(g.K) / 2, scale_row = mx4_scale_row(g.K);
  auto ref = [&](const Item &it, int) {
    const int f0 = it.tile * BF;
    const int klen = it.group < 0 ? 0 : g.K, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // parts of whole 128 k: their scales are whole words
    const Part k = KS > 1 ? part_of<128>(klen, wave, KS) : part_of<128>(klen, it.split, g.splits);
    GatedRef<S> t;
    if constexpr (ROWS4) {
      t.a.codes[0] = static_cast<const uint8_t *>(g.x) + static_cast<size_t>(it.row0) * code_row;
      t.a.scales[0] = m.x_scales + static_cast<size_t>(it.row0) * scale_row;
      t.a.k0 = k.k0;
    } else {
      t.a.p[0] = static_cast<const bf16_t *>(g.x) + static_cast<size_t>(it.row0) * g.K + k.k0;
    }
    const size_t row = static_cast<size_t>(max(it.group, 0)) * g.M + f0;
    t.b.codes[0] = static_cast<const uint8_t *>(g.w_gate) + row * code_row;
    t.b.scales[0] = m.gate_scales + row * scale_row;
    t.b.k0 = k.k0;
    if constexpr (MATS == 2) {
      t.b.codes[1] = static_cast<const uint8_t *>(g.w_up) + row * code_row;
      t.b.scales[1] = m.up_scales + row * scale_row;
    }
    t.at = static_cast<size_t>(it.row0) * g.M + f0;
    t.out = static_cast<bf16_t *>(g.a) + t.at;
    t.part = g.splits > 1 ? g.part + MATS * static_cast<size_t>(it.split) * g.S * g.M + t.at : nullptr;
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
    using Store = std::conditional_t<MATS == 2, GatedStore<bf16_t, LINES, S>, StoreTile<bf16_t, LINES, S>>;
    const Store store = [&]() -> Store {
      if constexpr (MATS == 2)
        return {g};
      else
        return {static_cast<size_t>(g.M)};
    }();
    if constexpr (KS > 1) {
      const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
      grouped_items<S>(item, n, g.K, g.K, smem + wave * S::LDS, ref, JoinStore<S, KS, Store>{store, smem + KS * S::LDS, 0});
    } else {
      grouped_items<S>(item, n, g.K, g.K, smem, ref, store);
    }
  }
}

// Few rows: tiles of 16, the reduction over the workgroup's four waves
constexpr int kSplitWaves = 4;
template <bool ROWS4, bool LINES, int MATS> __global__ __launch_bounds__(64 * kSplitWaves) void mx4_few_kernel(Mx4Args m) {
  using S = Mx4Tile<ROWS4, 1, 4, 1, 1, 3, 3, MATS>;
  __shared__ __align__(16) uint8_t smem[kSplitWaves * S::LDS + JoinStore<S, kSplitWaves, int>::LDS];
  mx4_rows<S, LINES, MATS, kSplitWaves>(m, smem);
}

template <class Sh, bool LINES, int MATS> __global__ __launch_bounds__(Sh::THREADS) void mx4_rows_kernel(Mx4Args m) {
  using S = typename Sh::template Tile<MATS>;
  __shared__ __align__(16) uint8_t smem[S::LDS];
  mx4_rows<S, LINES, MATS>(m, smem);
}

// The same with one of two shapes taken here, from the groups' sizes that only the device knows
template <class Low, class High, bool LINES, int MATS>
__global__ __launch_bounds__(512) void mx4_shapes_kernel(Mx4Args m) {
  using SL = typename Low::template Tile<MATS>;
  using SH = typename High::template Tile<MATS>;
  static_assert(Low::THREADS == 512 && High::THREADS == 512, "one launch");
  __shared__ __align__(16) uint8_t smem[SL::LDS > SH::LDS ? SL::LDS : SH::LDS];
  const GatedArgs &g = m.g;
  const int heights[2] = {Low::TM, High::TM};
  int tiles[2];
  RaggedTiles::count(g.offsets, g.N, g.S, heights, tiles, g.fill);
  const int slots = static_cast<int>(gridDim.x);
  auto cost = [&](int h, int width, int stage) {
    const long long items = static_cast<long long>(tiles[h]) * ((MATS * g.M + width - 1) / width);
    return (items + slots - 1) / slots * stage;
  };
  if (cost(0, Low::TN, Low::COST) <= cost(1, High::TN, High::COST))
    mx4_rows<SL, LINES, MATS>(m, smem);
  else
    mx4_rows<SH, LINES, MATS>(m, smem);
}

// COST: time of a stage of a tile with every CU busy, in units of 50 ns
template <bool ROWS4, int MB, int NB, int WR, int WC, int DA, int DB, int COST_ = 0> struct Mx4Shape {
  template <int MATS> using Tile = Mx4Tile<ROWS4, MB, NB, WR, WC, DA, DB, MATS>;
  static constexpr int TM = 16 * MB, TN = 16 * NB, THREADS = WR * WC * 64, COST = COST_;
  static constexpr int PER_CU = 160 * 1024 / Tile<1>::LDS;
  static_assert(PER_CU >= 1, "fits a CU");
};
// What they reach, on 128 groups of 768 x 2048 unless said otherwise (kernel times).  The small ones are bound by the
// weights' way from memory: 256 rows through gate and up 44 us, 4.2 TB/s of the 187 MB that the call needs (two workgroups a
// CU with rings of three; one with four 53, with six 56).  The large ones by the matrix cores and what a stage costs beside them:
//   bf16 rows   32768: 192 x 256 117 us (0.88 PFLOP/s; others: 160 x 256 121, 128 x 256 141, 320 x 192 by 64 k 145, 256 x 256
//               by 64 k 187); 8192 in one group of 4096 x 4096 233 (1.18 PFLOP/s; 160 x 256 261)
//   4-bit rows  32768: 320 x 192 66 us (1.57 PFLOP/s), 256 x 256 90; 8192 in one group of 4096 x 4096 140 and 99 (2.8)
// Codes become bf16 two at a time by an instruction of 4 cycles, in every wave that needs the column: waves as 2 x 4 turn
// each of them twice, as 4 x 2 four times.
// bf16 rows
using Wide16 = Mx4Shape<false, 1, 16, 1, 4, 3, 3>;
using Wide64 = Mx4Shape<false, 4, 8, 2, 2, 3, 3>;
using Wide192 = Mx4Shape<false, 12, 16, 2, 4, 2, 2>;
// rows in 4 bits
using Four16 = Mx4Shape<true, 1, 16, 1, 4, 3, 3>;
using Four64 = Mx4Shape<true, 4, 8, 2, 2, 4, 4>;
using Four256 = Mx4Shape<true, 16, 16, 4, 2, 3, 3, 30>;
using Four320 = Mx4Shape<true, 20, 12, 4, 2, 3, 3, 38>;

enum class Kind { kFew, k16, k64, kLarge };
struct Plan {
  Kind kind;
  int splits;
};

// Which kernel.  Few tiles of 16 rows x 64 columns: those, the reduction over the waves of a workgroup, against parts of the
// reduction and a launch that adds them (kernel times: 8 rows in 128 groups of 768 x 2048 8.6 us against 12.8, 64 rows
// in 64 groups 16.8 against 20.5, in one of 2048 x 4096 11.4 against 15.0).  More of them: 16 x 256 tiles up to 16 rows a
// group, 64 x 128 up to 96, then the large shapes.  Kernel times of each without parts, groups of 768 x 2048, bf16 rows plain
// and gated, rows in 4 bits plain and gated:
//   rows, groups    few                     16 x 256                64 x 128               large
//       8, 128      8.8   9.3   8.2   8.5  18.0  18.0 16.2  16.1   19.8  19.9 16.4  16.2  26.8  30.7 22.9 23.0
//      64,  64     17.2  27.2  15.8  24.6  18.2  23.8 16.8  21.2   21.5  34.3 17.8  28.2  26.3  54.7 23.4 39.8
//     256, 128     29.2  56.0  26.9  51.3  25.1  44.0 23.5  42.9   34.8  60.6 29.0  48.9  48.3  83.1 41.4 60.3
//    2048, 128     41.2  86.4  36.3  76.6  35.0  59.9 31.7  55.7   36.2  63.3 29.6  51.0  54.0  94.5 42.1 62.9
//    8192, 128    114.1 248.2  99.2 213.9  67.7 136.7 52.9 113.3   60.0 108.8 44.8  81.7  66.5 106.2 46.8 68.8
//   12288, 128    160.0 355.7 138.4 304.8  99.2 194.8 74.6 154.9   70.6 136.5 50.7 100.3  74.3 120.0 49.5 72.6
//   16384, 128    206.5 454.8 180.7 393.6 122.1 248.2 91.5 196.9   92.3 166.1 66.2 117.8  80.7 129.9 52.9 76.8
// The rules are the plain products'; the gated block would gain by the large shapes from 64 rows a group on.
Plan plan_mx4(const Mx4Args &m) {
  const GatedArgs &g = m.g;
  const int mats = m.gated ? 2 : 1, cols = mats * g.M;
  if (g.S <= 64ll * g.N && about_tiles(g.S, g.N, 16) * tiles_of(cols, 64) <= 4 * kCUs) return {Kind::kFew, 1};
  if (g.S <= 16ll * g.N) return {Kind::k16, 1};
  const long long items = about_tiles(g.S, g.N, 64) * tiles_of(cols, Wide64::TN);
  if (items <= 2 * kCUs)
    return {Kind::k64, pick_splits(items, kCUs * Wide64::PER_CU, tiles_of(g.K, 128), static_cast<size_t>(g.S) * cols, 0.8)};
  return {g.S <= 96ll * g.N ? Kind::k64 : Kind::kLarge, 1};
}

bool lines(const GatedArgs &g) { return g.M % 64 == 0 && reinterpret_cast<uintptr_t>(g.a) % 128 == 0; }

template <class Sh, int MATS> void launch_shape(const Mx4Args &m, hipStream_t s) {
  const GatedArgs &g = m.g;
  const long long items = ragged_max_tiles(g.S, g.N, Sh::TM) * tiles_of(MATS * g.M, Sh::TN) * g.splits;
  auto launch = [&](auto kernel) { kernel<<<grouped_grid(items, Sh::PER_CU), Sh::THREADS, 0, s>>>(m); };
  lines(g) ? launch(mx4_rows_kernel<Sh, true, MATS>) : launch(mx4_rows_kernel<Sh, false, MATS>);
}
template <bool ROWS4, int MATS> void launch_few(const Mx4Args &m, hipStream_t s) {
  const unsigned grid = grouped_grid(ragged_max_tiles(m.g.S, m.g.N, 16) * tiles_of(MATS * m.g.M, 64), 1);
  auto launch = [&](auto kernel) { kernel<<<grid, 64 * kSplitWaves, 0, s>>>(m); };
  lines(m.g) ? launch(mx4_few_kernel<ROWS4, true, MATS>) : launch(mx4_few_kernel<ROWS4, false, MATS>);
}
template <class Sh> void launch_kind(const Mx4Args &m, hipStream_t s) {
  m.gated ? launch_shape<Sh, 2>(m, s) : launch_shape<Sh, 1>(m, s);
}
template <class Low, class High, int MATS> void launch_shapes(const Mx4Args &m, hipStream_t s) {
  auto launch = [&](auto kernel) { kernel<<<kCUs, 512, 0, s>>>(m); };
  lines(m.g) ? launch(mx4_shapes_kernel<Low, High, true, MATS>) : launch(mx4_shapes_kernel<Low, High, false, MATS>);
}

unsigned convert_grid(uint32_t total) { return std::min<uint32_t>((total + 15) / 16, 16 * kCUs); }

template <typename F> hipError_t launch_convert(const Mx4Convert &a, hipStream_t s, F kernel) {
  if (a.total == 0) return hipSuccess;
  kernel<<<convert_grid(a.total), 256, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace

size_t mx4_part_bytes(const Mx4Args &m) {
  const int n = m.g.S > 0 ? plan_mx4(m).splits : 1;
  return n > 1 ? (m.gated ? 2 : 1) * n * static_cast<size_t>(m.g.S) * m.g.M * sizeof(float) : 0;
}

hipError_t launch_mx4(Mx4Args m, hipStream_t s) {
  GatedArgs &g = m.g;
  if (g.S <= 0) return hipSuccess;
  const Plan p = plan_mx4(m);
  g.splits = p.splits;
  const bool four = m.x_scales != nullptr;
  switch (p.kind) {
    case Kind::kFew:
      if (four)
        m.gated ? launch_few<true, 2>(m, s) : launch_few<true, 1>(m, s);
      else
        m.gated ? launch_few<false, 2>(m, s) : launch_few<false, 1>(m, s);
      break;
    case Kind::k16: four ? launch_kind<Four16>(m, s) : launch_kind<Wide16>(m, s); break;
    case Kind::k64: four ? launch_kind<Four64>(m, s) : launch_kind<Wide64>(m, s); break;
    case Kind::kLarge:
      if (four)
        m.gated ? launch_shape<Four256, 2>(m, s) : launch_shapes<Four256, Four320, 1>(m, s);
      else
        launch_kind<Wide192>(m, s);
      break;
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.splits == 1) return e;
  if (m.gated) return launch_gated_join(g, true, s);
  GroupedArgs j{};
  j.out = g.a;
  j.offsets = g.offsets;
  j.S = g.S;
  j.N = g.N;
  j.fill = g.fill;
  j.splits = p.splits;
  j.part = g.part;
  return launch_grouped_join(j, g.M, true, s);
}

hipError_t launch_mx4_quantize(const Mx4Convert &a, bool bf16, hipStream_t s) {
  if (a.K % 128 == 0)
    return launch_convert(a, s, bf16 ? mx4_quantize_kernel<bf16_t, true> : mx4_quantize_kernel<float, true>);
  return launch_convert(a, s, bf16 ? mx4_quantize_kernel<bf16_t, false> : mx4_quantize_kernel<float, false>);
}

hipError_t launch_mx4_dequantize(const Mx4Convert &a, bool bf16, hipStream_t s) {
  if (a.K % 128 == 0)
    return launch_convert(a, s, bf16 ? mx4_dequantize_kernel<bf16_t, true> : mx4_dequantize_kernel<float, true>);
  return launch_convert(a, s, bf16 ? mx4_dequantize_kernel<bf16_t, false> : mx4_dequantize_kernel<float, false>);
}

}  // namespace ace
