// Low-rank adapters of many requests at once beside a shared projection: row r of a request
// that carries adapter a gets
//   out[r] = base[r] + scale_a B_a v,   v = A_a x[r]
// and every other row gets base[r].  A_a [rank, din], B_a [dout, rank].
//
// v has to be whole before any of it is used.  Many rows: two launches, the first multiplies tiles of 64
// rows of one request by A_a, din split over the waves of a workgroup and over workgroups (partial
// sums [splits][S][rank], fp32), the second adds the splits in order and multiplies by B_a.  Few rows, where a
// launch costs as much as the work (decoding): one launch, each workgroup computes v of 16 rows
// for itself and multiplies it by its share of B_a's rows.
// Operands go from memory straight into the matrix cores' registers: a wave reads each fragment
// of A_a and B_a once and uses it for every row of its tile, so staging them would save nothing.
// v stays exact to 2^-16 in bf16 calls: it is multiplied as the sum of two bf16 numbers (a
// single rounding of v to 8 bits would cost as much as that of the output).
#include <algorithm>
#include <type_traits>

#include "lds_dma.h"
#include "ragged.h"

namespace ace {

namespace {

constexpr int kRowBlock = 16;
constexpr int kTileRows = 64;    // of the two launches
constexpr int kExpandWaves = 4;  // 64 columns each
constexpr int kMaxParts = 16;    // partial sums of v
constexpr int kCUs = 256;

template <typename T> using frag_of = typename Frag<T>::type;
template <typename T> __device__ __forceinline__ frag_of<T> zero_frag() {
  return __builtin_bit_cast(frag_of<T>, uint4{0, 0, 0, 0});
}
template <typename T> constexpr int kStepK = 64 / static_cast<int>(sizeof(T));  // k of a pair of fragments
// pairs of fragments that hold a rank of 16 RB
template <typename T, int RB> constexpr int kRankSteps = (16 * RB + kStepK<T> - 1) / kStepK<T>;

// adapter of a tile, or -1
__device__ __forceinline__ int tile_adapter(const AdapterArgs &p, const RaggedTile &t) {
  if (t.group < 0) return -1;
  const int a = p.adapter[t.group];
  return a >= 0 && a < p.L ? a : -1;
}

// acc[i][c] += rows 16 i .. of x times rows 16 c .. of A over k = first, first + step, .. (a fragment
// pair each): lane holds rank 16 c + 4 g + q of row 16 i + lane % 16.  Rows past the tile repeat its last.
// The whole steps begin at the rot-th, so that tiles side by side are not all at the same 64 bytes of A's rows, which
// lie in few cache channels (8192 rows, rank 128, 2048 columns: 90 us from the first, 81 so; where a wave has two
// steps only, 2048 fp32 rows of the same took 55 from the first, 66 so).
template <typename T, int RT, int RB>
__device__ __forceinline__ void shrink(const AdapterArgs &p, const RaggedTile &t, int ad, int first, int step, int rot,
                                       f32x4_t (&acc)[RT][RB]) {
  constexpr int E = kChunkElems<T>;
  const int lane = threadIdx.x & 63, r16 = lane & 15, g = lane >> 4;
  const T *xb = static_cast<const T *>(p.x) + static_cast<size_t>(t.row0) * p.din;
  const T *wb = static_cast<const T *>(p.a) + static_cast<size_t>(ad) * p.r * p.din;
  uint32_t x[RT], w[RB];  // this lane's rows from there on: at most 128 of 65536
#pragma unroll
  for (int i = 0; i < RT; ++i) x[i] = static_cast<uint32_t>(min(16 * i + r16, t.rows - 1) * p.din + E * g);
#pragma unroll
  for (int c = 0; c < RB; ++c) w[c] = static_cast<uint32_t>(min(16 * c + r16, p.r - 1) * p.din + E * g);
#pragma unroll
  for (int i = 0; i < RT; ++i)
#pragma unroll
    for (int c = 0; c < RB; ++c) acc[i][c] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  frag_of<T> xf[RT], wf[RB];
  auto multiply = [&]() {
#pragma unroll
    for (int s = 0; s < Frag<T>::steps; ++s)
#pragma unroll
      for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int c = 0; c < RB; ++c) acc[i][c] = Frag<T>::mma(wf[c], xf[i], s, acc[i][c]);
  };
  const int whole = max(p.din - first - kStepK<T> + step, 0) / step;  // steps that end within din
  int at = whole >= 4 ? rot % whole : 0;
#pragma unroll 2
  for (int s = 0; s < whole; ++s) {
    const int k0 = first + at * step;
    at = at + 1 == whole ? 0 : at + 1;
#pragma unroll
    for (int i = 0; i < RT; ++i) xf[i] = *reinterpret_cast<const frag_of<T> *>(xb + k0 + x[i]);
#pragma unroll
    for (int c = 0; c < RB; ++c) wf[c] = *reinterpret_cast<const frag_of<T> *>(wb + k0 + w[c]);
    multiply();
  }
  const int k0 = first + whole * step;
  if (k0 < p.din) {  // din ends inside the step: zeros behind the end, in both operands
    const bool in = k0 + E * g < p.din;
#pragma unroll
    for (int i = 0; i < RT; ++i) xf[i] = in ? *reinterpret_cast<const frag_of<T> *>(xb + k0 + x[i]) : zero_frag<T>();
#pragma unroll
    for (int c = 0; c < RB; ++c) wf[c] = in ? *reinterpret_cast<const frag_of<T> *>(wb + k0 + w[c]) : zero_frag<T>();
    multiply();
  }
}

// A lane's E values of v as fragments: bf16 the value cut off and the rest of it (of the same sign, so the two
// parts' products never cancel; a value between bf16's largest and fp32's stays finite), fp32 itself
template <typename T> struct VFrag {
  frag_of<T> hi, lo;
  __device__ __forceinline__ void set(const float *f) {
    if constexpr (sizeof(T) == 2) {
      uint32_t h[4], l[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t a = __float_as_uint(f[2 * i]) & 0xffff0000u, b = __float_as_uint(f[2 * i + 1]) & 0xffff0000u;
        h[i] = a >> 16 | b;
        l[i] = pack_bf16x2(f[2 * i] - __uint_as_float(a), f[2 * i + 1] - __uint_as_float(b));
      }
      hi = __builtin_bit_cast(frag_of<T>, uint4{h[0], h[1], h[2], h[3]});
      lo = __builtin_bit_cast(frag_of<T>, uint4{l[0], l[1], l[2], l[3]});
    } else {
      hi = __builtin_bit_cast(
          frag_of<T>, uint4{__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])});
    }
  }
};

// Rows of v in LDS, 16-byte quads, zeros behind the rank: odd strides, so that 16 rows' reads go to different banks
template <typename T, int KB> constexpr int kVQuads = KB * kStepK<T> / 4;
template <typename T, int KB> constexpr int kVStride = kVQuads<T, KB> + 1;
template <typename T, int KB>
__device__ __forceinline__ void read_v(const f32x4_t *vs, int row, VFrag<T> (&vf)[KB]) {
  constexpr int E = kChunkElems<T>;
  const int g = (threadIdx.x & 63) >> 4;
#pragma unroll
  for (int kb = 0; kb < KB; ++kb) {
    const int k = kb * kStepK<T> + E * g;
    float f[E];
#pragma unroll
    for (int j = 0; j < E; j += 4) {
      const f32x4_t u = vs[row * kVStride<T, KB> + k / 4 + j / 4];
#pragma unroll
      for (int l = 0; l < 4; ++l) f[j + l] = u[l];
    }
    vf[kb].set(f);
  }
}

// 64 columns of B_a from c0, as fragments.  bf16: the columns of two 16-column blocks interleaved in fours,
// so that a lane's results are 8 consecutive columns (see grouped.hip)
template <typename T, int KB> struct Columns {
  static constexpr bool PAIR = sizeof(T) == 2;
  static constexpr int E = kChunkElems<T>;
  frag_of<T> w[KB][4];
  int c0;
  __device__ __forceinline__ void load(const AdapterArgs &p, int ad, int c0_) {
    c0 = c0_;
    const int lane = threadIdx.x & 63, r16 = lane & 15, g = lane >> 4;
    const T *b = static_cast<const T *>(p.b) + static_cast<size_t>(ad) * p.dout * p.r;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const int col = min(c0 + (PAIR ? 32 * (c >> 1) + 8 * (r16 >> 2) + 4 * (c & 1) + (r16 & 3) : 16 * c + r16), p.dout - 1);
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) {
        const int k = kb * kStepK<T> + E * g;
        // loaded in any case and replaced behind the end of the rank, so that no load is a branch of its own
        const frag_of<T> f = *reinterpret_cast<const frag_of<T> *>(b + static_cast<size_t>(col) * p.r + min(k, p.r - E));
        w[kb][c] = k < p.r ? f : zero_frag<T>();
      }
    }
  }
  static constexpr int STEP = PAIR ? 2 : 1;
  static constexpr int PIECES = 4 / STEP;  // of 16 bytes of a row in a lane
  __device__ __forceinline__ int col(int i) const { return c0 + 16 * STEP * i + E * static_cast<int>((threadIdx.x & 63) >> 4); }

  // a row of base, in pieces of 16 bytes
  __device__ __forceinline__ void base_of(const AdapterArgs &p, size_t row, bool there, uint4 (&v)[PIECES]) const {
#pragma unroll
    for (int i = 0; i < PIECES; ++i)
      v[i] = there && col(i) < p.dout ? *reinterpret_cast<const uint4 *>(static_cast<const T *>(p.base) + row * p.dout + col(i))
                                      : uint4{0, 0, 0, 0};
  }
  // out = base + scale B v for the row of this lane.  The scale comes last, as the definition has it: on v, an infinite
  // one would make no number of the zeros that pad an adapter of lower rank.
  __device__ __forceinline__ void finish(const AdapterArgs &p, const VFrag<T> (&v)[KB], float scale, size_t row, bool there,
                                         uint4 (&bv)[PIECES]) const {
    f32x4_t acc[4];
    auto multiply = [&](f32x4_t (&d)[4], bool rest) {
#pragma unroll
      for (int c = 0; c < 4; ++c) d[c] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int s = 0; s < Frag<T>::steps; ++s) {
#pragma unroll
          for (int c = 0; c < 4; ++c) d[c] = Frag<T>::mma(w[kb][c], v[kb].hi, s, d[c]);
          if constexpr (PAIR)
            if (rest)
#pragma unroll
              for (int c = 0; c < 4; ++c) d[c] = Frag<T>::mma(w[kb][c], v[kb].lo, s, d[c]);
        }
    };
    multiply(acc, true);
    if constexpr (PAIR) {
      // An infinite b or v makes no number of its product with v's rest (infinity times zero).  Where a sum is not
      // finite, the products of v's first part alone say what it is.
      const f32x4_t t = (acc[0] + acc[1]) + (acc[2] + acc[3]);
      if (__any(!__builtin_isfinite((t[0] + t[1]) + (t[2] + t[3])))) {
        f32x4_t first[4];
        multiply(first, false);
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
          for (int j = 0; j < 4; ++j) acc[c][j] = __builtin_isfinite(first[c][j]) ? acc[c][j] : first[c][j];
      }
    }
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      if constexpr (PAIR) {
        uint32_t b[4] = {bv[i].x, bv[i].y, bv[i].z, bv[i].w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const f32x4_t &d = acc[2 * i + (j >> 1)];
          b[j] = pack_bf16x2(__uint_as_float(b[j] << 16) + scale * d[2 * (j & 1)],
                             __uint_as_float(b[j] & 0xffff0000u) + scale * d[2 * (j & 1) + 1]);
        }
        bv[i] = uint4{b[0], b[1], b[2], b[3]};
      } else {
        bv[i] = __builtin_bit_cast(uint4, __builtin_bit_cast(f32x4_t, bv[i]) + scale * acc[i]);
      }
    }
    put(p, row, there, bv);
  }
  __device__ __forceinline__ void put(const AdapterArgs &p, size_t row, bool there, const uint4 (&v)[PIECES]) const {
#pragma unroll
    for (int i = 0; i < PIECES; ++i)
      if (there && col(i) < p.dout) *reinterpret_cast<uint4 *>(static_cast<T *>(p.out) + row * p.dout + col(i)) = v[i];
  }
};

// Share `chunk` of p.chunks of the 64-column groups of the output
struct Groups {
  int first, last;
  __device__ __forceinline__ Groups(const AdapterArgs &p, int chunk) {
    const int groups = (p.dout + 63) >> 6, each = (groups + p.chunks - 1) / p.chunks;
    first = chunk * each;
    last = min(first + each, groups);
  }
};

// ---------------------------------------------------------------- many rows
template <typename T, int RB> __global__ __launch_bounds__(256) void adapter_shrink_kernel(AdapterArgs p) {
  constexpr int RT = kTileRows / kRowBlock;
  const int b = ragged_block();
  const RaggedTile t = RaggedTiles(p.offsets, p.R, p.S, kTileRows, false).find_uniform(b / p.splits);
  if (!t.valid) return;
  const int ad = tile_adapter(p, t);
  if (ad < 0) return;
  const int split = b % p.splits;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r16 = lane & 15, g = lane >> 4;
  __shared__ f32x4_t red[4][RB][64];
  // with as many row blocks as the tile has (1, 2 or all)
  auto run = [&](auto rt) {
    f32x4_t acc[rt()][RB];
    shrink<T, rt(), RB>(p, t, ad, (split * 4 + wave) * kStepK<T>, 4 * p.splits * kStepK<T>, t.row0 / kTileRows, acc);
    // the waves' sums: row block i's are added by wave i in wave order
#pragma unroll
    for (int i = 0; i < rt(); ++i) {
      if (i > 0) __syncthreads();
#pragma unroll
      for (int c = 0; c < RB; ++c) red[wave][c][lane] = acc[i][c];
      __syncthreads();
      const int row = 16 * i + r16;
      if (wave != i || row >= t.rows) continue;
      float *v = p.v + (static_cast<size_t>(split) * p.S + t.row0 + row) * p.r;
#pragma unroll
      for (int c = 0; c < RB; ++c) {
        const int col = 16 * c + 4 * g;
        if (col < p.r)
          *reinterpret_cast<f32x4_t *>(v + col) = red[0][c][lane] + red[1][c][lane] + red[2][c][lane] + red[3][c][lane];
      }
    }
  };
  if (t.rows <= 16)
    run(std::integral_constant<int, 1>{});
  else if (t.rows <= 32)
    run(std::integral_constant<int, 2>{});
  else
    run(std::integral_constant<int, RT>{});
}

// Tile = 64 rows x one of p.chunks shares of the columns, 64 of them a wave at a time: B_a's fragments
// are read once for the four row blocks.  Bound by the chain offsets -> adapter -> B_a -> products -> stores with
// two waves a SIMD to hide it; so base and v are asked for before the adapter's number, and no load hangs on a
// condition of its own (4096 rows, rank 64, 2048 columns: 15.6 us with such conditions, 13.8 without).
template <typename T, int KB> __global__ __launch_bounds__(64 * kExpandWaves) void adapter_expand_kernel(AdapterArgs p) {
  const int b = ragged_block();
  const RaggedTile t = RaggedTiles(p.offsets, p.R, p.S, kTileRows, p.out != p.base).find_uniform(b / p.chunks);
  if (!t.valid) return;
  const int r16 = threadIdx.x & 15, wave = threadIdx.x >> 6;
  const Groups cols(p, b % p.chunks);
  using Cols = Columns<T, KB>;
  Cols w;
  uint4 bv[Cols::PIECES], next[Cols::PIECES];
  const int blocks = (t.rows + 15) >> 4;
  auto row_of = [&](int i) { return static_cast<size_t>(t.row0) + 16 * i + r16; };
  auto there = [&](int i) { return 16 * i + r16 < t.rows; };
  // base's first rows and the first part of v are under way while the adapter's number is read
  w.c0 = 64 * (cols.first + wave);
  w.base_of(p, row_of(0), there(0), bv);
  constexpr int VQ = kVQuads<T, KB>, VT = kTileRows * VQ / (64 * kExpandWaves);  // quads of a thread
  static_assert(VT * 64 * kExpandWaves == kTileRows * VQ, "v of a tile in whole rounds");
  const float *v[VT];
  f32x4_t vsum[VT];
#pragma unroll
  for (int j = 0; j < VT; ++j) {
    const int i = static_cast<int>(threadIdx.x) + j * 64 * kExpandWaves;
    v[j] = p.v + (static_cast<size_t>(t.row0) + min(i / VQ, t.rows - 1)) * p.r + min(4 * (i % VQ), p.r - 4);
    vsum[j] = *reinterpret_cast<const f32x4_t *>(v[j]);
  }
  const int ad = tile_adapter(p, t);
  if (ad < 0) {
    if (p.out == p.base) return;
    for (int q = cols.first + wave; q < cols.last; q += kExpandWaves) {
      w.c0 = 64 * q;
      for (int i = 0; i < blocks; ++i) {
        w.base_of(p, row_of(i), there(i), bv);
        w.put(p, row_of(i), there(i), bv);
      }
    }
    return;
  }
  if (cols.first + wave < cols.last) w.load(p, ad, 64 * (cols.first + wave));
  // v of the tile's rows: the parts added in order, once for all waves
  __shared__ f32x4_t vs[kTileRows * kVStride<T, KB>];
  const float sc = p.scale ? p.scale[ad] : 1.f;
  for (int s = 1; s < p.splits; ++s)
#pragma unroll
    for (int j = 0; j < VT; ++j) vsum[j] += *reinterpret_cast<const f32x4_t *>(v[j] + static_cast<size_t>(s) * p.S * p.r);
#pragma unroll
  for (int j = 0; j < VT; ++j) {
    const int i = static_cast<int>(threadIdx.x) + j * 64 * kExpandWaves, q = i % VQ;
    vs[i / VQ * kVStride<T, KB> + q] = 4 * q < p.r ? vsum[j] : f32x4_t{0.f, 0.f, 0.f, 0.f};
  }
  __syncthreads();
  for (int q = cols.first + wave; q < cols.last; q += kExpandWaves) {
    if (q != cols.first + wave) {
      w.load(p, ad, 64 * q);
      w.base_of(p, row_of(0), there(0), bv);
    }
    for (int i = 0; i < blocks; ++i) {
      VFrag<T> vf[KB];
      read_v<T, KB>(vs, 16 * i + r16, vf);
      // the next block's rows of base are under way while this one's are finished
      if (i + 1 < blocks) w.base_of(p, row_of(i + 1), there(i + 1), next);
      w.finish(p, vf, sc, row_of(i), there(i), bv);
#pragma unroll
      for (int j = 0; j < Cols::PIECES; ++j) bv[j] = next[j];
    }
  }
}

// ---------------------------------------------------------------- few rows
constexpr int kSmallWaves = 8;

// Tile = 16 rows x one of p.chunks shares of the columns; din split over the waves
template <typename T, int RB> __global__ __launch_bounds__(64 * kSmallWaves) void adapter_small_kernel(AdapterArgs p) {
  constexpr int KB = kRankSteps<T, RB>;
  const int b = ragged_block();
  const RaggedTile t = RaggedTiles(p.offsets, p.R, p.S, kRowBlock, p.out != p.base).find_uniform(b / p.chunks);
  if (!t.valid) return;
  const int ad = tile_adapter(p, t);
  if (ad < 0 && p.out == p.base) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r16 = lane & 15, g = lane >> 4;
  const Groups cols(p, b % p.chunks);
  const int g0 = cols.first, g1 = cols.last;
  const size_t row = static_cast<size_t>(t.row0) + r16;
  const bool there = r16 < t.rows;
  using Cols = Columns<T, KB>;
  Cols w;
  uint4 bv[Cols::PIECES];
  if (ad < 0) {
    for (int q = g0 + wave; q < g1; q += kSmallWaves) {
      w.c0 = 64 * q;
      w.base_of(p, row, there, bv);
      w.put(p, row, there, bv);
    }
    return;
  }
  // the first column group's operands are under way while v is computed
  if (g0 + wave < g1) {
    w.load(p, ad, 64 * (g0 + wave));
    w.base_of(p, row, there, bv);
  }
  __shared__ f32x4_t red[kSmallWaves][RB][64];
  __shared__ f32x4_t vs[kRowBlock * kVStride<T, KB>];
  f32x4_t acc[1][RB];
  shrink<T, 1, RB>(p, t, ad, wave * kStepK<T>, kSmallWaves * kStepK<T>, t.row0 / kRowBlock, acc);
#pragma unroll
  for (int c = 0; c < RB; ++c) red[wave][c][lane] = acc[0][c];
  __syncthreads();
  const float sc = p.scale ? p.scale[ad] : 1.f;
  for (int c = wave; c < RB; c += kSmallWaves) {
    f32x4_t s = red[0][c][lane];
#pragma unroll
    for (int i = 1; i < kSmallWaves; ++i) s += red[i][c][lane];
    const int q = 4 * c + g;
    vs[r16 * kVStride<T, KB> + q] = 4 * q < p.r ? s : f32x4_t{0.f, 0.f, 0.f, 0.f};
  }
  for (int i = threadIdx.x; i < kRowBlock * (kVQuads<T, KB> - 4 * RB); i += 64 * kSmallWaves)
    vs[i % kRowBlock * kVStride<T, KB> + 4 * RB + i / kRowBlock] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  __syncthreads();
  VFrag<T> vf[KB];
  read_v<T, KB>(vs, r16, vf);
  for (int q = g0 + wave; q < g1; q += kSmallWaves) {
    if (q != g0 + wave) {
      w.load(p, ad, 64 * q);
      w.base_of(p, row, there, bv);
    }
    w.finish(p, vf, sc, row, there, bv);
  }
}

// Column shares of one launch: as many as give every CU a workgroup, a 64-column group a wave at least (1024 rows of 7
// requests, rank 64, 2048 columns: 18.7 us, with twice as many shares 28.7, in two launches 20.6).
constexpr int kSmallTiles = 256;
int small_shares(long long tiles, int dout) {
  const int groups = (dout + 63) / 64, most = (groups + kSmallWaves - 1) / kSmallWaves;
  return static_cast<int>(std::max(1ll, std::min<long long>(most, kCUs / tiles)));
}

// One launch for up to kSmallTiles 16-row tiles, unless computing v in each share takes longer than another launch: past
// 512 KB of A_a in bf16, 256 KB in fp32, whose products take 16 times as long; or a share's part of B_a does: past
// 512 KB (2048 rows of 7 requests, 768 x 4096: rank 128 46 us and in two launches 40, rank 64 29 and 27, 3000 rows 30 and
// 33).  Requests of few rows would leave most of a 64-row tile empty: one launch
// for any number of them, with half of that A_a (2048 columns, rank 16: 1000 rows of 300 requests 16.5 us, in two
// launches 27, 8000 rows of 700 48 and 67; rank 64 37.6 and 44, 84 and 99; fp32 rank 64 with 768 columns 99 and 87).
bool is_small(int S, int R, int r, int din, int dout, bool bf16) {
  const long long tiles = ragged_max_tiles(S, R, kRowBlock), row = (r + 15) / 16 * 16 * (bf16 ? 2 : 4);
  const long long most = (bf16 ? 512 : 256) << 10;
  if (row * dout / small_shares(tiles, dout) > 512 << 10) return false;
  return (tiles <= kSmallTiles && row * din <= most) || (S <= 16ll * R && row * din <= most / 2);
}

template <typename T, int RB> hipError_t launch_rank(AdapterArgs p, hipStream_t s) {
  if (is_small(p.S, p.R, p.r, p.din, p.dout, sizeof(T) == 2)) {
    const long long tiles = ragged_max_tiles(p.S, p.R, kRowBlock);
    p.chunks = small_shares(tiles, p.dout);
    adapter_small_kernel<T, RB><<<ragged_grid(tiles * p.chunks), 64 * kSmallWaves, 0, s>>>(p);
    return hipGetLastError();
  }
  const long long tiles = ragged_max_tiles(p.S, p.R, kTileRows);
  // column shares: eight workgroups a CU, where there are more tiles fewer, longer ones (582 tiles, 3280 columns: 57 us
  // with a workgroup for every 256 columns, 38 so)
  const long long most = (p.dout + 64 * kExpandWaves - 1) / (64 * kExpandWaves);
  p.chunks = static_cast<int>(std::min(most, (8 * kCUs + tiles - 1) / tiles));
  const long long shrink = tiles * p.splits, expand = tiles * p.chunks;
  if (std::max(shrink, expand) > kRaggedMaxBlocks) return hipErrorInvalidValue;
  adapter_shrink_kernel<T, RB><<<ragged_grid(shrink), 256, 0, s>>>(p);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  adapter_expand_kernel<T, kRankSteps<T, RB>><<<ragged_grid(expand), 64 * kExpandWaves, 0, s>>>(p);
  return hipGetLastError();
}

template <typename T> hipError_t launch_t(const AdapterArgs &p, hipStream_t s) {
  if (p.r <= 16) return launch_rank<T, 1>(p, s);
  if (p.r <= 32) return launch_rank<T, 2>(p, s);
  if (p.r <= 48) return launch_rank<T, 3>(p, s);
  if (p.r <= 64) return launch_rank<T, 4>(p, s);
  if (p.r <= 96) return launch_rank<T, 6>(p, s);
  return launch_rank<T, 8>(p, s);
}

}  // namespace

int adapter_splits(int S, int R, int r, int din, int dout, bool bf16) {
  if (is_small(S, R, r, din, dout, bf16)) return 0;
  const long long tiles = ragged_max_tiles(S, R, kTileRows);
  const int step = bf16 ? kStepK<bf16_t> : kStepK<float>;
  int n = 1;
  // four workgroups a CU, at least four steps for each of a workgroup's four waves
  while (n < kMaxParts && tiles * n * 2 <= 4 * kCUs && din >= 4 * 4 * 2 * n * step) n *= 2;
  return n;
}

hipError_t launch_adapter(const AdapterArgs &p, bool bf16, hipStream_t stream) {
  if (p.S <= 0) return hipSuccess;
  return bf16 ? launch_t<bf16_t>(p, stream) : launch_t<float>(p, stream);
}

}  // namespace ace
