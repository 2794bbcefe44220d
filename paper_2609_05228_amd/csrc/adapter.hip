// Low-rank adapters of many requests at once beside a shared projection: row r of a request
// that carries adapter a gets
//   out[r] = base[r] + scale_a B_a v,   v = A_a x[r]
// and every other row gets base[r].  A_a [rank, din], B_a [dout, rank].
// Two launches: v has to be whole before any of it is used.  The first multiplies 16 rows of
// one request by A_a, din split over the waves of a workgroup and, where there are few rows,
// over workgroups (partial sums [splits][S][rank], fp32); the second adds the splits in order and
// multiplies by B_a.  Operands go from memory straight into the matrix cores' registers: each is
// used by one wave.  v stays exact to 16 bits in bf16 calls: it is multiplied as the sum of two
// bf16 numbers (a single rounding of v to 8 bits would cost as much as that of the output).
#include <algorithm>

#include "lds_dma.h"
#include "ragged.h"

namespace ace {

namespace {

constexpr int kAdRows = 16;

template <typename T> __device__ __forceinline__ typename Frag<T>::type zero_frag() {
  return __builtin_bit_cast(typename Frag<T>::type, uint4{0, 0, 0, 0});
}

// adapter of a tile, or -1
__device__ __forceinline__ int tile_adapter(const AdapterArgs &p, const RaggedTile &t) {
  if (t.group < 0) return -1;
  const int a = p.adapter[t.group];
  return a >= 0 && a < p.L ? a : -1;
}

// RB: 16-wide blocks of the rank
template <typename T, int RB> __global__ __launch_bounds__(256) void adapter_shrink_kernel(AdapterArgs p) {
  constexpr int KS = 64 / sizeof(T);  // k of one fragment pair
  constexpr int E = kChunkElems<T>;
  typedef typename Frag<T>::type frag_t;
  const int b = ragged_block();
  const RaggedTile t = RaggedTiles(p.offsets, p.R, p.S, kAdRows, false).find_uniform(b / p.splits);
  if (!t.valid) return;
  const int ad = tile_adapter(p, t);
  if (ad < 0) return;
  const int split = b % p.splits;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r16 = lane & 15, g = lane >> 4;
  const T *x = static_cast<const T *>(p.x) + static_cast<size_t>(t.row0 + min(r16, t.rows - 1)) * p.din;
  const T *w = static_cast<const T *>(p.a) + static_cast<size_t>(ad) * p.r * p.din;
  f32x4_t acc[RB];
#pragma unroll
  for (int c = 0; c < RB; ++c) acc[c] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  const int step = 4 * p.splits * KS;
#pragma unroll 4
  for (int k = (split * 4 + wave) * KS + E * g; k - E * g < p.din; k += step) {
    const bool in = k < p.din;
    const frag_t xf = in ? *reinterpret_cast<const frag_t *>(x + k) : zero_frag<T>();
#pragma unroll
    for (int c = 0; c < RB; ++c) {
      const int row = min(16 * c + r16, p.r - 1);
      const frag_t wf = in ? *reinterpret_cast<const frag_t *>(w + static_cast<size_t>(row) * p.din + k) : zero_frag<T>();
#pragma unroll
      for (int s = 0; s < Frag<T>::steps; ++s) acc[c] = Frag<T>::mma(wf, xf, s, acc[c]);
    }
  }
  __shared__ f32x4_t red[4][RB][64];
#pragma unroll
  for (int c = 0; c < RB; ++c) red[wave][c][lane] = acc[c];
  __syncthreads();
  if (r16 >= t.rows) return;
  float *v = p.v + (static_cast<size_t>(split) * p.S + t.row0 + r16) * p.r;
  for (int c = wave; c < RB; c += 4) {
    const int col = 16 * c + 4 * g;
    if (col < p.r) *reinterpret_cast<f32x4_t *>(v + col) = red[0][c][lane] + red[1][c][lane] + red[2][c][lane] + red[3][c][lane];
  }
}

constexpr int kAdCols = 256;  // output columns of a workgroup: 64 per wave

template <typename T, int KB> __global__ __launch_bounds__(256) void adapter_expand_kernel(AdapterArgs p) {
  constexpr int KS = 64 / sizeof(T);
  constexpr int E = kChunkElems<T>;
  constexpr bool PAIR = sizeof(T) == 2;
  typedef typename Frag<T>::type frag_t;
  const int nN = (p.dout + kAdCols - 1) / kAdCols;
  const int b = ragged_block();
  const RaggedTile t = RaggedTiles(p.offsets, p.R, p.S, kAdRows, true).find_uniform(b / nN);
  if (!t.valid) return;
  const int ad = tile_adapter(p, t);
  if (ad < 0 && p.out == p.base) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r16 = lane & 15, g = lane >> 4;
  const int c0 = (b % nN) * kAdCols + wave * 64;
  f32x4_t acc[4];
#pragma unroll
  for (int c = 0; c < 4; ++c) acc[c] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  if (ad >= 0) {
    const float sc = p.scale ? p.scale[ad] : 1.f;
    const float *v = p.v + static_cast<size_t>(t.row0 + min(r16, t.rows - 1)) * p.r;
    const T *w = static_cast<const T *>(p.b) + static_cast<size_t>(ad) * p.dout * p.r;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      const int k = kb * KS + E * g;
      const bool in = k < p.r;
      float f[E];
#pragma unroll
      for (int i = 0; i < E; ++i) f[i] = 0.f;
      if (in)
        for (int s = 0; s < p.splits; ++s) {
          const float *q = v + static_cast<size_t>(s) * p.S * p.r + k;
#pragma unroll
          for (int i = 0; i < E; i += 4) {
            const f32x4_t u = *reinterpret_cast<const f32x4_t *>(q + i);
#pragma unroll
            for (int j = 0; j < 4; ++j) f[i + j] += u[j];
          }
        }
      frag_t hi, lo;
#pragma unroll
      for (int i = 0; i < E; ++i) f[i] *= sc;
      if constexpr (PAIR) {
        uint32_t h4[4], l4[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          h4[i] = pack_bf16x2(f[2 * i], f[2 * i + 1]);
          l4[i] = pack_bf16x2(f[2 * i] - __uint_as_float(h4[i] << 16), f[2 * i + 1] - __uint_as_float(h4[i] & 0xffff0000u));
        }
        hi = __builtin_bit_cast(frag_t, uint4{h4[0], h4[1], h4[2], h4[3]});
        lo = __builtin_bit_cast(frag_t, uint4{l4[0], l4[1], l4[2], l4[3]});
      } else {
        hi = __builtin_bit_cast(frag_t, uint4{__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])});
      }
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const int col = min(PAIR ? c0 + 32 * (c >> 1) + 8 * (r16 >> 2) + 4 * (c & 1) + (r16 & 3) : c0 + 16 * c + r16, p.dout - 1);
        const frag_t wf = in ? *reinterpret_cast<const frag_t *>(w + static_cast<size_t>(col) * p.r + k) : zero_frag<T>();
#pragma unroll
        for (int s = 0; s < Frag<T>::steps; ++s) acc[c] = Frag<T>::mma(wf, hi, s, acc[c]);
        if constexpr (PAIR) acc[c] = Frag<T>::mma(wf, lo, 0, acc[c]);
      }
    }
  }
  if (r16 >= t.rows) return;
  const size_t ro = static_cast<size_t>(t.row0 + r16) * p.dout;
  const T *base = static_cast<const T *>(p.base) + ro;
  T *out = static_cast<T *>(p.out) + ro;
#pragma unroll
  for (int c = 0; c < 4; c += PAIR ? 2 : 1) {
    const int col = c0 + 16 * c + E * g;
    if (col >= p.dout) continue;
    uint4 bv = *reinterpret_cast<const uint4 *>(base + col);
    if (ad >= 0) {
      if constexpr (PAIR) {
        uint32_t *bw = reinterpret_cast<uint32_t *>(&bv);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const f32x4_t &d = acc[c + (i >> 1)];
          bw[i] = pack_bf16x2(__uint_as_float(bw[i] << 16) + d[2 * (i & 1)], __uint_as_float(bw[i] & 0xffff0000u) + d[2 * (i & 1) + 1]);
        }
      } else {
        const f32x4_t s = __builtin_bit_cast(f32x4_t, bv) + acc[c];
        bv = __builtin_bit_cast(uint4, s);
      }
    }
    *reinterpret_cast<uint4 *>(out + col) = bv;
  }
}

template <typename T, int RB> hipError_t launch_rank(const AdapterArgs &p, hipStream_t s) {
  constexpr int KB = (16 * RB * static_cast<int>(sizeof(T)) + 63) / 64;
  const long long tiles = ragged_max_tiles(p.S, p.R, kAdRows);
  const long long shrink = tiles * p.splits, expand = tiles * ((p.dout + kAdCols - 1) / kAdCols);
  if (std::max(shrink, expand) > kRaggedMaxBlocks) return hipErrorInvalidValue;
  adapter_shrink_kernel<T, RB><<<ragged_grid(shrink), 256, 0, s>>>(p);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  adapter_expand_kernel<T, KB><<<ragged_grid(expand), 256, 0, s>>>(p);
  return hipGetLastError();
}

template <typename T> hipError_t launch_t(const AdapterArgs &p, hipStream_t s) {
  if (p.r <= 16)
    return launch_rank<T, 1>(p, s);
  if (p.r <= 32)
    return launch_rank<T, 2>(p, s);
  if (p.r <= 64)
    return launch_rank<T, 4>(p, s);
  return launch_rank<T, 8>(p, s);
}

}  // namespace

int adapter_splits(int S, int R, int din, bool bf16) {
  const long long tiles = ragged_max_tiles(S, R, kAdRows);
  const int ks = bf16 ? 32 : 16;
  int n = 1;
  while (n < 8 && tiles * n * 2 <= 512 && din / ks >= 8 * 2 * n) n *= 2;
  return n;
}

hipError_t launch_adapter(const AdapterArgs &p, bool bf16, hipStream_t stream) {
  if (p.S <= 0) return hipSuccess;
  return bf16 ? launch_t<bf16_t>(p, stream) : launch_t<float>(p, stream);
}

}  // namespace ace
