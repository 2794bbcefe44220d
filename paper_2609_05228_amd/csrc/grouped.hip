// Matrix products grouped by expert with ragged sizes, and their gradients.  Rows of x
// [S, K] lie in group order (group e: rows offsets[e] .. offsets[e + 1] - 1), group e has
// the weights w[e] [M, K] (nn.Linear layout):
//   forward          y[r]  = w[e] x[r]                      reduced over K
//   rows' gradient   dx[r] = w[e]^T dy[r]                   reduced over M
//   weights' one     dw[e] = sum over rows r of e: dy[r] x[r]^T   reduced over the group's rows
// One tile body serves the three: C[i, j] = sum_k A(i, k) B(j, k), where an operand lies
// either with k along its rows ("k-major": x, dy, and w in the forward) or with k down its
// rows ("k down": w in the rows' gradient, dy and x in the weights' one).
//
// Staging: a stage of 128 bytes of k per row (64 bf16, 32 fp32) is copied HBM/L2 -> LDS in
// units of 8 rows x 128 bytes, one buffer_load_dwordx4 .. lds each, whole cache lines.  The
// buffer descriptor ends at the operand's last row of the tile, so rows past a ragged end
// read as zero; chunks past the end of k or of the columns get an offset outside it.  Zeros
// in both operands add nothing, whatever bits (NaN, infinities) lie behind the end.
// bf16 operands with k down are read back through the transposing LDS read
// (ds_read_b64_tr_b16), so no transposed copy of w, x or dy is ever made.
//
// The products go to the matrix cores as mfma(B, A): a lane then holds consecutive columns
// of one row, and with the columns of two 16-column blocks interleaved in fours (bf16) it
// stores 16 bytes at a time.  Sums are fp32, rounded once.
#include "lds_dma.h"
#include "ragged.h"

namespace ace {

namespace {

typedef int i32x4_rsrc __attribute__((ext_vector_type(4)));
typedef short i16x4_t __attribute__((ext_vector_type(4)));

constexpr uint32_t kOutside = 0x7ffffff0u;  // past any descriptor (a tile spans less than 2^31 bytes)

// 16 bytes per lane from descriptor + off into LDS at lds + 16 * lane (see dma16)
__device__ __forceinline__ void dma16_buf(i32x4_rsrc rsrc, uint32_t off, uint32_t lds) {
  asm volatile(
      "s_mov_b32 m0, %2\n\t"
      "s_nop 0\n\t"
      "buffer_load_dwordx4 %0, %1, 0 offen lds"
      :
      : "v"(off), "s"(rsrc), "s"(__builtin_amdgcn_readfirstlane(lds))
      : "memory", "m0");
}

__device__ __forceinline__ i32x4_rsrc make_rsrc(const void *p, uint32_t bytes) {
  const uint64_t b = reinterpret_cast<uint64_t>(p);
  return i32x4_rsrc{__builtin_amdgcn_readfirstlane(static_cast<int>(b)),
                    __builtin_amdgcn_readfirstlane(static_cast<int>(b >> 32) & 0xffff),
                    __builtin_amdgcn_readfirstlane(static_cast<int>(bytes)), 0x00020000};
}

// One operand of a tile: BLK 16-row blocks of C's rows (or columns).
//   DOWN = false: p points at the tile's first row; `valid` rows of ld elements, k along them
//   DOWN = true:  p points at the tile's first column of k's first row; `valid` columns
// PAIR (bf16 columns of C): the columns of a 32-column pair of blocks interleaved in fours:
// position q of block b holds column 8 (q / 4) + 4 b + q % 4.
template <typename T, bool DOWN, int BLK, bool PAIR, int W> struct Operand {
  static constexpr int ES = sizeof(T), E = kChunkElems<T>, BK = kStageElems<T>;
  static constexpr int UNITS = 2 * BLK;              // per stage
  static constexpr int NU = (UNITS + W - 1) / W;     // per wave
  static constexpr int OU = DOWN ? BLK * 16 / BK : 1;  // k down: units across
  static constexpr int BYTES = UNITS * kUnitBytes;
  static_assert(UNITS % W == 0, "units spread evenly over the waves");
  static_assert(!DOWN || (BLK * 16) % BK == 0, "whole units across");
  typedef typename Frag<T>::type frag_t;

  const uint8_t *base;
  uint32_t row_bytes, span;  // span: k-major: bytes to the end of the last row; k down: of a row, from p on
  int klen, chunk_k;
  uint32_t voff[NU];

  // LDS slot of chunk c in row r of unit u: k-major reads take one chunk of 16 rows (see
  // lds_dma.h); transposing reads take 8 bytes of two or four chunks from 4 rows of every
  // other unit, so rows two apart and neighbouring units go to other banks
  static __device__ __forceinline__ int swz(int r, int ku) {
    if (!DOWN) return r;
    return ES == 2 ? (((r & 2) << 1) ^ ((ku & 1) << 1)) : (r & 4);
  }

  __device__ __forceinline__ void init(const void *p, int ld, int valid, int k, int wave, int lane) {
    base = static_cast<const uint8_t *>(p);
    klen = k;
    row_bytes = static_cast<uint32_t>(ld) * ES;
    const int ur = lane >> 3, slot = lane & 7;
    if (!DOWN) {
      span = static_cast<uint32_t>(valid) * row_bytes;
      chunk_k = E * (slot ^ swz(ur, 0));
    } else {
      span = static_cast<uint32_t>(valid) * ES;
    }
#pragma unroll
    for (int t = 0; t < NU; ++t) {
      const int u = wave * NU + t;
      if (!DOWN) {
        const int blk = u >> 1, q = 8 * (u & 1) + ur;
        const int row = PAIR ? 32 * (blk >> 1) + 8 * (q >> 2) + 4 * (blk & 1) + (q & 3) : 16 * blk + q;
        voff[t] = static_cast<uint32_t>(row) * row_bytes + static_cast<uint32_t>(chunk_k) * ES;
      } else {
        const int ku = u / OU, ou = u % OU;
        const uint32_t col = static_cast<uint32_t>(ou * BK + E * (slot ^ swz(ur, ku))) * ES;
        voff[t] = col < span ? static_cast<uint32_t>(8 * ku + ur) * row_bytes + col : kOutside;
      }
    }
  }

  // stage s into LDS at `lds`
  __device__ __forceinline__ void issue(int s, uint32_t lds, int wave) const {
    const int left = klen - s * BK;  // k from this stage on
    if (!DOWN) {
      const i32x4_rsrc r = make_rsrc(base + static_cast<size_t>(s) * BK * ES, span - static_cast<uint32_t>(s * BK * ES));
      const bool in = chunk_k < left;
#pragma unroll
      for (int t = 0; t < NU; ++t) dma16_buf(r, in ? voff[t] : kOutside, lds + (wave * NU + t) * kUnitBytes);
    } else {
      const i32x4_rsrc r = make_rsrc(base + static_cast<size_t>(s) * BK * row_bytes,
                                     static_cast<uint32_t>(min(left, BK) - 1) * row_bytes + span);
#pragma unroll
      for (int t = 0; t < NU; ++t) dma16_buf(r, voff[t], lds + (wave * NU + t) * kUnitBytes);
    }
  }

  // fragment of block blk for half h of the stage at `s`: k 8 g .. 8 g + 7 of the half's 32
  // (fp32: 4 g .. 4 g + 3 of 16) for row (column) lane % 16
  static __device__ __forceinline__ frag_t read(const uint8_t *s, int blk, int h, int lane) {
    if constexpr (!DOWN) {
      return *reinterpret_cast<const frag_t *>(s + blk * 2 * kUnitBytes + unit_read_offset(lane, h));
    } else if constexpr (ES == 2) {
      const int i = lane & 15, g = lane >> 4, r = i >> 2, j = i & 3, ku = 4 * h + g;
      const int chunk = PAIR ? 4 * ((blk >> 1) & 1) + j : 2 * (blk & 3) + (j >> 1);
      const int half = PAIR ? 8 * (blk & 1) : 8 * (j & 1);
      const uint8_t *u = s + (ku * OU + (blk >> 2)) * kUnitBytes + r * 128 + ((chunk ^ swz(r, ku)) << 4) + half;
      typedef __attribute__((address_space(3))) i16x4_t lds_t;
      // rows r and r + 4 share their swizzle
      const i16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t *)(u));
      const i16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t *)(u + 4 * 128));
      typedef short i16x8_t __attribute__((ext_vector_type(8)));
      return __builtin_bit_cast(frag_t, i16x8_t{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]});
    } else {
      const int i = lane & 15, g = lane >> 4, ku = 2 * h + (g >> 1);
      const int chunk = 4 * (blk & 1) + (i >> 2);
      frag_t f;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int r = 4 * (g & 1) + j;
        f[j] = *reinterpret_cast<const float *>(s + (ku * OU + (blk >> 1)) * kUnitBytes + r * 128 +
                                                 ((chunk ^ swz(r, ku)) << 4) + 4 * (i & 3));
      }
      return f;
    }
  }
};

// waits for this wave's LDS reads and all but n of its copies, then for the workgroup
template <int N> __device__ __forceinline__ void stage_barrier() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

// One tile of C: MB x NB 16-blocks at (rows 0.., columns 0..) of out (leading dimension
// ldo), rows_valid x cols_valid of it stored.  WR x WC waves, a ring of D stages.
template <typename T, bool ADOWN, bool BDOWN, int MB, int NB, int WR, int WC, int D>
__device__ __forceinline__ void grouped_tile(const void *a, int lda, const void *b, int ldb, int klen, T *out,
                                             size_t ldo, int rows_valid, int cols_valid, uint8_t *smem) {
  constexpr int W = WR * WC, MW = MB / WR, NW = NB / WC;
  constexpr bool PAIR = sizeof(T) == 2;
  using A = Operand<T, ADOWN, MB, false, W>;
  using B = Operand<T, BDOWN, NB, PAIR, W>;
  constexpr int STAGE = A::BYTES + B::BYTES;
  constexpr int OPS = A::NU + B::NU;
  constexpr int BK = A::BK;
  static_assert(MB % WR == 0 && NB % WC == 0 && NW % 2 == 0, "whole blocks, pairs of column blocks per wave");
  static_assert(D >= 2 && (D - 2) * OPS <= 63, "outstanding copies exceed the wait counter");
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wr = wave / WC, wc = wave % WC;
  A oa;
  B ob;
  oa.init(a, lda, rows_valid, klen, wave, lane);
  ob.init(b, ldb, cols_valid, klen, wave, lane);
  f32x4_t acc[MW][NW];
#pragma unroll
  for (int i = 0; i < MW; ++i)
#pragma unroll
    for (int j = 0; j < NW; ++j) acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  const int nk = (klen + BK - 1) / BK;
  const uint32_t lds = lds_addr(smem);
  auto issue = [&](int s) {
    const uint32_t st = lds + (s % D) * STAGE;
    oa.issue(s, st, wave);
    ob.issue(s, st + A::BYTES, wave);
  };
#pragma unroll
  for (int s = 0; s < D - 1; ++s)
    if (s < nk) issue(s);
  for (int kt = 0; kt < nk; ++kt) {
    // stage kt landed for every wave, and every wave is done with the slot refilled below
    if (kt + D - 2 < nk)
      stage_barrier<(D - 2) * OPS>();
    else if (D > 3 && kt + D - 3 < nk)
      stage_barrier<(D > 3 ? D - 3 : 0) * OPS>();
    else
      stage_barrier<0>();
    if (kt + D - 1 < nk) issue(kt + D - 1);
    const uint8_t *sa = smem + (kt % D) * STAGE, *sb = sa + A::BYTES;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      typename B::frag_t bf[NW];
#pragma unroll
      for (int j = 0; j < NW; ++j) bf[j] = B::read(sb, wc * NW + j, h, lane);
#pragma unroll
      for (int i = 0; i < MW; ++i) {
        const typename A::frag_t af = A::read(sa, wr + WR * i, h, lane);
#pragma unroll
        for (int s = 0; s < Frag<T>::steps; ++s)
#pragma unroll
          for (int j = 0; j < NW; ++j) acc[i][j] = Frag<T>::mma(bf[j], af, s, acc[i][j]);
      }
    }
  }
  const int r16 = lane & 15, g = lane >> 4;
#pragma unroll
  for (int i = 0; i < MW; ++i) {
    const int row = 16 * (wr + WR * i) + r16;
    if (row >= rows_valid) continue;
    T *o = out + static_cast<size_t>(row) * ldo;
    if constexpr (PAIR) {
#pragma unroll
      for (int j = 0; j < NW; j += 2) {
        const int col = 16 * (wc * NW + j) + 8 * g;
        if (col >= cols_valid) continue;
        const f32x4_t lo = acc[i][j], hi = acc[i][j + 1];
        *reinterpret_cast<uint4 *>(o + col) = uint4{pack_bf16x2(lo[0], lo[1]), pack_bf16x2(lo[2], lo[3]),
                                                    pack_bf16x2(hi[0], hi[1]), pack_bf16x2(hi[2], hi[3])};
      }
    } else {
#pragma unroll
      for (int j = 0; j < NW; ++j) {
        const int col = 16 * (wc * NW + j) + 4 * g;
        if (col < cols_valid) *reinterpret_cast<f32x4_t *>(o + col) = acc[i][j];
      }
    }
  }
}

// zeros into rows_valid x cols_valid of out
template <typename T>
__device__ __forceinline__ void zero_tile(T *out, size_t ldo, int rows_valid, int cols_valid) {
  constexpr int E = kChunkElems<T>;
  const int chunks = cols_valid / E;
  for (int i = threadIdx.x; i < rows_valid * chunks; i += blockDim.x)
    *reinterpret_cast<uint4 *>(out + static_cast<size_t>(i / chunks) * ldo + (i % chunks) * E) = uint4{0, 0, 0, 0};
}

// Forward (GX = false) and rows' gradient (GX = true): tile = TM rows of one group x BN columns
template <typename T, bool GX, int MB, int NB, int WR, int WC, int D>
__global__ __launch_bounds__(WR *WC * 64) void grouped_rows_kernel(GroupedArgs g) {
  constexpr int TM = 16 * MB, BN = 16 * NB;
  constexpr int TML = TM == 256 ? 8 : TM == 128 ? 7 : TM == 64 ? 6 : TM == 32 ? 5 : 4;
  static_assert(1 << TML == TM, "tile rows");
  __shared__ __align__(16) uint8_t smem[D * (MB + NB) * 2 * kUnitBytes];
  const int cols = GX ? g.K : g.M, klen = GX ? g.M : g.K;
  const int nN = (cols + BN - 1) / BN;
  // the column tiles of one row tile share an XCD (block b runs on XCD b % 8), so the rows
  // they share stay in its L2
  const int b = ragged_block();
  const int tile = (b & 7) + 8 * ((b >> 3) / nN), nt = (b >> 3) % nN;
  const RaggedTile t = ragged_tile(g.offsets, g.N, g.S, TML, tile, g.fill);
  if (!t.valid) return;
  const int c0 = nt * BN, cv = min(BN, cols - c0);
  T *out = static_cast<T *>(g.out) + static_cast<size_t>(t.row0) * cols + c0;
  if (t.group < 0) {
    zero_tile(out, cols, t.rows, cv);
    return;
  }
  const T *rows = static_cast<const T *>(g.rows) + static_cast<size_t>(t.row0) * klen;
  const T *w = static_cast<const T *>(g.other) + static_cast<size_t>(t.group) * g.M * g.K;
  grouped_tile<T, false, GX, MB, NB, WR, WC, D>(rows, klen, GX ? w + c0 : w + static_cast<size_t>(c0) * g.K, g.K, klen,
                                                 out, cols, t.rows, cv, smem);
}

// Weights' gradient: tile = 16 MB rows x 16 NB columns of one group's dw
template <typename T, int MB, int NB, int WR, int WC, int D>
__global__ __launch_bounds__(WR *WC * 64) void grouped_weights_kernel(GroupedArgs g) {
  constexpr int BM = 16 * MB, BN = 16 * NB;
  __shared__ __align__(16) uint8_t smem[D * (MB + NB) * 2 * kUnitBytes];
  const int nM = (g.M + BM - 1) / BM, nN = (g.K + BN - 1) / BN;
  const int b = ragged_block();
  const int e = (b & 7) + 8 * ((b >> 3) / (nM * nN)), q = (b >> 3) % (nM * nN);
  if (e >= g.N) return;
  const int r0 = min(max(g.offsets[e], 0), g.S), r1 = min(max(g.offsets[e + 1], r0), g.S);
  const int m0 = q / nN * BM, k0 = q % nN * BN;
  const int mv = min(BM, g.M - m0), kv = min(BN, g.K - k0);
  const T *dy = static_cast<const T *>(g.rows) + static_cast<size_t>(r0) * g.M + m0;
  const T *x = static_cast<const T *>(g.other) + static_cast<size_t>(r0) * g.K + k0;
  T *out = static_cast<T *>(g.out) + (static_cast<size_t>(e) * g.M + m0) * g.K + k0;
  grouped_tile<T, true, true, MB, NB, WR, WC, D>(dy, g.M, x, g.K, r1 - r0, out, g.K, mv, kv, smem);
}

template <typename T, bool GX> hipError_t launch_rows(const GroupedArgs &g, hipStream_t s) {
  constexpr int MB = sizeof(T) == 2 ? 8 : 4, NB = sizeof(T) == 2 ? 8 : 4;
  const int nN = ((GX ? g.K : g.M) + 16 * NB - 1) / (16 * NB);
  const long long blocks = (ragged_max_tiles(g.S, g.N, 16 * MB) + 7) / 8 * 8 * nN;
  if (blocks > kRaggedMaxBlocks) return hipErrorInvalidValue;
  grouped_rows_kernel<T, GX, MB, NB, 2, 2, 2><<<ragged_grid(blocks), 256, 0, s>>>(g);
  return hipGetLastError();
}

template <typename T> hipError_t launch_weights(const GroupedArgs &g, hipStream_t s) {
  constexpr int MB = sizeof(T) == 2 ? 8 : 4, NB = sizeof(T) == 2 ? 8 : 4;
  const long long nM = (g.M + 16 * MB - 1) / (16 * MB), nN = (g.K + 16 * NB - 1) / (16 * NB);
  const long long blocks = (g.N + 7) / 8 * 8 * nM * nN;
  if (blocks > kRaggedMaxBlocks) return hipErrorInvalidValue;
  grouped_weights_kernel<T, MB, NB, 2, 2, 2><<<ragged_grid(blocks), 256, 0, s>>>(g);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_grouped_rows(const GroupedArgs &g, bool grad, bool bf16, hipStream_t stream) {
  if (g.S <= 0) return hipSuccess;
  if (bf16) return grad ? launch_rows<bf16_t, true>(g, stream) : launch_rows<bf16_t, false>(g, stream);
  return grad ? launch_rows<float, true>(g, stream) : launch_rows<float, false>(g, stream);
}

hipError_t launch_grouped_weights(const GroupedArgs &g, bool bf16, hipStream_t stream) {
  return bf16 ? launch_weights<bf16_t>(g, stream) : launch_weights<float>(g, stream);
}

}  // namespace ace
