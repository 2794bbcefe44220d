// Operands of products held in microscaled 4-bit floating point (mx4.hip): blocks of 32 consecutive numbers
// of a row, each a sign, two bits of exponent and one of mantissa (0, .5, 1, 1.5, 2, 3, 4, 6), with one
// power of two, 2^(s - 127), as their scale (s = 255: the block stands for NaN).
//   codes  [rows, K / 2] bytes, the even number of a pair in the low half
//   scales [rows, K / 32 rounded up to four] bytes; those past K / 32 are never used
//
// A stage is 128 k: per row 64 bytes of codes and four scales.  Lane (row r, group g) of a
// matrix instruction holds 32 consecutive k of a row, which is one block with one scale byte: in
// v_mfma_scale_f32_16x16x128_f8f6f4 by its definition, and in four v_mfma_f32_16x16x32_bf16, step j of which
// multiplies k 8 j .. 8 j + 7 of every lane's block, since the order of k is free as long as both operands
// agree.  So a block is read from LDS once, 16 bytes, and its scale once, wherever it goes.
#pragma once

#include "grouped_tile.h"

namespace ace {

typedef int i32x4_t __attribute__((ext_vector_type(4)));
typedef int i32x8_t __attribute__((ext_vector_type(8)));

constexpr int kMx4Block = 32;
constexpr int kMx4Stage = 128;  // k of a stage

__host__ __device__ constexpr uint32_t mx4_scale_row(int K) { return static_cast<uint32_t>((K + 127) / 128) * 4u; }

// 4 bytes per lane from descriptor + off into LDS at lds + 4 * lane (see dma16)
__device__ __forceinline__ void dma4_buf(i32x4_rsrc rsrc, uint32_t off, uint32_t lds) {
  asm volatile(
      "s_mov_b32 m0, %2\n\t"
      "s_nop 0\n\t"
      "buffer_load_dword %0, %1, 0 offen lds"
      :
      : "v"(off), "s"(rsrc), "s"(__builtin_amdgcn_readfirstlane(lds))
      : "memory", "m0");
}

template <int MATS> struct Mx4Mats {
  const uint8_t *codes[MATS], *scales[MATS];
};

// BLK 16-row blocks in 4 bits.  A unit is a block's 16 rows x 64 bytes: copy lane i brings a 16-byte chunk of row
// i / 4 to byte 16 i, chunk c of row r in slot c ^ (r / 4), so that the 16 lanes that read one chunk of all rows
// cover 256 bytes.  The scales of 64 rows are one copy of four bytes a lane.  Waves that have no unit or no rows of
// scales left copy zeros into a place of their own behind the rest, so that every wave waits for equal counts.
template <int BLK, bool PAIR, int W, int MATS = 1> struct Mx4Operand {
  using Src = Mx4Mats<MATS>;
  static constexpr int BK = kMx4Stage;
  static constexpr int UNITS = BLK, NU = (UNITS + W - 1) / W;
  static constexpr int GROUPS = (16 * BLK / MATS + 63) / 64;         // 64 rows of scales, of one matrix
  static constexpr int NS = (MATS * GROUPS + W - 1) / W;             // copies of scales of a wave
  static constexpr int COPIES = NU + NS;
  static constexpr int SCALES = UNITS * kUnitBytes;                  // where the scales lie
  static constexpr int SPARE = SCALES + MATS * GROUPS * 256;         // and what nobody reads
  static constexpr int BYTES = SPARE + (UNITS % W ? kUnitBytes : (MATS * GROUPS) % W ? 256 : 0);
  static_assert(MATS == 1 || NU == 1 || NU % 2 == 0, "two matrices: a wave's units see issue");

  const uint8_t *codes[MATS], *scales[NS];
  uint32_t code_row, scale_row;  // bytes
  uint32_t code_span, scale_span;
  int klen, chunk_k;
  uint32_t voff[NU], soff[NS];

  __device__ __forceinline__ void init(const Src &src, int ld, int valid, int k, int wave, int lane) {
    klen = k;
    code_row = static_cast<uint32_t>(ld) / 2;
    scale_row = mx4_scale_row(ld);
    code_span = static_cast<uint32_t>(valid) * code_row;
    scale_span = static_cast<uint32_t>(valid) * scale_row;
#pragma unroll
    for (int m = 0; m < MATS; ++m) codes[m] = src.codes[m];
    // offsets, not choices between pointers: those would be indexes into the arrays at run time and put them in memory
    if (MATS == 2 && NU == 1) codes[0] += (src.codes[MATS - 1] - src.codes[0]) * (wave % 2);
    const int r = lane >> 2, chunk = (lane & 3) ^ (r >> 2);
    chunk_k = kMx4Block * chunk;
#pragma unroll
    for (int t = 0; t < NU; ++t) {
      const int u = wave * NU + t;
      voff[t] = u < UNITS ? static_cast<uint32_t>(block_row<PAIR>(u / MATS, r)) * code_row + 16u * chunk : kOutside;
    }
#pragma unroll
    for (int t = 0; t < NS; ++t) {
      const int i = wave * NS + t, p = (i % GROUPS) * 64 + lane;
      const bool in = i < MATS * GROUPS && p < 16 * BLK / MATS;
      soff[t] = in ? static_cast<uint32_t>(block_row<PAIR>(p >> 4, p & 15)) * scale_row : kOutside;
      scales[t] = src.scales[0] + (MATS == 2 ? (src.scales[MATS - 1] - src.scales[0]) * min(i / GROUPS, 1) : 0);
    }
  }

  // the copies of stage s, which is within k
  __device__ __forceinline__ void issue(int s, uint32_t lds, int wave, bool once) const {
    const bool in = chunk_k < klen - s * BK;
    const uint32_t at = static_cast<uint32_t>(s) * 64u;
    const i32x4_rsrc first = make_rsrc(codes[0] + at, code_span - at);
    const i32x4_rsrc second = MATS == 2 && NU > 1 ? make_rsrc(codes[MATS - 1] + at, code_span - at) : first;
#pragma unroll
    for (int t = 0; t < NU; ++t) {
      const int u = wave * NU + t;
      const uint32_t to = lds + (u < UNITS ? u * kUnitBytes : SPARE);
      if (once)
        dma16_buf_stream(t % 2 ? second : first, in ? voff[t] : kOutside, to);
      else
        dma16_buf(t % 2 ? second : first, in ? voff[t] : kOutside, to);
    }
#pragma unroll
    for (int t = 0; t < NS; ++t) {
      const int i = wave * NS + t;
      // four scales, of which those past the end of k are not used
      dma4_buf(make_rsrc(scales[t] + 4 * s, scale_span - 4u * s), soff[t], lds + (i < MATS * GROUPS ? SCALES + i * 256 : SPARE));
    }
  }

  // block of lane (r, g) = (lane % 16, lane / 16) in 16-row block blk: k 32 g .. 32 g + 31 of row r
  static __device__ __forceinline__ i32x4_t read(const uint8_t *s, int blk, int lane) {
    const int r = lane & 15, g = lane >> 4;
    return *reinterpret_cast<const i32x4_t *>(s + blk * kUnitBytes + r * 64 + ((g ^ (r >> 2)) << 4));
  }
  // its scale; `blocks` of the stage's four are within k (the others' codes are zeros)
  static __device__ __forceinline__ int read_scale(const uint8_t *s, int blk, int lane, int blocks) {
    const int r = lane & 15, g = lane >> 4;
    const int v = s[SCALES + ((blk % MATS) * GROUPS * 64 + (blk / MATS) * 16 + r) * 4 + g];
    return g < blocks ? v : 0;
  }
};

// BLK 16-row blocks of bf16 rows, staged 128 k at a time: two halves of 64 k, each in units of 8 rows x 128 bytes as
// Operand has them
template <int BLK, int W> struct WideRows {
  using Src = Mats<1>;
  static constexpr int BK = kMx4Stage;
  static constexpr int UNITS = 4 * BLK, NU = UNITS / W, COPIES = NU;
  static constexpr int BYTES = UNITS * kUnitBytes;
  static_assert(UNITS % W == 0, "units spread evenly over the waves");

  const uint8_t *base;
  uint32_t row_bytes, span;
  int klen, chunk_k;
  uint32_t voff[NU];

  // unit u: half u / (2 BLK) of the stage
  __device__ __forceinline__ void init(const Src &src, int ld, int valid, int k, int wave, int lane) {
    base = static_cast<const uint8_t *>(src.p[0]);
    klen = k;
    row_bytes = static_cast<uint32_t>(ld) * 2;
    span = static_cast<uint32_t>(valid) * row_bytes;
    chunk_k = 8 * unit_chunk(lane);
#pragma unroll
    for (int t = 0; t < NU; ++t) {
      const int u = wave * NU + t, row = 8 * (u % (2 * BLK)) + (lane >> 3);
      voff[t] = static_cast<uint32_t>(row) * row_bytes + static_cast<uint32_t>(128 * (u / (2 * BLK)) + 2 * chunk_k);
    }
  }
  __device__ __forceinline__ void issue(int s, uint32_t lds, int wave, bool) const {
    const int left = klen - s * BK;
    const uint32_t at = static_cast<uint32_t>(s) * 256u;
    const i32x4_rsrc rsrc = make_rsrc(base + at, span - at);
#pragma unroll
    for (int t = 0; t < NU; ++t) {
      const int u = wave * NU + t;
      dma16_buf(rsrc, 64 * (u / (2 * BLK)) + chunk_k < left ? voff[t] : kOutside, lds + u * kUnitBytes);
    }
  }
  // k 32 g + 8 j .. + 7 of row lane % 16 of block blk, g = lane / 16
  static __device__ __forceinline__ bf16x8_t read(const uint8_t *s, int blk, int j, int lane) {
    const int r = lane & 15, g = lane >> 4, rlo = r & 7;
    return *reinterpret_cast<const bf16x8_t *>(s + ((g >> 1) * 2 * BLK + 2 * blk + (r >> 3)) * kUnitBytes + rlo * 128 +
                                               (((4 * (g & 1) + j) ^ rlo) << 4));
  }
};

// 8 numbers of a block as bf16, which holds every one of them exactly: dword j of its codes, times 2^(s - 127) in `scale`,
// of which the conversion takes the exponent alone (s = 255 gives NaN)
__device__ __forceinline__ bf16x8_t mx4_to_bf16(uint32_t codes, float scale) {
  typedef __bf16 bf16x2_v __attribute__((ext_vector_type(2)));
  typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
  const bf16x2_v a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0);
  const bf16x2_v b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1);
  const bf16x2_v c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2);
  const bf16x2_v d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3);
  return __builtin_bit_cast(bf16x8_t, u32x4_t{__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b),
                                              __builtin_bit_cast(uint32_t, c), __builtin_bit_cast(uint32_t, d)});
}

// Tiles of bf16 results (see DenseTile) on 4-bit weights: rows in bf16 (ROWS4 = false) by bf16 matrix instructions on
// the weights' exact values, or rows in 4 bits too, by the scaled instruction
template <bool ROWS4, int MB_, int NB_, int WR_, int WC_, int DA_, int DB_, int MATS> struct Mx4Tile {
  using T = bf16_t;
  static constexpr int MB = MB_, NB = NB_, WR = WR_, WC = WC_, DA = DA_, DB = DB_, SEG = 1;
  static constexpr int MW = MB / WR, NW = NB / WC;
  using A = std::conditional_t<ROWS4, Mx4Operand<MB, false, WR * WC>, WideRows<MB, WR * WC>>;
  using B = Mx4Operand<NB, true, WR * WC, MATS>;
  using Ref = TileRef<T, typename A::Src, typename B::Src>;
  static constexpr int LDS = DA * A::BYTES + DB * B::BYTES;

  static __device__ __forceinline__ void multiply(const uint8_t *pa, const uint8_t *pb, int wr, int wc, int lane, int rows,
                                                  int left, f32x4_t (&acc)[MW][NW]) {
    const int blocks = left / kMx4Block;
    i32x4_t bq[NW];
    int bs[NW];
#pragma unroll
    for (int j = 0; j < NW; ++j) {
      bq[j] = B::read(pb, wc * NW + j, lane);
      bs[j] = B::read_scale(pb, wc * NW + j, lane, blocks);
    }
    if constexpr (ROWS4) {
      i32x4_t aq[MW];
      int as[MW];
#pragma unroll
      for (int i = 0; i < MW; ++i) {
        aq[i] = A::read(pa, wr + WR * i, lane);
        as[i] = A::read_scale(pa, wr + WR * i, lane, blocks);
      }
      auto wide = [](i32x4_t v) { return i32x8_t{v[0], v[1], v[2], v[3], 0, 0, 0, 0}; };
#pragma unroll
      for (int i = 0; i < MW; ++i)
        if (16 * (wr + WR * i) < rows) {  // wave-uniform
#pragma unroll
          for (int j = 0; j < NW; ++j)    // 4: both operands in this format
            acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wide(bq[j]), wide(aq[i]), acc[i][j], 4, 4, 0, bs[j],
                                                                        0, as[i]);
        }
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        bf16x8_t bf[NW], af[MW];
#pragma unroll
        for (int i = 0; i < MW; ++i) af[i] = A::read(pa, wr + WR * i, j, lane);
#pragma unroll
        for (int c = 0; c < NW; ++c) bf[c] = mx4_to_bf16(bq[c][j], __uint_as_float(static_cast<uint32_t>(bs[c]) << 23));
#pragma unroll
        for (int i = 0; i < MW; ++i)
          if (16 * (wr + WR * i) < rows) {  // wave-uniform
#pragma unroll
            for (int c = 0; c < NW; ++c) acc[i][c] = Frag<bf16_t>::mma(bf[c], af[i], 0, acc[i][c]);
          }
      }
    }
  }
};

}  // namespace ace
