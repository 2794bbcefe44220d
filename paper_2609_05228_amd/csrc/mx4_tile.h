// Operands of products held in microscaled 4-bit floating point (mx4.hip): blocks of 32 consecutive numbers
// of a row, each a sign, two bits of exponent and one of mantissa (0, .5, 1, 1.5, 2, 3, 4, 6), with one
// power of two, 2^(s - 127), as their scale (s = 255: the block stands for NaN).
//   codes  [rows, K / 2] bytes, the even number of a pair in the low half
//   scales [rows, K / 32 rounded up to four] bytes; those past K / 32 are never used
//
// A stage is 128 k.  Lane (row r, group g) of a matrix instruction takes k 32 g .. 32 g + 31 of a row, which is one block
// with one scale: in v_mfma_scale_f32_16x16x128_f8f6f4 by definition, and in four v_mfma_f32_16x16x32_bf16, step j of
// which multiplies k 8 j .. 8 j + 7 of every lane's block, since the order of k is free as long as both operands agree.
// So a lane reads its codes of a stage from LDS at once and one scale for them.
//
// LDS: ds_read_b128 serves 16 lanes at a time, four from each end of one group of 16 rows and the middle eight of the next group
// (0-3, 12-15, 20-27, as timing of address patterns shows), so chunks of neighbouring groups have to go to other banks too.
//
// Scales come in panels of 512 k, 16 bytes a row: a stage's own four bytes of each row would be as many trips to
// the cache as the codes.
#pragma once

#include "grouped_tile.h"

namespace ace {

typedef int i32x4_t __attribute__((ext_vector_type(4)));
typedef int i32x8_t __attribute__((ext_vector_type(8)));

constexpr int kMx4Block = 32;
constexpr int kMx4Stage = 128;  // k of a stage
constexpr int kMx4Panel = 512;  // of a panel of scales

__host__ __device__ constexpr uint32_t mx4_scale_row(int K) { return static_cast<uint32_t>((K + 127) / 128) * 4u; }

// Where an operand lies: its first rows from their first k, of which the reduction starts at k0
template <int MATS> struct Mx4Mats {
  const uint8_t *codes[MATS], *scales[MATS];
  int k0;  // whole stages
};

// BLK 16-row blocks in 4 bits.  With two matrices block b is block b / 2 of matrix b % 2; in LDS all of the first one's come
// first.  A unit is a block, 1 KB: copy lane i brings a 16-byte chunk of row i / 4 to byte 16 i, chunk c of row r in slot
// c ^ (r / 2 % 4), which reads at the full rate (twice that of r / 4).  Waves that have no unit left copy zeros into a
// place behind the rest, so that every wave waits for equal counts.  A panel is 64 rows a copy, 16 bytes a lane (its rows
// are padded to 4 bytes only, so the addresses are multiples of 4).  Where less than that is left of a row a copy brings the
// start of the next one, so the descriptors end with the last row, which k0 brings nearer to where they start.
template <int BLK, bool PAIR, int W, int MATS = 1> struct Mx4Operand {
  using Src = Mx4Mats<MATS>;
  static constexpr int BK = kMx4Stage;
  static constexpr int UNITS = BLK, NU = (UNITS + W - 1) / W, COPIES = NU;
  static constexpr int BYTES = (UNITS + (UNITS % W ? 1 : 0)) * kUnitBytes;
  static constexpr int ROWS = 16 * BLK / MATS, GROUPS = (ROWS + 63) / 64;  // of one matrix; copies of its panel
  static constexpr int NP = (MATS * GROUPS + W - 1) / W;
  static constexpr int PANEL = MATS * GROUPS * kUnitBytes, PANEL_STAGES = kMx4Panel / BK;
  static_assert(UNITS % MATS == 0 && (MATS == 1 || W == 1 || UNITS / MATS % NU == 0),
                "all units of a wave of one matrix where there are several waves");

  const uint8_t *codes, *codes2, *scales[NP];
  uint32_t code_row, scale_row;  // bytes
  uint32_t code_span, scale_span;
  int klen, chunk_k;
  uint32_t voff[NU], poff[NP];

  __host__ __device__ __forceinline__ void init(const Src &src, int ld, int valid, int k, int wave, int lane) {
    klen = k;
    code_row = static_cast<uint32_t>(ld) / 2;
    scale_row = mx4_scale_row(ld);
    const uint32_t codes0 = static_cast<uint32_t>(src.k0) / 2, scales0 = static_cast<uint32_t>(src.k0) / kMx4Block;
    code_span = static_cast<uint32_t>(valid) * code_row - codes0;
    scale_span = static_cast<uint32_t>(valid) * scale_row - scales0;
    // offsets, not choices between pointers: those would be indexes into the arrays at run time and put them in memory
    codes = src.codes[0] + codes0;
    codes2 = src.codes[MATS - 1] + codes0;  // a lone wave's second half of units
    if (MATS == 2 && W > 1) codes += (src.codes[MATS - 1] - src.codes[0]) * (wave * NU >= UNITS / MATS);
    const int r = lane >> 2, chunk = (lane & 3) ^ swap(r);
    chunk_k = kMx4Block * chunk;
#pragma unroll
    for (int t = 0; t < NU; ++t) {
      const int u = wave * NU + t;
      voff[t] = u < UNITS ? static_cast<uint32_t>(block_row<PAIR>(u % (UNITS / MATS), r)) * code_row + 16u * chunk : kOutside;
    }
#pragma unroll
    for (int t = 0; t < NP; ++t) {
      const int i = wave * NP + t, p = i % GROUPS * 64 + lane;
      poff[t] = p < ROWS ? static_cast<uint32_t>(block_row<PAIR>(p >> 4, p & 15)) * scale_row : kOutside;
      scales[t] = src.scales[0] + scales0;
      if (MATS == 2) scales[t] += (src.scales[MATS - 1] - src.scales[0]) * (i >= GROUPS);
    }
  }
  static __host__ __device__ __forceinline__ int swap(int r) { return (r >> 1) & 3; }
  // of a stage: bytes that its codes, and the panel that holds its scales, lie behind the part's first ones
  static __host__ __device__ __forceinline__ uint32_t codes_at(int s) { return static_cast<uint32_t>(s) * (BK / 2); }
  static __host__ __device__ __forceinline__ uint32_t panel_at(int s) { return static_cast<uint32_t>(s / PANEL_STAGES) * 16u; }
  __host__ __device__ __forceinline__ bool in_stage(int s) const { return chunk_k < klen - s * BK; }

  // the copies of stage s, which is within k, and of its panel where there is a place for it
  __device__ __forceinline__ void issue(int s, uint32_t lds, uint32_t panel, int wave, bool) const {
    if (panel) {
      const uint32_t at = panel_at(s);
#pragma unroll
      for (int t = 0; t < NP; ++t)
        if (wave * NP + t < MATS * GROUPS)
          dma16_buf(make_rsrc(scales[t] + at, scale_span - at), poff[t], panel + (wave * NP + t) * kUnitBytes);
    }
    const bool in = in_stage(s);
    const uint32_t at = codes_at(s);
    const i32x4_rsrc first = make_rsrc(codes + at, code_span - at);
    const i32x4_rsrc second = MATS == 2 && W == 1 ? make_rsrc(codes2 + at, code_span - at) : first;
#pragma unroll
    for (int t = 0; t < NU; ++t) {
      const uint32_t to = lds + min(wave * NU + t, UNITS) * kUnitBytes;
      // no non-temporal hint: a stage takes half or a quarter of a line of each row, and the next ones the rest (products
      // of 256 rows in 128 groups, 2048 x 768: 35.4 us with the hint, 29.1 without)
      dma16_buf(t < UNITS / MATS ? first : second, in ? voff[t] : kOutside, to);
    }
  }

  // the lane's codes: k 32 g .. 32 g + 31 of row r of block blk, (r, g) = (lane % 16, lane / 16)
  static __host__ __device__ __forceinline__ i32x4_t read(const uint8_t *s, int blk, int lane) {
    const int r = lane & 15, g = lane >> 4;
    return *reinterpret_cast<const i32x4_t *>(s + (blk % MATS * (BLK / MATS) + blk / MATS) * kUnitBytes + r * 64 +
                                              ((g ^ swap(r)) << 4));
  }
  // their scale, for the stage from k on of klen: one that is not of a block within klen (whose codes are zeros) may
  // be anything, and is 0 here
  static __host__ __device__ __forceinline__ int read_scale(const uint8_t *panel, int blk, int lane, int k, int klen) {
    const int b = lane >> 4;  // of the stage's blocks
    const int row = blk % MATS * (GROUPS * 64) + blk / MATS * 16 + (lane & 15);
    const int v = panel[row * 16 + (k % kMx4Panel / kMx4Block + b)];
    return k + kMx4Block * b < klen ? v : 0;
  }
};

// BLK 16-row blocks of bf16 rows: halves of 64 k of the stage, each in units of 8 rows x 128 bytes as Operand has them, but
// chunk c of row r in slot turn(c) ^ r: chunks that neighbouring groups of lanes read together, c and c + 4, then
// differ in the slot's last bit (as c ^ r they meet in the same banks: half the rate).
template <int BLK, int W> struct Mx4Rows {
  using Src = Mats<1>;
  static constexpr int BK = kMx4Stage, UNITS = 4 * BLK, NU = UNITS / W, COPIES = NU;
  static constexpr int BYTES = UNITS * kUnitBytes, PANEL = 0, PANEL_STAGES = kMx4Panel / BK;
  static_assert(UNITS % W == 0, "units spread evenly over the waves");

  const uint8_t *base;
  uint32_t row_bytes, span;
  int klen, chunk_k;
  uint32_t voff[NU];

  static __device__ __forceinline__ int turn(int c) { return (c & 3) << 1 | c >> 2; }
  static __device__ __forceinline__ int turn_back(int s) { return s >> 1 | (s & 1) << 2; }

  // unit u: half u / (2 BLK) of the stage
  __device__ __forceinline__ void init(const Src &src, int ld, int valid, int k, int wave, int lane) {
    base = static_cast<const uint8_t *>(src.p[0]);
    klen = k;
    row_bytes = static_cast<uint32_t>(ld) * 2;
    span = static_cast<uint32_t>(valid) * row_bytes;
    chunk_k = 8 * turn_back((lane & 7) ^ (lane >> 3));
#pragma unroll
    for (int t = 0; t < NU; ++t) {
      const int u = wave * NU + t, row = 8 * (u % (2 * BLK)) + (lane >> 3);
      voff[t] = static_cast<uint32_t>(row) * row_bytes + static_cast<uint32_t>(128 * (u / (2 * BLK)) + 2 * chunk_k);
    }
  }
  __device__ __forceinline__ void issue(int s, uint32_t lds, uint32_t, int wave, bool) const {
    const int left = klen - s * BK;
    const uint32_t at = static_cast<uint32_t>(s) * (2 * BK);
    const i32x4_rsrc rsrc = make_rsrc(base + at, span - at);
#pragma unroll
    for (int t = 0; t < NU; ++t) {
      const int u = wave * NU + t;
      dma16_buf(rsrc, 64 * (u / (2 * BLK)) + chunk_k < left ? voff[t] : kOutside, lds + u * kUnitBytes);
    }
  }
  // k 32 g + 8 j .. + 7 of row r of block blk, (r, g) = (lane % 16, lane / 16)
  static __device__ __forceinline__ bf16x8_t read(const uint8_t *s, int blk, int j, int lane) {
    const int r = lane & 15, rlo = r & 7, g = lane >> 4;
    return *reinterpret_cast<const bf16x8_t *>(s + ((g >> 1) * 2 * BLK + 2 * blk + (r >> 3)) * kUnitBytes + rlo * 128 +
                                               ((turn(4 * (g & 1) + j) ^ rlo) << 4));
  }
};

// 8 numbers of a block as bf16, which holds every one below 2^128 exactly, subnormal ones among them (the others, which only
// scales 253 and 254 reach, become infinite): dword j of its codes, times 2^(s - 127) in `scale`, of which the conversion
// takes the exponent alone (s = 255 gives NaN)
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
// the weights in bf16 (see mx4_to_bf16), or rows in 4 bits too, by the scaled instruction
template <bool ROWS4_, int MB_, int NB_, int WR_, int WC_, int DA_, int DB_, int MATS> struct Mx4Tile {
  using T = bf16_t;
  static constexpr bool ROWS4 = ROWS4_;
  static constexpr int MB = MB_, NB = NB_, WR = WR_, WC = WC_, DA = DA_, DB = DB_, SEG = 1;
  static constexpr int MW = MB / WR, NW = NB / WC;
  using A = std::conditional_t<ROWS4, Mx4Operand<MB, false, WR * WC>, Mx4Rows<MB, WR * WC>>;
  using B = Mx4Operand<NB, true, WR * WC, MATS>;
  using Ref = TileRef<T, typename A::Src, typename B::Src>;
  static constexpr int LDS = DA * (A::BYTES + A::PANEL) + DB * (B::BYTES + B::PANEL);

  template <typename M>
  static __device__ __forceinline__ void multiply(const uint8_t *pa, const uint8_t *pb, const uint8_t *qa, const uint8_t *qb,
                                                  int wr, int wc, int lane, int rows, int k, int klen,
                                                  f32x4_t (&acc)[MW][NW], M mid) {
    i32x4_t bq[NW];
    int bs[NW];
#pragma unroll
    for (int j = 0; j < NW; ++j) {
      bq[j] = B::read(pb, wc * NW + j, lane);
      bs[j] = B::read_scale(qb, wc * NW + j, lane, k, klen);
    }
    if constexpr (ROWS4) {
      i32x4_t aq[MW];
      int as[MW];
#pragma unroll
      for (int i = 0; i < MW; ++i) {
        aq[i] = A::read(pa, wr + WR * i, lane);
        as[i] = A::read_scale(qa, wr + WR * i, lane, k, klen);
      }
      auto wide = [](i32x4_t v) { return i32x8_t{v[0], v[1], v[2], v[3], 0, 0, 0, 0}; };
#pragma unroll
      for (int i = 0; i < MW; ++i) {
        if (i == MW / 2) mid();
        if (16 * (wr + WR * i) < rows) {  // wave-uniform
#pragma unroll
          for (int j = 0; j < NW; ++j)    // 4: both operands in this format
            acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wide(bq[j]), wide(aq[i]), acc[i][j], 4, 4, 0, bs[j],
                                                                        0, as[i]);
        }
      }
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (j == 2) mid();
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
