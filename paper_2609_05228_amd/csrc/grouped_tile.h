// The tile pipeline of the products grouped by expert (grouped.hip, gated.hip, mx4.hip):
// C[i, j] = sum_k A(i, k) B(j, k) for a workgroup's list of tiles, operands staged through
// rings in LDS.  An operand lies either with k along its rows ("k-major") or with k down its
// rows ("k down").
//
// Staging: a stage of 128 bytes of k per row (64 bf16, 32 fp32) is copied HBM/L2 -> LDS in
// units of 8 rows x 128 bytes, one buffer_load_dwordx4 .. lds each, whole cache lines.  The
// buffer descriptor ends at the operand's last row of the tile, so rows past a ragged end
// read as zero; chunks past the end of k or of the columns get an offset outside it.  Zeros
// in both operands add nothing, whatever bits (NaN, infinities) lie behind the end.
// bf16 operands with k down are read back through the transposing LDS read
// (ds_read_b64_tr_b16), so no transposed copy is ever made.
//
// The products go to the matrix cores as mfma(B, A): a lane then holds consecutive columns
// of one row, and with the columns of two 16-column blocks interleaved in fours (bf16) it
// stores 16 bytes at a time.  Sums are fp32, rounded once.
#pragma once

#include <algorithm>
#include <type_traits>

#include "lds_dma.h"
#include "ragged.h"

namespace ace {

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

// the same with the non-temporal hint, for data that is read once
__device__ __forceinline__ void dma16_buf_stream(i32x4_rsrc rsrc, uint32_t off, uint32_t lds) {
  asm volatile(
      "s_mov_b32 m0, %2\n\t"
      "s_nop 0\n\t"
      "buffer_load_dwordx4 %0, %1, 0 offen nt lds"
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

// Row (column) of an operand in position q of its 16-row block blk.  PAIR (bf16 columns of C):
// the columns of a 32-column pair of blocks interleaved in fours: position q of block b holds
// column 8 (q / 4) + 4 b + q % 4.
template <bool PAIR> __host__ __device__ constexpr int block_row(int blk, int q) {
  return PAIR ? 32 * (blk >> 1) + 8 * (q >> 2) + 4 * (blk & 1) + (q & 3) : 16 * blk + q;
}

// Where an operand lies; two matrices: their blocks alternate (see gated.hip)
template <int MATS> struct Mats {
  const void *p[MATS];
};

// One operand of a tile: BLK 16-row blocks of C's rows (or columns).
//   DOWN = false: p points at the tile's first row; `valid` rows of ld elements, k along them
//   DOWN = true:  p points at the tile's first column of k's first row; `valid` columns
// MATS = 2 (not DOWN): block b is block b / 2 of matrix b % 2.
template <typename T, bool DOWN, int BLK, bool PAIR, int W, int MATS = 1> struct Operand {
  using Src = Mats<MATS>;
  static constexpr int ES = sizeof(T), E = kChunkElems<T>, BK = kStageElems<T>;
  static constexpr int UNITS = 2 * BLK;              // per stage
  static constexpr int NU = (UNITS + W - 1) / W;     // per wave
  static constexpr int COPIES = NU;                  // copies of a wave per stage
  static constexpr int PANEL = 0, PANEL_STAGES = 1;  // nothing that comes for several stages at once (see mx4_tile.h)
  static constexpr int OU = DOWN ? BLK * 16 / BK : 1;  // k down: units across
  static constexpr int BYTES = UNITS * kUnitBytes;
  static_assert(UNITS % W == 0, "units spread evenly over the waves");
  static_assert(!DOWN || (BLK * 16) % BK == 0, "whole units across");
  static_assert(MATS == 1 || (!DOWN && (NU <= 2 || NU % 4 == 0)), "two matrices: k-major, a wave's units see issue");
  typedef typename Frag<T>::type frag_t;

  const uint8_t *base[MATS];
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

  __device__ __forceinline__ void init(const Src &src, int ld, int valid, int k, int wave, int lane) {
#pragma unroll
    for (int m = 0; m < MATS; ++m) base[m] = static_cast<const uint8_t *>(src.p[m]);
    // an offset, not a choice between the two: that would be an index into the array at run time and put it in memory
    if (MATS == 2 && NU <= 2) base[0] += (base[MATS - 1] - base[0]) * ((wave * NU / 2) % 2);
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
        const int row = block_row<PAIR>((u >> 1) / MATS, 8 * (u & 1) + ur);
        voff[t] = static_cast<uint32_t>(row) * row_bytes + static_cast<uint32_t>(chunk_k) * ES;
      } else {
        const int ku = u / OU, ou = u % OU;
        const uint32_t col = static_cast<uint32_t>(ou * BK + E * (slot ^ swz(ur, ku))) * ES;
        voff[t] = col < span ? static_cast<uint32_t>(8 * ku + ur) * row_bytes + col : kOutside;
      }
    }
  }

  // the copies of stage s into LDS at `lds`; once: no other tile reads this data
  __device__ __forceinline__ void issue(int s, uint32_t lds, uint32_t, int wave, bool once) const {
    bool in = true;
    const int left = klen - s * BK;  // k from this stage on
    auto rsrc_of = [&](const uint8_t *b) {
      return DOWN ? make_rsrc(b + static_cast<size_t>(s) * BK * row_bytes,
                              static_cast<uint32_t>(min(left, BK) - 1) * row_bytes + span)
                  : make_rsrc(b + static_cast<size_t>(s) * BK * ES, span - static_cast<uint32_t>(s * BK * ES));
    };
    if (!DOWN) in = chunk_k < left;
    // units come two a block, so a wave's belong to one matrix (see init), or alternate in twos
    const i32x4_rsrc first = rsrc_of(base[0]);
    const i32x4_rsrc second = MATS == 2 && NU > 2 ? rsrc_of(base[MATS - 1]) : first;
    auto of = [&](int t) { return (t >> 1) % 2 ? second : first; };
    if (once) {
#pragma unroll
      for (int t = 0; t < NU; ++t) dma16_buf_stream(of(t), in ? voff[t] : kOutside, lds + (wave * NU + t) * kUnitBytes);
    } else {
#pragma unroll
      for (int t = 0; t < NU; ++t) dma16_buf(of(t), in ? voff[t] : kOutside, lds + (wave * NU + t) * kUnitBytes);
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

// waits for this wave's LDS reads and all but n of its copies, then for the workgroup (ALONE: the rings are the wave's own)
template <int N, bool ALONE> __device__ __forceinline__ void stage_barrier() {
  if constexpr (ALONE)
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N) : "memory");
  else
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

// One tile of C in a workgroup's list: rows and columns of the output, and the group
struct Item {
  int group;       // -1: rows of no group, whose result is zero
  int row0, rows;  // rows of x / dy: the tile's rows, or (weights' gradient) the group's
  int tile;        // column tile, or (weights' gradient) tile of the group's matrix
  int once;        // no other row tile of the group
  int split;       // part of the reduction (weights' gradient: slot of the partial sums, -1: none)
};
constexpr int kFlush = 4;   // stages of an fp32 partial sum
constexpr int kItems = 64;  // of one list, one in each lane: longer work is done in several

// Operands, sizes and place of a tile
template <typename T, class SA = Mats<1>, class SB = Mats<1>> struct TileRef {
  SA a;
  SB b;
  T *out;
  float *part;     // where the fp32 sums of a part of the reduction go instead, or null
  int rows, cols;  // rows of a, and of b as the operand has them
  int klen;        // 0: the result is zero
  int rot;         // stage that comes first
  bool once;       // b is read by no other tile
};

// Stage that a tile of nk stages starts with: groups start at different ones, and whole panels apart
template <class Op> __device__ __forceinline__ int first_stage(int rot, int nk) {
  constexpr int P = Op::PANEL_STAGES;
  return nk > 0 ? rot % ((nk + P - 1) / P) * P : 0;
}

// The copying side of one operand: the stages of the list's tiles in order (of the segments of their
// reductions, `n` in all), through a ring of D LDS slots.  A panel, what an operand has for PANEL_STAGES stages at
// once, is copied ahead of the first of them, through a ring of its own with as many slots: no more than D
// panels are in use or under way, since each belongs to one of D stages at least.
template <class Op, int D, bool IS_A> struct Feed {
  Op op;
  int pi = -1, ps = 0, pnk = 0, prot = 0, slot = 0, pslot = 0;
  bool once = false;

  // on to the next tile that has stages, if the present one has none left
  template <typename F> __device__ __forceinline__ void advance(int n, int ld, int wave, int lane, F ref) {
    while (pi < n && ps == pnk) {
      if (++pi == n) return;
      const auto t = ref(pi);
      if constexpr (IS_A)
        op.init(t.a, ld, t.rows, t.klen, wave, lane);
      else
        op.init(t.b, ld, t.cols, t.klen, wave, lane);
      pnk = (t.klen + Op::BK - 1) / Op::BK;
      ps = 0;
      prot = first_stage<Op>(t.rot, pnk);
      once = !IS_A && t.once;
    }
  }
  // the next stage's copies, and those of its panel where it is the first that needs it
  __device__ __forceinline__ void issue(uint32_t lds, int wave) {
    const int s = ps + prot < pnk ? ps + prot : ps + prot - pnk;
    uint32_t panel = 0;
    if constexpr (Op::PANEL > 0)
      if (s % Op::PANEL_STAGES == 0) {
        panel = lds + D * Op::BYTES + pslot * Op::PANEL;
        pslot = pslot + 1 == D ? 0 : pslot + 1;
      }
    op.issue(s, lds + slot * Op::BYTES, panel, wave, once);
    slot = slot + 1 == D ? 0 : slot + 1;
    ++ps;
  }
};

// 16 bytes of a result.  Nothing here reads it again, so where rows are whole 128-byte lines it goes with the
// non-temporal hint and takes no cache from the operands (the weights' gradient of 128 groups of 768 x 2048
// and 128 rows: 136 -> 114 us).  Where a line is shared by two rows, the caches have to put it together
// (34 groups of 3712 x 1288 with 58 rows: 190 us with the hint).
template <bool LINES> __device__ __forceinline__ void put16(void *p, uint4 v) {
  typedef unsigned u32x4_t __attribute__((ext_vector_type(4)));
  if constexpr (LINES)
    __builtin_nontemporal_store(__builtin_bit_cast(u32x4_t, v), reinterpret_cast<u32x4_t *>(p));
  else
    *reinterpret_cast<uint4 *>(p) = v;
}

// lane r of 16 <-> lane r ^ 8
__device__ __forceinline__ uint32_t swap8(uint32_t v) {
  return static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(static_cast<int>(v), 0x128, 0xf, 0xf, true));  // row_ror:8
}

// A wave's share of a tile: row blocks wr + WR i, columns c0 .. c0 + 16 NW - 1.  A lane holds row
// lane % 16 of each block.  bf16: 8 consecutive columns from each pair of column blocks, so two pairs are
// 128 bytes of a row over 4 lanes each; lanes r and r + 8 exchange one of them, and a store writes whole
// lines of 8 rows in place of half lines of 16.
template <typename T, bool LINES, int MW, int NW, int WR>
__device__ __forceinline__ void store_rows(T *out, int rows, int cols, size_t ldo, const f32x4_t (&acc)[MW][NW],
                                           int wr, int c0, int lane) {
  const int r16 = lane & 15, g = lane >> 4;
  if constexpr (sizeof(T) == 2) {
    const bool lower = r16 < 8;
    const int col = c0 + 8 * g + (lower ? 0 : 32);
#pragma unroll
    for (int i = 0; i < MW; ++i) {
      const int row = 16 * (wr + WR * i) + (r16 & 7);
      if (16 * (wr + WR * i) >= rows) break;  // wave-uniform
      T *o = out + static_cast<size_t>(row) * ldo + col;
#pragma unroll
      for (int j = 0; j < NW; j += 4) {
        uint32_t p[2][4];
#pragma unroll
        for (int q = 0; q < 2 && j + 2 * q < NW; ++q) {
          const f32x4_t lo = acc[i][j + 2 * q], hi = acc[i][j + 2 * q + 1];
          p[q][0] = pack_bf16x2(lo[0], lo[1]);
          p[q][1] = pack_bf16x2(lo[2], lo[3]);
          p[q][2] = pack_bf16x2(hi[0], hi[1]);
          p[q][3] = pack_bf16x2(hi[2], hi[3]);
        }
        if (j + 2 < NW) {
          uint32_t first[4], second[4];  // rows r16 % 8 and r16 % 8 + 8
#pragma unroll
          for (int d = 0; d < 4; ++d) {
            const uint32_t got = swap8(lower ? p[1][d] : p[0][d]);
            first[d] = lower ? p[0][d] : got;
            second[d] = lower ? got : p[1][d];
          }
          if (col + 16 * j >= cols) continue;
          if (row < rows) put16<LINES>(o + 16 * j, uint4{first[0], first[1], first[2], first[3]});
          if (row + 8 < rows) put16<LINES>(o + 16 * j + 8 * ldo, uint4{second[0], second[1], second[2], second[3]});
        } else {  // a pair left over: half lines
          const int own = 16 * (wr + WR * i) + r16, at = c0 + 8 * g + 16 * j;
          if (own < rows && at < cols)
            put16<LINES>(out + static_cast<size_t>(own) * ldo + at, uint4{p[0][0], p[0][1], p[0][2], p[0][3]});
        }
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < MW; ++i) {
      const int row = 16 * (wr + WR * i) + r16;
      if (row >= rows) continue;
      T *o = out + static_cast<size_t>(row) * ldo;
#pragma unroll
      for (int j = 0; j < NW; ++j) {
        const int col = c0 + 16 * j + 4 * g;
        if (col < cols) put16<LINES>(o + col, __builtin_bit_cast(uint4, acc[i][j]));
      }
    }
  }
}

// The same sums as fp32: a part of the reduction, which grouped_join_kernel adds up
template <typename T, int MW, int NW, int WR>
__device__ __forceinline__ void store_part(float *part, int rows, int cols, size_t ldo, const f32x4_t (&acc)[MW][NW],
                                           int wr, int c0, int lane) {
  const int r16 = lane & 15, g = lane >> 4;
#pragma unroll
  for (int i = 0; i < MW; ++i) {
    const int row = 16 * (wr + WR * i) + r16;
    if (row >= rows) continue;
    float *o = part + static_cast<size_t>(row) * ldo;
#pragma unroll
    for (int j = 0; j < NW; ++j) {
      const int col = c0 + (sizeof(T) == 2 ? 16 * (j & ~1) + 8 * g + 4 * (j & 1) : 16 * j + 4 * g);
      if (col < cols) *reinterpret_cast<f32x4_t *>(o + col) = acc[i][j];
    }
  }
}

// A tile's shape, rings and products: MB x NB 16-blocks, WR x WC waves, rings of DA and DB slots.  SEG: segments of
// a reduction, each with operands of its own.
template <typename T_, bool ADOWN, bool BDOWN, int MB_, int NB_, int WR_, int WC_, int DA_, int DB_, int MATS = 1,
          int SEG_ = 1>
struct DenseTile {
  using T = T_;
  static constexpr int MB = MB_, NB = NB_, WR = WR_, WC = WC_, DA = DA_, DB = DB_, SEG = SEG_;
  static constexpr int MW = MB / WR, NW = NB / WC, LDS = (DA * MB + DB * NB) * 2 * kUnitBytes;
  using A = Operand<T, ADOWN, MB, false, WR * WC>;
  using B = Operand<T, BDOWN, NB, sizeof(T) == 2, WR * WC, MATS>;
  using Ref = TileRef<T, typename A::Src, typename B::Src>;

  // adds a stage's products, and calls mid halfway; blocks past the tile's rows are read too and not multiplied
  template <typename M>
  static __device__ __forceinline__ void multiply(const uint8_t *pa, const uint8_t *pb, const uint8_t *, const uint8_t *,
                                                  int wr, int wc, int lane, int rows, int, int, f32x4_t (&acc)[MW][NW],
                                                  M mid) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if (h == 1) {
        mid();
        // fp32: keeps the halves apart; as one block the compiler moves the sums from and to the accumulation registers with
        // every stage (products of 2069 rows in 32 groups of 512 x 1024: 50.8 us, 45.9 so)
        if (sizeof(T) == 4) asm volatile("" ::: "memory");
      }
      typename B::frag_t bf[NW];
      typename A::frag_t af[MW];
#pragma unroll
      for (int j = 0; j < NW; ++j) bf[j] = B::read(pb, wc * NW + j, h, lane);
#pragma unroll
      for (int i = 0; i < MW; ++i) af[i] = A::read(pa, wr + WR * i, h, lane);
#pragma unroll
      for (int i = 0; i < MW; ++i)
        if (16 * (wr + WR * i) < rows) {  // wave-uniform
#pragma unroll
          for (int s = 0; s < Frag<T>::steps; ++s)
#pragma unroll
            for (int j = 0; j < NW; ++j) acc[i][j] = Frag<T>::mma(bf[j], af[i], s, acc[i][j]);
        }
    }
  }
};

// The tiles of a workgroup's list (item j in lane j of every wave, n of them) as one pipeline:
// stages of a tile's operands are copied DA - 1 and DB - 1 ahead of their use through rings of DA
// and DB LDS slots, and across the end of a tile, so the next tile's first stages are under way
// while a tile ends and stores.  Where PENDING is 0 (both rings two deep: the weights' gradient in 256 x 256 tiles) the
// next tile's first products wait for those stores.  A shape of one wave is a pipeline of its own for each wave, which
// waits for no other; smem is then that wave's.  ref(item, segment) gives a tile's operands; lda, ldb are common;
// store(ref, sums, wr, wc, lane) puts a wave's share of the sums where they belong.
template <class S, typename F, typename E>
__device__ __forceinline__ void grouped_items(const Item &list, int n, int lda, int ldb, uint8_t *smem, F ref, E store) {
  using T = typename S::T;
  using A = typename S::A;
  using B = typename S::B;
  constexpr int MB = S::MB, NB = S::NB, WR = S::WR, WC = S::WC, DA = S::DA, DB = S::DB, SEG = S::SEG;
  constexpr int MW = MB / WR, NW = NB / WC;
  constexpr bool PAIR = sizeof(T) == 2;
  constexpr int BK = A::BK;
  // copies that may be outstanding when stage c is needed: those after the copies of A(c), that
  // is of iterations c - DA + 1 (its B only, which lies ahead of B(c)) to c - 1.  Panels are not counted: those
  // among them only make the wait longer
  constexpr int PENDING = (DB > DA ? B::COPIES : 0) + (DA - 2) * (A::COPIES + B::COPIES);
  static_assert(A::BK == B::BK, "stages of the same k");
  static_assert(MB % WR == 0 && NB % WC == 0 && (!PAIR || NW % 2 == 0), "whole blocks, in bf16 pairs of column blocks, per wave");
  static_assert(DA >= 2 && DB >= DA && PENDING <= 63, "ring depths, outstanding copies within the wait counter");
  const int lane = threadIdx.x & 63;
  constexpr bool ALONE = WR * WC == 1;
  const int wave = ALONE ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wr = wave / WC, wc = wave % WC;
  constexpr int RING_A = DA * (A::BYTES + A::PANEL);
  const uint32_t ldsa = lds_addr(smem), ldsb = ldsa + RING_A;
  auto at = [&](int i) {
    const int seg = i % SEG;
    i /= SEG;
    return ref(Item{__builtin_amdgcn_readlane(list.group, i), __builtin_amdgcn_readlane(list.row0, i),
                    __builtin_amdgcn_readlane(list.rows, i), __builtin_amdgcn_readlane(list.tile, i), __builtin_amdgcn_readlane(list.once, i), __builtin_amdgcn_readlane(list.split, i)}, seg);
  };
  Feed<A, DA, true> fa;
  Feed<B, DB, false> fb;
  auto issue_a = [&]() {
    fa.issue(ldsa, wave);
    fa.advance(SEG * n, lda, wave, lane, at);
  };
  auto issue_b = [&]() {
    fb.issue(ldsb, wave);
    fb.advance(SEG * n, ldb, wave, lane, at);
  };
  fa.advance(SEG * n, lda, wave, lane, at);
  fb.advance(SEG * n, ldb, wave, lane, at);
#pragma unroll
  for (int s = 0; s < DB - 1; ++s)
    if (fb.pi < SEG * n) issue_b();
#pragma unroll
  for (int s = 0; s < DA - 1; ++s)
    if (fa.pi < SEG * n) issue_a();
  int sa = 0, sb = 0;                                               // slots of the stage multiplied next
  [[maybe_unused]] int qa = DA - 1, qb = DB - 1;                    // and of its panels
  int warm = DA - 1;   // the first stages wait for everything
  auto copies = [&]() {
    if (fa.pi < SEG * n) issue_a();
    if (fb.pi < SEG * n) {
      issue_b();
      warm = max(warm - 1, 0);
    } else {
      warm = 1;
    }
  };
  // of the two waves of a SIMD one copies before its products and one between them
  const bool late = S::WR * S::WC == 8 && wave >= 4;
  for (int ci = 0; ci < n; ++ci) {
    f32x4_t acc[MW][NW];
    auto clear = [](f32x4_t (&c)[MW][NW]) {
#pragma unroll
      for (int i = 0; i < MW; ++i)
#pragma unroll
        for (int j = 0; j < NW; ++j) c[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    };
    clear(acc);
    // fp32 results: the products of kFlush stages are summed apart and then added to the rest, so the
    // rounding of a long sum grows with the root of its parts, not of its terms (1.1e-6 of the result
    // without it for 1024 terms, 4e-7 with it)
    [[maybe_unused]] f32x4_t total[sizeof(T) == 4 ? MW : 1][NW];
    auto flush = [&]() {
      if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < MW; ++i)
#pragma unroll
          for (int j = 0; j < NW; ++j) total[i][j] += acc[i][j];
        clear(acc);
      }
    };
    if constexpr (sizeof(T) == 4) clear(total);
    for (int seg = 0; seg < SEG; ++seg) {
      const auto t = at(ci * SEG + seg);
      const int nk = (t.klen + BK - 1) / BK, rot = first_stage<B>(t.rot, nk);
      for (int kt = 0; kt < nk; ++kt) {
        // this stage landed for every wave, and every wave is done with the slots refilled next;
        // while B still had a stage to copy one iteration ago, the count is the constant one
        if (PENDING > 0 && warm == 0)
          stage_barrier<PENDING, ALONE>();
        else
          stage_barrier<0, ALONE>();
        if (!late) copies();
        const int ks = kt + rot < nk ? kt + rot : kt + rot - nk;
        if (A::PANEL > 0 && ks % A::PANEL_STAGES == 0) qa = qa + 1 == DA ? 0 : qa + 1;
        if (B::PANEL > 0 && ks % B::PANEL_STAGES == 0) qb = qb + 1 == DB ? 0 : qb + 1;
        S::multiply(smem + sa * A::BYTES, smem + RING_A + sb * B::BYTES, smem + DA * A::BYTES + qa * A::PANEL,
                    smem + RING_A + DB * B::BYTES + qb * B::PANEL, wr, wc, lane, t.rows, ks * BK, t.klen, acc, [&]() {
                      if (late) copies();
                    });
        if (sizeof(T) == 4 && (kt + 1) % kFlush == 0) flush();
        sa = sa + 1 == DA ? 0 : sa + 1;
        sb = sb + 1 == DB ? 0 : sb + 1;
      }
      flush();
    }
    const f32x4_t(&sum)[MW][NW] = [&]() -> const f32x4_t(&)[MW][NW] {
      if constexpr (sizeof(T) == 4)
        return total;
      else
        return acc;
    }();
    store(at(ci * SEG), sum, wr, wc, lane);
  }
}

// A wave's share of a tile as it is, rows of ldo elements: rounded to T, or the fp32 sums of a part
template <typename T, bool LINES, class S> struct StoreTile {
  size_t ldo;
  __device__ __forceinline__ void operator()(const typename S::Ref &t, const f32x4_t (&sum)[S::MW][S::NW], int wr, int wc,
                                             int lane) const {
    if (t.part)
      store_part<T, S::MW, S::NW, S::WR>(t.part, t.rows, t.cols, ldo, sum, wr, 16 * wc * S::NW, lane);
    else
      store_rows<T, LINES, S::MW, S::NW, S::WR>(t.out, t.rows, t.cols, ldo, sum, wr, 16 * wc * S::NW, lane);
  }
};

// The reduction of a tile of 16 rows split over the KS waves of a workgroup, each with a pipeline of its own (shapes of
// one wave): their sums meet in LDS, the first wave adds them up in order and stores.  Two places in turn, so that one wait
// per tile is enough: the first wave has read a place before it comes to the wait behind which it is written again.
template <class S, int KS, class E> struct JoinStore {
  static constexpr int PLACE = (KS - 1) * 64 * 16 * S::NW, LDS = 2 * PLACE;
  static_assert(S::MW == 1 && S::WR * S::WC == 1 && sizeof(typename S::T) == 2, "tiles of one wave, 16 rows");
  E store;
  uint8_t *smem;
  int turn;
  template <class R>
  __device__ __forceinline__ void operator()(const R &t, const f32x4_t (&sum)[1][S::NW], int wr, int wc, int lane) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    f32x4_t *place = reinterpret_cast<f32x4_t *>(smem + turn * PLACE) + lane;
    turn ^= 1;
    if (wave > 0) {
#pragma unroll
      for (int j = 0; j < S::NW; ++j) place[((wave - 1) * S::NW + j) * 64] = sum[0][j];
    }
    // LDS writes done; the copies under way need no wait
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    if (wave > 0) return;
    f32x4_t all[1][S::NW];
#pragma unroll
    for (int j = 0; j < S::NW; ++j) {
      all[0][j] = sum[0][j];
#pragma unroll
      for (int w = 0; w < KS - 1; ++w) {
        const f32x4_t v = place[(w * S::NW + j) * 64];
#pragma unroll
        for (int q = 0; q < 4; ++q) all[0][j][q] += v[q];
      }
    }
    store(t, all, wr, wc, lane);
  }
};

// Block b runs on XCD b % 8.  Each XCD takes a run of consecutive items, all columns of a row tile (or all
// tiles of a group's dw) before the next, its workgroups side by side: the rows that
// column tiles share and the weights that the row tiles of a group share are read into one L2
// at about the same time.  Workgroup `slot` of an XCD takes the items slot, slot + slots, .. of its run.
struct Share {
  long long first, mine;
  int slot, slots;
  __device__ __forceinline__ explicit Share(long long all)
      : slot(blockIdx.x >> 3), slots(static_cast<int>(gridDim.x) >> 3) {
    const long long run = (all + 7) >> 3;
    first = (blockIdx.x & 7) * run;
    mine = min(run, max(all - first, 0ll));
  }
  // this workgroup's items from its `done`-th on: how many a list takes of them, and this lane's
  __device__ __forceinline__ int count(long long done) const {
    const long long left = mine - slot - done * slots;
    return left <= 0 ? 0 : static_cast<int>(min((left + slots - 1) / slots, static_cast<long long>(kItems)));
  }
  __device__ __forceinline__ long long item(long long done) const {
    return first + min(slot + (done + (threadIdx.x & 63)) * slots, max(mine - 1, 0ll));
  }
};

// part `s` of `splits` of a reduction of klen: whole stages, as even as they come
struct Part {
  int k0, len;
};
template <int BK> __host__ __device__ __forceinline__ Part part_of(int klen, int s, int splits) {
  if (splits == 1) return {0, klen};
  const int nk = (klen + BK - 1) / BK, each = nk / splits, more = nk % splits;
  const int b = s * each + min(s, more), n = each + (s < more);
  return {b * BK, max(min(n * BK, klen - b * BK), 0)};
}

constexpr int kCUs = 256;
constexpr int kMaxSplits = 64;

// A kernel's tile and rings; PER_CU workgroups of it share a CU's LDS
template <int MB_, int NB_, int WR_, int WC_, int DA_, int DB_> struct TileShape {
  static constexpr int MB = MB_, NB = NB_, WR = WR_, WC = WC_, DA = DA_, DB = DB_;
  static constexpr int TM = 16 * MB, TN = 16 * NB, THREADS = WR * WC * 64;
  static constexpr int PER_CU = 160 * 1024 / ((DA * MB + DB * NB) * 2 * kUnitBytes);
};
inline long long tiles_of(long long n, int t) { return (n + t - 1) / t; }

// Tiles that S rows in N groups make, about: half a tile more than full ones for a group, at least one
inline long long about_tiles(long long S, long long N, int tm) {
  return std::max(S / tm + std::min(N, S) / 2, std::min(N, S));
}

// Parts of the reduction: few tiles with a long reduction leave CUs idle.  Each part is at least one
// workgroup more; what it saves are its stages' times, what it costs the launch that adds the parts
// and their traffic (us, as measured: 2 groups of 1024 x 2048 with 4 rows 33 us whole and 12 in 8 parts,
// 16 groups of 1024 x 1024 with one row 12.8 whole and 13.4 in two).
inline int pick_splits(long long items, int slots, long long nk, size_t elems, double stage_us) {
  int best = 1;
  double least = static_cast<double>(nk) * stage_us;
  for (int s = 2; s <= kMaxSplits && items * s <= slots && s <= nk; s *= 2) {
    const double t = static_cast<double>((nk + s - 1) / s) * stage_us + 4.5 + 2e-6 * s * static_cast<double>(elems);
    if (t < least) {
      least = t;
      best = s;
    }
  }
  return best;
}

// Workgroups of a launch: whole rounds of the XCDs, per_cu of them on every CU
inline unsigned grouped_grid(long long items, int per_cu) {
  return static_cast<unsigned>(std::min<long long>((items + 7) / 8 * 8, kCUs * per_cu));
}

}  // namespace ace
