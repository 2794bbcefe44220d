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
#include <algorithm>
#include <type_traits>

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

  // the copies of stage s into LDS at `lds`; once: no other tile reads this data
  __device__ __forceinline__ void issue(int s, uint32_t lds, int wave, bool once) const {
    i32x4_rsrc rsrc;
    bool in = true;
    const int left = klen - s * BK;  // k from this stage on
    if (!DOWN) {
      rsrc = make_rsrc(base + static_cast<size_t>(s) * BK * ES, span - static_cast<uint32_t>(s * BK * ES));
      in = chunk_k < left;
    } else {
      rsrc = make_rsrc(base + static_cast<size_t>(s) * BK * row_bytes,
                       static_cast<uint32_t>(min(left, BK) - 1) * row_bytes + span);
    }
    if (once) {
#pragma unroll
      for (int t = 0; t < NU; ++t) dma16_buf_stream(rsrc, in ? voff[t] : kOutside, lds + (wave * NU + t) * kUnitBytes);
    } else {
#pragma unroll
      for (int t = 0; t < NU; ++t) dma16_buf(rsrc, in ? voff[t] : kOutside, lds + (wave * NU + t) * kUnitBytes);
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

// One tile of C in a workgroup's list: rows and columns of the output, and the group
struct Item {
  int group;       // -1: rows of no group, whose result is zero
  int row0, rows;  // rows of x / dy: the tile's rows, or (weights' gradient) the group's
  int tile;        // column tile, or (weights' gradient) tile of the group's matrix
  int once;        // no other row tile of the group
  int split;       // part of the reduction (weights' gradient: slot of the partial sums, -1: none)
};
constexpr int kFlush = 4;  // stages of an fp32 partial sum
constexpr int kItems = 64;  // of one list, one in each lane: longer work is done in several

// Operands, sizes and place of a tile
template <typename T> struct TileRef {
  const T *a, *b;
  T *out;
  float *part;     // where the fp32 sums of a part of the reduction go instead, or null
  int rows, cols;  // stored
  int klen;        // 0: the result is zero
  int rot;         // stage that comes first
  bool once;       // b is read by no other tile
};

// The copying side of one operand: the stages of the list's tiles in order, through a ring of
// D LDS slots
template <class Op, int D, bool IS_A> struct Feed {
  Op op;
  int pi = -1, ps = 0, pnk = 0, prot = 0, slot = 0;
  bool once = false;

  // on to the next tile that has stages, if the present one has none left
  template <typename F> __device__ __forceinline__ void advance(int n, int ld, int wave, int lane, F ref) {
    while (pi < n && ps == pnk) {
      if (++pi == n) return;
      const auto t = ref(pi);
      op.init(IS_A ? t.a : t.b, ld, IS_A ? t.rows : t.cols, t.klen, wave, lane);
      pnk = (t.klen + Op::BK - 1) / Op::BK;
      ps = 0;
      prot = pnk > 0 ? t.rot % pnk : 0;
      once = !IS_A && t.once;
    }
  }
  // the next stage's copies
  __device__ __forceinline__ void issue(uint32_t lds, int wave) {
    op.issue(ps + prot < pnk ? ps + prot : ps + prot - pnk, lds + slot * Op::BYTES, wave, once);
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
__device__ __forceinline__ void store_rows(const TileRef<T> &t, size_t ldo, const f32x4_t (&acc)[MW][NW], int wr,
                                           int c0, int lane) {
  const int r16 = lane & 15, g = lane >> 4;
  if constexpr (sizeof(T) == 2) {
    const bool lower = r16 < 8;
    const int col = c0 + 8 * g + (lower ? 0 : 32);
#pragma unroll
    for (int i = 0; i < MW; ++i) {
      const int row = 16 * (wr + WR * i) + (r16 & 7);
      if (16 * (wr + WR * i) >= t.rows) break;  // wave-uniform
      T *o = t.out + static_cast<size_t>(row) * ldo + col;
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
          if (col + 16 * j >= t.cols) continue;
          if (row < t.rows) put16<LINES>(o + 16 * j, uint4{first[0], first[1], first[2], first[3]});
          if (row + 8 < t.rows) put16<LINES>(o + 16 * j + 8 * ldo, uint4{second[0], second[1], second[2], second[3]});
        } else {  // a pair left over: half lines
          const int own = 16 * (wr + WR * i) + r16, at = c0 + 8 * g + 16 * j;
          if (own < t.rows && at < t.cols)
            put16<LINES>(t.out + static_cast<size_t>(own) * ldo + at, uint4{p[0][0], p[0][1], p[0][2], p[0][3]});
        }
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < MW; ++i) {
      const int row = 16 * (wr + WR * i) + r16;
      if (row >= t.rows) continue;
      T *o = t.out + static_cast<size_t>(row) * ldo;
#pragma unroll
      for (int j = 0; j < NW; ++j) {
        const int col = c0 + 16 * j + 4 * g;
        if (col < t.cols) put16<LINES>(o + col, __builtin_bit_cast(uint4, acc[i][j]));
      }
    }
  }
}

// The same sums as fp32: a part of the reduction, which grouped_join_kernel adds up
template <typename T, int MW, int NW, int WR>
__device__ __forceinline__ void store_part(const TileRef<T> &t, size_t ldo, const f32x4_t (&acc)[MW][NW], int wr,
                                           int c0, int lane) {
  const int r16 = lane & 15, g = lane >> 4;
#pragma unroll
  for (int i = 0; i < MW; ++i) {
    const int row = 16 * (wr + WR * i) + r16;
    if (row >= t.rows) continue;
    float *o = t.part + static_cast<size_t>(row) * ldo;
#pragma unroll
    for (int j = 0; j < NW; ++j) {
      const int col = c0 + (sizeof(T) == 2 ? 16 * (j & ~1) + 8 * g + 4 * (j & 1) : 16 * j + 4 * g);
      if (col < t.cols) *reinterpret_cast<f32x4_t *>(o + col) = acc[i][j];
    }
  }
}

// The tiles of a workgroup's list (item j in lane j of every wave, n of them) as one pipeline:
// stages of a tile's operands are copied DA - 1 and DB - 1 ahead of their use through rings of DA
// and DB LDS slots, and across the end of a tile, so the next tile's first stages are under way
// while a tile ends and stores.  Where PENDING is 0 (both rings two deep: the weights' gradient in 256 x 256 tiles) the
// next tile's first products wait for those stores.  A tile is MB x NB 16-blocks, WR x WC waves.  ref(item) gives a
// tile's operands; lda, ldb, ldo are common.
template <typename T, bool ADOWN, bool BDOWN, bool LINES, int MB, int NB, int WR, int WC, int DA, int DB, typename F>
__device__ __forceinline__ void grouped_items(const Item &list, int n, int lda, int ldb, size_t ldo, uint8_t *smem,
                                              F ref) {
  constexpr int W = WR * WC, MW = MB / WR, NW = NB / WC;
  constexpr bool PAIR = sizeof(T) == 2;
  using A = Operand<T, ADOWN, MB, false, W>;
  using B = Operand<T, BDOWN, NB, PAIR, W>;
  constexpr int BK = A::BK;
  // copies that may be outstanding when stage c is needed: those after the copies of A(c), that
  // is of iterations c - DA + 1 (its B only, which lies ahead of B(c)) to c - 1
  constexpr int PENDING = (DB > DA ? B::NU : 0) + (DA - 2) * (A::NU + B::NU);
  static_assert(MB % WR == 0 && NB % WC == 0 && (!PAIR || NW % 2 == 0), "whole blocks, in bf16 pairs of column blocks, per wave");
  static_assert(DA >= 2 && DB >= DA && PENDING <= 63, "ring depths, outstanding copies within the wait counter");
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wr = wave / WC, wc = wave % WC;
  const uint32_t ldsa = lds_addr(smem), ldsb = ldsa + DA * A::BYTES;
  auto at = [&](int i) {
    return ref(Item{__builtin_amdgcn_readlane(list.group, i), __builtin_amdgcn_readlane(list.row0, i),
                    __builtin_amdgcn_readlane(list.rows, i), __builtin_amdgcn_readlane(list.tile, i), __builtin_amdgcn_readlane(list.once, i), __builtin_amdgcn_readlane(list.split, i)});
  };
  Feed<A, DA, true> fa;
  Feed<B, DB, false> fb;
  auto issue_a = [&]() {
    fa.issue(ldsa, wave);
    fa.advance(n, lda, wave, lane, at);
  };
  auto issue_b = [&]() {
    fb.issue(ldsb, wave);
    fb.advance(n, ldb, wave, lane, at);
  };
  fa.advance(n, lda, wave, lane, at);
  fb.advance(n, ldb, wave, lane, at);
#pragma unroll
  for (int s = 0; s < DB - 1; ++s)
    if (fb.pi < n) issue_b();
#pragma unroll
  for (int s = 0; s < DA - 1; ++s)
    if (fa.pi < n) issue_a();
  int sa = 0, sb = 0;  // slots of the stage multiplied next
  int warm = DA - 1;   // the first stages wait for everything
  for (int ci = 0; ci < n; ++ci) {
    const TileRef<T> t = at(ci);
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
    const int nk = (t.klen + BK - 1) / BK;
    for (int kt = 0; kt < nk; ++kt) {
      // this stage landed for every wave, and every wave is done with the slots refilled next;
      // while B still had a stage to copy one iteration ago, the count is the constant one
      if (PENDING > 0 && warm == 0)
        stage_barrier<PENDING>();
      else
        stage_barrier<0>();
      if (fa.pi < n) issue_a();
      if (fb.pi < n) {
        issue_b();
        warm = max(warm - 1, 0);
      } else {
        warm = 1;
      }
      const uint8_t *pa = smem + sa * A::BYTES, *pb = smem + DA * A::BYTES + sb * B::BYTES;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        typename B::frag_t bf[NW];
        typename A::frag_t af[MW];
#pragma unroll
        for (int j = 0; j < NW; ++j) bf[j] = B::read(pb, wc * NW + j, h, lane);
        // blocks past the tile's rows are read too and not multiplied
#pragma unroll
        for (int i = 0; i < MW; ++i) af[i] = A::read(pa, wr + WR * i, h, lane);
#pragma unroll
        for (int i = 0; i < MW; ++i)
          if (16 * (wr + WR * i) < t.rows) {  // wave-uniform
#pragma unroll
            for (int s = 0; s < Frag<T>::steps; ++s)
#pragma unroll
              for (int j = 0; j < NW; ++j) acc[i][j] = Frag<T>::mma(bf[j], af[i], s, acc[i][j]);
          }
      }
      if (sizeof(T) == 4 && (kt + 1) % kFlush == 0) flush();
      sa = sa + 1 == DA ? 0 : sa + 1;
      sb = sb + 1 == DB ? 0 : sb + 1;
    }
    flush();
    const f32x4_t(&sum)[MW][NW] = [&]() -> const f32x4_t(&)[MW][NW] {
      if constexpr (sizeof(T) == 4)
        return total;
      else
        return acc;
    }();
    if (t.part)
      store_part<T, MW, NW, WR>(t, ldo, sum, wr, 16 * wc * NW, lane);
    else
      store_rows<T, LINES, MW, NW, WR>(t, ldo, sum, wr, 16 * wc * NW, lane);
  }
}

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
template <typename T> __device__ __forceinline__ Part part_of(int klen, int s, int splits) {
  if (splits == 1) return {0, klen};
  constexpr int BK = kStageElems<T>;
  const int nk = (klen + BK - 1) / BK, each = nk / splits, more = nk % splits;
  const int b = s * each + min(s, more), n = each + (s < more);
  return {b * BK, max(min(n * BK, klen - b * BK), 0)};
}

// Tiles of x's or dy's rows by columns, the whole work of a workgroup
template <typename T, bool GX, bool LINES, int MB, int NB, int WR, int WC, int DA, int DB>
__device__ __forceinline__ void grouped_rows(const GroupedArgs &g, const RaggedTiles &tiles, uint8_t *smem) {
  constexpr int BN = 16 * NB;
  const int cols = GX ? g.K : g.M, klen = GX ? g.M : g.K;
  const int nN = (cols + BN - 1) / BN, per = nN * g.splits;
  const Share share(static_cast<long long>(tiles.total) * per);
  auto ref = [&](const Item &it) {
    const int c0 = it.tile * BN;
    const Part k = part_of<T>(it.group < 0 ? 0 : klen, it.split, g.splits);
    TileRef<T> t;
    t.a = static_cast<const T *>(g.rows) + static_cast<size_t>(it.row0) * klen + k.k0;
    const T *w = static_cast<const T *>(g.other) + static_cast<size_t>(max(it.group, 0)) * g.M * g.K;
    t.b = GX ? w + static_cast<size_t>(k.k0) * g.K + c0 : w + static_cast<size_t>(c0) * g.K + k.k0;
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
    grouped_items<T, false, GX, LINES, MB, NB, WR, WC, DA, DB>(
        Item{t.group, t.row0, t.rows, q % nN, t.only, q / nN}, n, klen, g.K, cols, smem, ref);
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
// Rounds of a CU times the time of a stage, in units of 50 ns as measured with every CU busy.  Four tile bodies
// in one kernel spill 49 vector registers in the rows' gradient and 6 in the forward.
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

// Weights' gradient: tile = 16 MB rows x 16 NB columns of one group's dw
template <typename T, bool LINES, int MB, int NB, int WR, int WC, int DA, int DB>
__global__ __launch_bounds__(WR *WC * 64) void grouped_weights_kernel(GroupedArgs g) {
  constexpr int BM = 16 * MB, BN = 16 * NB;
  __shared__ __align__(16) uint8_t smem[(DA * MB + DB * NB) * 2 * kUnitBytes];
  const int nM = (g.M + BM - 1) / BM, nN = (g.K + BN - 1) / BN, per = nM * nN;
  const RaggedTiles tiles(g.offsets, g.N, g.S, g.chunk, false, true);
  const Share share(static_cast<long long>(tiles.total) * per);
  auto ref = [&](const Item &it) {
    const int m0 = it.tile / nN * BM, c0 = it.tile % nN * BN;
    const size_t at = static_cast<size_t>(m0) * g.K + c0, size = static_cast<size_t>(g.M) * g.K;
    TileRef<T> t;
    t.a = static_cast<const T *>(g.rows) + static_cast<size_t>(it.row0) * g.M + m0;
    t.b = static_cast<const T *>(g.other) + static_cast<size_t>(it.row0) * g.K + c0;
    t.out = static_cast<T *>(g.out) + static_cast<size_t>(it.group) * size + at;
    t.part = it.split >= 0 ? g.part + static_cast<size_t>(it.split) * size + at : nullptr;
    t.rows = min(BM, g.M - m0);
    t.cols = min(BN, g.K - c0);
    t.klen = it.rows;
    t.rot = 0;
    t.once = false;
    return t;
  };
  long long done = 0;
  for (int n; (n = share.count(done)) > 0; done += n) {
    const long long i = share.item(done);
    const RaggedTile t = tiles.find(static_cast<int>(i / per));
    // offsets that do not ascend can make more parts than there is room for: those go to the last
    const int slot = t.only ? -1 : min(max(t.slot, 0), g.splits - 1);
    __syncthreads();  // every wave is done with the rings
    grouped_items<T, true, true, LINES, MB, NB, WR, WC, DA, DB>(
        Item{max(t.group, 0), t.row0, t.rows, static_cast<int>(i % per), 0, slot}, n, g.M, g.K, g.K, smem, ref);
  }
}

// dw of the groups of more than `chunk` rows: their parts' sum in order, 16 bytes of dw a thread.  Workgroups
// (x, y): the y-th such group, if there is one.
template <typename T> __global__ __launch_bounds__(256) void grouped_weights_join_kernel(GroupedArgs g) {
  constexpr int E = kChunkElems<T>;
  const int lane = threadIdx.x & 63;
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
      const float *p = g.part + static_cast<size_t>(min(max(slot + s, 0), g.splits - 1)) * size + i;
#pragma unroll
      for (int j = 0; j < E; j += 4) {
        const f32x4_t u = *reinterpret_cast<const f32x4_t *>(p + j);
#pragma unroll
        for (int k = 0; k < 4; ++k) v[j + k] += u[k];
      }
    }
    T *o = static_cast<T *>(g.out) + static_cast<size_t>(group) * size + i;
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

constexpr int kCUs = 256;
constexpr int kMaxSplits = 64;

// A kernel's tile and rings; PER_CU workgroups of it share a CU's LDS
template <int MB_, int NB_, int WR_, int WC_, int DA_, int DB_> struct Shape {
  static constexpr int MB = MB_, NB = NB_, WR = WR_, WC = WC_, DA = DA_, DB = DB_;
  static constexpr int TM = 16 * MB, TN = 16 * NB, THREADS = WR * WC * 64;
  static constexpr int PER_CU = 160 * 1024 / ((DA * MB + DB * NB) * 2 * kUnitBytes);
};
using Tile64 = Shape<4, 4, 2, 2, 4, 4>;     // bf16: few tiles, deep rings
using Tile64x128 = Shape<4, 8, 2, 2, 3, 3>;  // bf16: a few rows a group
using Tile128 = Shape<8, 8, 2, 2, 2, 3>;     // bf16
using Tile256 = Shape<16, 16, 4, 2, 2, 2>;   // bf16, weights' gradient
using TileF32 = Shape<2, 4, 2, 2, 3, 3>;     // fp32
using TileF32Weights = Shape<4, 4, 2, 2, 3, 3>;

enum class Kind { k64, k64x128, k128, kLarge, kF32 };

struct Plan {
  Kind kind;
  int splits;         // parts of the reduction (weights' gradient: room for so many parts of groups)
  size_t part_elems;  // of one part
  int chunk;          // weights' gradient: most rows of a part
};

long long tiles_of(long long n, int t) { return (n + t - 1) / t; }

// Tiles that S rows in N groups make, about: half a tile more than full ones for a group, at least one
long long about_tiles(long long S, long long N, int tm) {
  return std::max(S / tm + std::min(N, S) / 2, std::min(N, S));
}

// Parts of the reduction: few tiles with a long reduction leave CUs idle.  Each part is at least one
// workgroup more; what it saves are its stages' times, what it costs the launch that adds the parts
// and their traffic (us, as measured: 2 groups of 1024 x 2048 with 4 rows 33 us whole and 12 in 8 parts,
// 16 groups of 1024 x 1024 with one row 12.8 whole and 13.4 in two).
int pick_splits(long long items, int slots, long long nk, size_t elems, double stage_us) {
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

// Which kernel for the forward and the rows' gradient.  us on 128 groups of 768 x 2048 (forward):
//   rows a group               2    16    48    96   128   256  1024
//   128 x 128 (two a CU)      66    68    73    81   119   173   543
//   large (best of its four)  64    71    74    82    94   140   478
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

// ... and for the weights' gradient.  128 groups of 768 x 2048 and 128 rows: 256 x 256 tiles 114 us, 128 x 128 134
// (the former spill 27 registers and wait for each tile's stores).
// A group of more than p.chunk rows is summed in parts of at most that many, which a second launch adds: a few
// long groups would otherwise be a few workgroups' work.  Parts are four times the mean group (2048 rows at least),
// so that their sums take no more room than dw itself (bf16); or fewer rows where all tiles together
// would leave CUs idle, as far as the time of their stages pays for the launch and the traffic (us; 74 groups of
// 464 x 256, the largest a quarter of 39997 rows: 122 us whole, 54 in parts).
Plan plan_weights(const GroupedArgs &g, bool bf16) {
  const size_t elems = static_cast<size_t>(g.M) * g.K;
  const long long mean = (static_cast<long long>(g.S) + g.N - 1) / g.N;
  auto tiles = [&](int t) { return tiles_of(g.M, t) * tiles_of(g.K, t); };
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
      const double t = static_cast<double>(c) / 64 * stage + 4.5 + 2e-6 * (g.S / c) * static_cast<double>(elems);
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

// Workgroups of a launch: whole rounds of the XCDs, per_cu of them on every CU
unsigned grouped_grid(long long items, int per_cu) {
  return static_cast<unsigned>(std::min<long long>((items + 7) / 8 * 8, kCUs * per_cu));
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
  const long long items = (g.N + g.splits) * tiles_of(g.M, Sh::TM) * tiles_of(g.K, Sh::TN);
  auto launch = [&](auto kernel) { kernel<<<grouped_grid(items, Sh::PER_CU), Sh::THREADS, 0, s>>>(g); };
  if (whole_lines(g, g.K, sizeof(T)))
    launch(grouped_weights_kernel<T, true, Sh::MB, Sh::NB, Sh::WR, Sh::WC, Sh::DA, Sh::DB>);
  else
    launch(grouped_weights_kernel<T, false, Sh::MB, Sh::NB, Sh::WR, Sh::WC, Sh::DA, Sh::DB>);
}

hipError_t launch_join(const GroupedArgs &g, size_t total, int cols, bool bf16, hipStream_t s) {
  const size_t blocks = (total / (bf16 ? 8 : 4) + 255) / 256;
  const unsigned grid = static_cast<unsigned>(std::min<size_t>(std::max<size_t>(blocks, 1), 8 * kCUs));
  if (bf16)
    grouped_join_kernel<bf16_t><<<grid, 256, 0, s>>>(g, total, cols);
  else
    grouped_join_kernel<float><<<grid, 256, 0, s>>>(g, total, cols);
  return hipGetLastError();
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
  return launch_join(g, p.part_elems, cols, bf16, s);
}

}  // namespace

size_t grouped_workspace_bytes(const GroupedArgs &g, bool weights, bool grad, bool bf16) {
  if (g.S <= 0 && !weights) return 0;
  const Plan p = weights ? plan_weights(g, bf16) : plan_rows(g, grad, bf16);
  return p.splits > 1 ? p.splits * p.part_elems * sizeof(float) : 0;
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
  const dim3 grid(static_cast<unsigned>(std::min<size_t>(blocks, 64)), static_cast<unsigned>(std::min(g.N, g.S / g.chunk)));
  if (bf16)
    grouped_weights_join_kernel<bf16_t><<<grid, 256, 0, stream>>>(g);
  else
    grouped_weights_join_kernel<float><<<grid, 256, 0, stream>>>(g);
  return hipGetLastError();
}

}  // namespace ace
