// Host-side check of how 4-bit operands are staged (mx4_tile.h): for every operand of the kernels' shapes, reduction
// lengths from one block to several panels, whole and in parts (the four waves of a workgroup, or 2 .. 64 launched
// parts), replay each lane's copies of codes and panels of scales, a dword at a time as the descriptors bound them, from
// tensors that end where their memory ends.  No dword comes from outside, and what the products read from LDS is the
// row's codes and scales, zeros behind a part's end and past the last row.  Prints "ok" and exits 0, else the first mismatch.
#include <cstdio>
#include <cstring>
#include <memory>
#include <vector>

#include "../paper_2609_05228_amd/csrc/mx4_tile.h"

namespace {

uint8_t code_at(int m, int row, int i) { return static_cast<uint8_t>(17 * m + 31 * row + 7 * i + 1); }
uint8_t scale_at(int m, int row, int i) { return static_cast<uint8_t>(1 + (101 * m + 13 * row + 5 * i) % 254); }

// 16 bytes as buffer_load_dwordx4 brings them: dwords past the descriptor are zero; false: one lies outside the tensor
bool copy16(uint8_t *to, const uint8_t *base, uint32_t bytes, uint32_t off, const std::vector<uint8_t> &from) {
  for (uint32_t d = off; d < off + 16; d += 4, to += 4) {
    if (d + 4 > bytes) {
      std::memset(to, 0, 4);
      continue;
    }
    const uint8_t *p = base + d;
    if (p < from.data() || p + 4 > from.data() + from.size()) return false;
    std::memcpy(to, p, 4);
  }
  return true;
}

template <int BLK, bool PAIR, int W, int MATS> bool part(int K, int valid, ace::Part k) {
  using Op = ace::Mx4Operand<BLK, PAIR, W, MATS>;
  const int code_row = K / 2, scale_row = static_cast<int>(ace::mx4_scale_row(K));
  std::vector<uint8_t> codes[MATS], scales[MATS];
  typename Op::Src src;
  for (int m = 0; m < MATS; ++m) {
    for (int r = 0; r < valid; ++r) {
      for (int i = 0; i < code_row; ++i) codes[m].push_back(code_at(m, r, i));
      for (int i = 0; i < scale_row; ++i) scales[m].push_back(scale_at(m, r, i));
    }
    codes[m].shrink_to_fit();
    scales[m].shrink_to_fit();
    src.codes[m] = codes[m].data();
    src.scales[m] = scales[m].data();
  }
  src.k0 = k.k0;
  std::unique_ptr<ace::i32x4_t[]> ring(new ace::i32x4_t[Op::BYTES / 16]), place(new ace::i32x4_t[Op::PANEL / 16]);
  uint8_t *lds = reinterpret_cast<uint8_t *>(ring.get()), *panel = reinterpret_cast<uint8_t *>(place.get());
  auto fail = [&](const char *what, int s, int lane) {
    std::printf("BLK=%d W=%d MATS=%d K=%d valid=%d k0=%d len=%d stage %d lane %d: %s\n", BLK, W, MATS, K, valid, k.k0, k.len,
                s, lane, what);
    return false;
  };
  const int nk = (k.len + Op::BK - 1) / Op::BK;
  for (int s = 0; s < nk; ++s) {
    for (int wave = 0; wave < W; ++wave)
      for (int lane = 0; lane < 64; ++lane) {
        Op op;
        op.init(src, K, valid, k.len, wave, lane);
        if (s % Op::PANEL_STAGES == 0)
          for (int t = 0; t < Op::NP; ++t) {
            const int i = wave * Op::NP + t;
            if (i >= MATS * Op::GROUPS) continue;
            const uint32_t at = Op::panel_at(s);
            if (!copy16(panel + i * ace::kUnitBytes + 16 * lane, op.scales[t] + at, op.scale_span - at, op.poff[t],
                        scales[i / Op::GROUPS]))
              return fail("a panel's dword outside the scales", s, lane);
          }
        for (int t = 0; t < Op::NU; ++t) {
          const int u = wave * Op::NU + t, to = u < Op::UNITS ? u : Op::UNITS, m = u < Op::UNITS ? u / (Op::UNITS / MATS) : 0;
          const uint32_t at = Op::codes_at(s);
          const uint8_t *base = MATS == 2 && W == 1 && t >= Op::UNITS / MATS ? op.codes2 : op.codes;
          if (!copy16(lds + to * ace::kUnitBytes + 16 * lane, base + at, op.code_span - at,
                      op.in_stage(s) ? op.voff[t] : ace::kOutside, codes[m]))
            return fail("a chunk's dword outside the codes", s, lane);
        }
      }
    for (int blk = 0; blk < BLK; ++blk)
      for (int lane = 0; lane < 64; ++lane) {
        const int m = blk % MATS, row = ace::block_row<PAIR>(blk / MATS, lane & 15), b = lane >> 4, kk = s * Op::BK + 32 * b;
        const bool there = row < valid && kk < k.len;
        const ace::i32x4_t got = Op::read(lds, blk, lane);
        uint8_t bytes[16];
        std::memcpy(bytes, &got, 16);
        for (int i = 0; i < 16; ++i)
          if (bytes[i] != (there ? code_at(m, row, (k.k0 + kk) / 2 + i) : 0)) return fail("codes", s, lane);
        const int scale = Op::read_scale(panel, blk, lane, s * Op::BK, k.len);
        if (there ? scale != scale_at(m, row, (k.k0 + kk) / 32) : kk >= k.len && scale != 0) return fail("scale", s, lane);
      }
  }
  return true;
}

template <int BLK, bool PAIR, int W, int MATS> bool check(bool waves, bool parts) {
  for (int K : {32, 64, 96, 128, 160, 352, 480, 512, 544, 640, 768, 1024, 1056, 1536, 2048, 2080, 7168})
    for (int valid : {1, 8, 16 * BLK / MATS - 8, 16 * BLK / MATS}) {
      if (valid < 1) continue;
      for (int n = 1; n <= (parts ? 64 : waves ? 4 : 1); n *= 2) {
        if (n == 2 && !parts) continue;
        for (int s = 0; s < n; ++s)
          if (!part<BLK, PAIR, W, MATS>(K, valid, ace::part_of<128>(K, s, n))) return false;
      }
    }
  return true;
}

}  // namespace

int main() {
  // weights: few rows, 16, 64 and the large tiles; rows in 4 bits of the same
  const bool ok = check<4, true, 1, 1>(true, false) && check<4, true, 1, 2>(true, false) && check<1, false, 1, 1>(true, false) &&
                  check<16, true, 4, 1>(false, false) && check<16, true, 4, 2>(false, false) && check<1, false, 4, 1>(false, false) &&
                  check<8, true, 4, 1>(false, true) && check<8, true, 4, 2>(false, true) && check<4, false, 4, 1>(false, true) &&
                  check<16, true, 8, 1>(false, false) && check<16, true, 8, 2>(false, false) && check<12, true, 8, 1>(false, false) &&
                  check<16, false, 8, 1>(false, false) && check<20, false, 8, 1>(false, false);
  if (ok) std::printf("ok\n");
  return ok ? 0 : 1;
}
