// The activations of the gated feed-forward block, and what becomes of a tile's two projections (gated.hip, mx4.hip).
#pragma once

#include "grouped_tile.h"

namespace ace {

// z^2 / 2 log2(e) = -(e + rest) for 0 <= z <= 20 to 4e-12: what z^2 and its product with log2(e) / 2 lose to rounding, in rest
struct HalfSquare {
  float e, rest;
};
__host__ __device__ __forceinline__ HalfSquare half_square(float z) {
  constexpr float c = 0.72134752f, c_rest = 9.6298150e-9f;  // log2(e) / 2 = c + c_rest
  const float h = z * z, l = fmaf(z, z, -h), e = -c * h;
  return {e, -fmaf(c, h, e) - c * l - c_rest * h};
}

// exp(-z^2 / 2) for 0 <= z <= 20, to the roundings of the hardware base-2 exponential and of two operations; where it
// is below the least normal number (z > 13.2) it may be 0
__device__ __forceinline__ float half_square_exp(float z) {
  const HalfSquare v = half_square(z);
  return __builtin_amdgcn_exp2f(v.e) * fmaf(v.rest, 0.69314718f, 1.f);
}

// Phi(-z) e^(z^2 / 2) for z >= 0, which falls smoothly from 1/2 as 1 / (sqrt(2 pi) z): t P(t) with t = 1 / (1 + 0.32 z)
// and P a polynomial fitted to the least relative error (4.5e-8 over all z >= 0 with the coefficients as they are; 3.3e-7
// with fp32 arithmetic)
constexpr float kTail[10] = {-0.0210784f, 0.095408306f, -0.14670941f, 0.06532997f, -0.009378675f,
                             0.058654312f, 0.087829046f, 0.11462236f, 0.12766095f, 0.12766153f};
template <typename R> __host__ __device__ __forceinline__ R tail_of(R t) {
  R p = kTail[0];
#pragma unroll
  for (int i = 1; i < 10; ++i) p = fma(p, t, static_cast<R>(kTail[i]));
  return p * t;
}
__device__ __forceinline__ float normal_tail(float z) { return tail_of(__builtin_amdgcn_rcpf(fmaf(0.32f, z, 1.f))); }

// act(g), and with SLOPE act'(g).  SiLU of bf16 results: hardware exponential and reciprocal (see silu_for_bf16).
template <typename T, int ACT> struct Activation {
  static __device__ __forceinline__ float value(float g) {
    float s;
    return both<false>(g, s);
  }
  template <bool SLOPE> static __device__ __forceinline__ float both(float g, float &slope) {
    if constexpr (ACT == kActSilu) {
      const float s = sizeof(T) == 2 ? __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(g * -1.4426950408889634f))
                                     : 1.f / (1.f + expf(-g));
      if (SLOPE) slope = s * fmaf(g, 1.f - s, 1.f);
      return g * s;
    } else {
      const float z = fminf(fabsf(g), 20.f);  // Phi(-20) is 0 in fp32
      const float e = half_square_exp(z), tail = e * normal_tail(z), phi = g < 0.f ? tail : 1.f - tail;
      if (SLOPE) slope = fmaf(g * 0.39894228f, e, phi);
      return g * phi;
    }
  }
};

// 4 consecutive elements of a row
__device__ __forceinline__ void load4(const float *p, f32x4_t &v) { v = *reinterpret_cast<const f32x4_t *>(p); }
__device__ __forceinline__ void load4(const bf16_t *p, f32x4_t &v) {
  const uint2 b = *reinterpret_cast<const uint2 *>(p);
  v = f32x4_t{__uint_as_float(b.x << 16), __uint_as_float(b.x & 0xffff0000u), __uint_as_float(b.y << 16),
              __uint_as_float(b.y & 0xffff0000u)};
}
__device__ __forceinline__ void store4(float *p, f32x4_t v) { *reinterpret_cast<f32x4_t *>(p) = v; }
__device__ __forceinline__ void store4(bf16_t *p, f32x4_t v) {
  *reinterpret_cast<uint2 *>(p) = uint2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
}

// a tile of both projections
template <class S> struct GatedRef : S::Ref {
  size_t at;  // its first element in g, u, a, da, dg and du
};

// A wave's share of g and u: what is asked of them, a 16-row block at a time (the whole share at once would hold
// a second copy of the accumulators)
template <typename T, bool LINES, class S> struct GatedStore {
  const GatedArgs &g;
  static constexpr int NH = S::NW / 2;
  typedef f32x4_t Block[1][NH];

  __device__ __forceinline__ void put(const GatedRef<S> &t, void *out, const Block &v, int blk, int c0, int lane) const {
    store_rows<T, LINES, 1, NH, 1>(static_cast<T *>(out) + t.at, t.rows, t.cols, g.M, v, blk, c0, lane);
  }
  // dg into the place of g, du into that of u
  template <int ACT>
  __device__ __forceinline__ void slopes(const GatedRef<S> &t, Block &vg, Block &vu, int blk, int c0, int lane) const {
    const int row = 16 * blk + (lane & 15), l4 = lane >> 4;
    const T *p = static_cast<const T *>(g.da) + t.at + static_cast<size_t>(row) * g.M;
    f32x4_t da[NH];
#pragma unroll
    for (int j = 0; j < NH; ++j) {
      const int col = c0 + (sizeof(T) == 2 ? 16 * (j & ~1) + 8 * l4 + 4 * (j & 1) : 16 * j + 4 * l4);
      da[j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
      if (row < t.rows && col < t.cols) load4(p + col, da[j]);
    }
#pragma unroll
    for (int j = 0; j < NH; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        float slope;
        const float f = Activation<T, ACT>::template both<true>(vg[0][j][q], slope);
        vg[0][j][q] = da[j][q] * vu[0][j][q] * slope;
        vu[0][j][q] = da[j][q] * f;
      }
  }
  template <int ACT> __device__ __forceinline__ void values(Block &vg, const Block &vu) const {
#pragma unroll
    for (int j = 0; j < NH; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q) vg[0][j][q] = Activation<T, ACT>::value(vg[0][j][q]) * vu[0][j][q];
  }

  __device__ __forceinline__ void operator()(const GatedRef<S> &t, const f32x4_t (&sum)[S::MW][S::NW], int wr, int wc,
                                             int lane) const {
    const int c0 = 8 * wc * S::NW;
#pragma unroll
    for (int i = 0; i < S::MW; ++i) {
      const int blk = wr + S::WR * i;
      if (16 * blk >= t.rows) break;  // wave-uniform
      Block vg, vu;
#pragma unroll
      for (int j = 0; j < NH; ++j) {
        vg[0][j] = sum[i][2 * j];
        vu[0][j] = sum[i][2 * j + 1];
      }
      if (t.part) {
        store_part<T, 1, NH, 1>(t.part, t.rows, t.cols, g.M, vg, blk, c0, lane);
        store_part<T, 1, NH, 1>(t.part + static_cast<size_t>(g.S) * g.M, t.rows, t.cols, g.M, vu, blk, c0, lane);
      } else if (g.da) {
        if (g.act == kActSilu)
          slopes<kActSilu>(t, vg, vu, blk, c0, lane);
        else
          slopes<kActGelu>(t, vg, vu, blk, c0, lane);
        put(t, g.dg, vg, blk, c0, lane);
        put(t, g.du, vu, blk, c0, lane);
      } else {
        if (g.g) {
          put(t, g.g, vg, blk, c0, lane);
          put(t, g.u, vu, blk, c0, lane);
        }
        if (g.act == kActSilu)
          values<kActSilu>(vg, vu);
        else
          values<kActGelu>(vg, vu);
        put(t, g.a, vg, blk, c0, lane);
      }
    }
  }
};

}  // namespace ace
