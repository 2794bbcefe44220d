// The norms after one block and before the next, fused with the block's gate and the residual
// scale: one pass over the rows.
//   u  = y / rms(y) w_post      (y without a post-norm),  rms(v) = sqrt(mean(v^2) + eps)
//   h' = res_scale h + branch_scale gate u
//   n  = h' / rms(h') w_pre
// and the gradients, from the gradients dh' and dn of the two outputs:
//   p   = dn w_pre,  t = dh' + (p - h' (sum p h') / (d rms^2)) / rms        (rms of h')
//   dh  = res_scale t,  db = branch_scale t,  dgate = db u,  du = db gate
//   q   = du w_post, dy = (q - y (sum q y) / (d rms^2)) / rms               (rms of y)
//   dw_pre = sum over rows of dn h' / rms,  dw_post = sum over rows of du y / rms
// A row belongs to one workgroup whose threads keep its elements in registers between the
// sums, so every operand is read once and every result written once: HBM-bound.  All
// arithmetic and every sum is fp32, each result rounded once.
#include <algorithm>
#include <type_traits>

#include "ace_internal.h"

namespace ace {

namespace {

template <typename T> constexpr int kVec = 16 / static_cast<int>(sizeof(T));  // elements of a 16-byte access

template <typename T> __device__ __forceinline__ void load_vec(const T *p, float *f) {
  const uint4 v = *reinterpret_cast<const uint4 *>(p);
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 2) {
      f[2 * i] = __uint_as_float(w[i] << 16);
      f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    } else {
      f[i] = __uint_as_float(w[i]);
    }
  }
}

template <typename T> __device__ __forceinline__ void store_vec(T *p, const float *f) {
  uint4 v;
  if constexpr (sizeof(T) == 2)
    v = uint4{pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7])};
  else
    v = uint4{__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])};
  *reinterpret_cast<uint4 *>(p) = v;
}

// Sums over the workgroup, the same in every thread, in a fixed order.  Successive calls
// alternate between two LDS slots, so one barrier per call is enough.
template <int NT, int N> struct BlockSum {
  float (*red)[N][NT / 64];
  int par = 0;
  __device__ __forceinline__ void operator()(float (&v)[N]) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1)
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] += __shfl_xor(v[i], o);
    if constexpr (NT > 64) {
      const int wave = threadIdx.x >> 6;
      if ((threadIdx.x & 63) == 0)
#pragma unroll
        for (int i = 0; i < N; ++i) red[par][i][wave] = v[i];
      __syncthreads();
#pragma unroll
      for (int i = 0; i < N; ++i) {
        float s = 0.f;
#pragma unroll
        for (int w = 0; w < NT / 64; ++w) s += red[par][i][w];
        v[i] = s;
      }
      par ^= 1;
    }
  }
};

template <typename T> __device__ __forceinline__ float gate_of_row(const NormArgs &a, int row) {
  return a.gate_kind == 2 ? Elem<T>::load(static_cast<const T *>(a.gate) + row) : 1.f;
}

template <typename T, int NT, int CH> __global__ __launch_bounds__(NT) void block_norm_kernel(NormArgs a) {
  constexpr int V = kVec<T>;
  __shared__ float red[2][1][NT / 64];
  BlockSum<NT, 1> sum{red};
  const float inv_d = 1.f / static_cast<float>(a.d);
  for (int row = blockIdx.x; row < a.T; row += gridDim.x) {
    const size_t ro = static_cast<size_t>(row) * a.d;
    float h[CH][V], y[CH][V];
    float ss[1] = {0.f};
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int col = (c * NT + threadIdx.x) * V;
#pragma unroll
      for (int i = 0; i < V; ++i) h[c][i] = y[c][i] = 0.f;
      if (col < a.d) {
        load_vec(static_cast<const T *>(a.h) + ro + col, h[c]);
        if (a.y) load_vec(static_cast<const T *>(a.y) + ro + col, y[c]);
      }
#pragma unroll
      for (int i = 0; i < V; ++i) ss[0] += y[c][i] * y[c][i];
    }
    float s = 1.f;
    if (a.w_post) {
      sum(ss);
      s = 1.f / sqrtf(ss[0] * inv_d + a.eps);
    }
    const float gt = a.branch_scale * gate_of_row<T>(a, row);
    ss[0] = 0.f;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int col = (c * NT + threadIdx.x) * V;
      if (col < a.d && a.y) {
        float w[V], g[V];
#pragma unroll
        for (int i = 0; i < V; ++i) w[i] = g[i] = 1.f;
        if (a.w_post) load_vec(static_cast<const T *>(a.w_post) + col, w);
        if (a.gate_kind == 1) load_vec(static_cast<const T *>(a.gate) + col, g);
        if (a.gate_kind == 3) load_vec(static_cast<const T *>(a.gate) + ro + col, g);
#pragma unroll
        for (int i = 0; i < V; ++i) h[c][i] = a.res_scale * h[c][i] + gt * (g[i] * (y[c][i] * s * w[i]));
        store_vec(static_cast<T *>(a.out_h) + ro + col, h[c]);
      }
#pragma unroll
      for (int i = 0; i < V; ++i) ss[0] += h[c][i] * h[c][i];
    }
    if (a.w_pre) {
      sum(ss);
      const float r = 1.f / sqrtf(ss[0] * inv_d + a.eps);
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        const int col = (c * NT + threadIdx.x) * V;
        if (col < a.d) {
          float w[V];
          load_vec(static_cast<const T *>(a.w_pre) + col, w);
#pragma unroll
          for (int i = 0; i < V; ++i) w[i] *= h[c][i] * r;
          store_vec(static_cast<T *>(a.out_n) + ro + col, w);
        }
      }
    }
  }
}

// The parameter gradients are sums over rows: each workgroup takes the rows blockIdx.x,
// blockIdx.x + gridDim.x, .. and keeps its threads' columns of the sums in registers, then
// writes them to part [w_pre, w_post, gate [d]][gridDim.x][d], which param_sum_kernel adds in
// a fixed order (no atomics: equal calls give equal bits).
template <typename T, int NT, int CH> __global__ __launch_bounds__(NT) void block_norm_grad_kernel(NormArgs a) {
  constexpr int V = kVec<T>;
  __shared__ float red3[2][3][NT / 64], red2[2][2][NT / 64];
  BlockSum<NT, 3> sum3{red3};
  BlockSum<NT, 2> sum2{red2};
  const float inv_d = 1.f / static_cast<float>(a.d);
  float pre[CH][V], post[CH][V], gc[CH][V];
#pragma unroll
  for (int c = 0; c < CH; ++c)
#pragma unroll
    for (int i = 0; i < V; ++i) pre[c][i] = post[c][i] = gc[c][i] = 0.f;
  const bool need_y = a.y && (a.w_post || a.gate_kind);
  for (int row = blockIdx.x; row < a.T; row += gridDim.x) {
    const size_t ro = static_cast<size_t>(row) * a.d;
    float h[CH][V], y[CH][V], p[CH][V], t[CH][V];
    float s3[3] = {0.f, 0.f, 0.f};  // sum h'^2, sum p h', sum y^2
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int col = (c * NT + threadIdx.x) * V;
#pragma unroll
      for (int i = 0; i < V; ++i) h[c][i] = y[c][i] = p[c][i] = t[c][i] = 0.f;
      if (col < a.d) {
        if (a.dn) {
          load_vec(static_cast<const T *>(a.h) + ro + col, h[c]);
          load_vec(static_cast<const T *>(a.dn) + ro + col, p[c]);
        }
        if (need_y) load_vec(static_cast<const T *>(a.y) + ro + col, y[c]);
        if (a.dh) load_vec(static_cast<const T *>(a.dh) + ro + col, t[c]);
      }
      if (a.dn && col < a.d) {
        float w[V];
        load_vec(static_cast<const T *>(a.w_pre) + col, w);
#pragma unroll
        for (int i = 0; i < V; ++i) s3[1] += p[c][i] * w[i] * h[c][i];
      }
#pragma unroll
      for (int i = 0; i < V; ++i) {
        s3[0] += h[c][i] * h[c][i];
        s3[2] += y[c][i] * y[c][i];
      }
    }
    sum3(s3);
    const float r = 1.f / sqrtf(s3[0] * inv_d + a.eps);
    const float m = s3[1] * inv_d * r * r;
    const float s = a.w_post ? 1.f / sqrtf(s3[2] * inv_d + a.eps) : 1.f;
    const float gt = gate_of_row<T>(a, row);
    float s2[2] = {0.f, 0.f};  // sum q y, sum db u
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int col = (c * NT + threadIdx.x) * V;
      if (col >= a.d) continue;
      if (a.dn) {
        float w[V];
        load_vec(static_cast<const T *>(a.w_pre) + col, w);
#pragma unroll
        for (int i = 0; i < V; ++i) {
          pre[c][i] += p[c][i] * (h[c][i] * r);
          t[c][i] += r * (p[c][i] * w[i] - h[c][i] * m);
        }
      }
      float o[V];
#pragma unroll
      for (int i = 0; i < V; ++i) o[i] = a.res_scale * t[c][i];
      store_vec(static_cast<T *>(a.g_h) + ro + col, o);
      if (!a.y) continue;
      float w[V], g[V];
#pragma unroll
      for (int i = 0; i < V; ++i) w[i] = g[i] = 1.f;
      if (a.w_post) load_vec(static_cast<const T *>(a.w_post) + col, w);
      if (a.gate_kind == 1) load_vec(static_cast<const T *>(a.gate) + col, g);
      if (a.gate_kind == 3) load_vec(static_cast<const T *>(a.gate) + ro + col, g);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float db = a.branch_scale * t[c][i], yn = y[c][i] * s, du = db * (g[i] * gt);
        o[i] = db * (yn * w[i]);
        gc[c][i] += o[i];
        s2[1] += o[i];
        post[c][i] += du * yn;
        t[c][i] = du * w[i];
        s2[0] += t[c][i] * y[c][i];
      }
      if (a.gate_kind == 3) store_vec(static_cast<T *>(a.g_gate) + ro + col, o);
    }
    if (!a.y) continue;
    if (a.w_post || a.gate_kind == 2) sum2(s2);
    if (a.gate_kind == 2 && threadIdx.x == 0) static_cast<T *>(a.g_gate)[row] = Elem<T>::from_f32(s2[1]);
    const float k = a.w_post ? s2[0] * inv_d * s * s : 0.f;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int col = (c * NT + threadIdx.x) * V;
      if (col >= a.d) continue;
      float o[V];
#pragma unroll
      for (int i = 0; i < V; ++i) o[i] = s * (t[c][i] - y[c][i] * k);
      store_vec(static_cast<T *>(a.g_y) + ro + col, o);
    }
  }
  float *part = a.part;
  auto put = [&](const float (&acc)[CH][V]) {
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int col = (c * NT + threadIdx.x) * V;
      if (col >= a.d) continue;
      float *o = part + static_cast<size_t>(blockIdx.x) * a.d + col;
#pragma unroll
      for (int i = 0; i < V; i += 4)
        *reinterpret_cast<f32x4_t *>(o + i) = f32x4_t{acc[c][i], acc[c][i + 1], acc[c][i + 2], acc[c][i + 3]};
    }
    part += static_cast<size_t>(gridDim.x) * a.d;
  };
  if (a.g_pre) put(pre);
  if (a.g_post) put(post);
  if (a.gate_kind == 1) put(gc);
}

// Sums of `blocks` partial rows: 64 columns per workgroup, 16 waves take every 16th row
template <typename T> __global__ __launch_bounds__(1024) void param_sum_kernel(NormArgs a) {
  __shared__ float red[16][64];
  T *outs[3];
  int n = 0;
  if (a.g_pre) outs[n++] = static_cast<T *>(a.g_pre);
  if (a.g_post) outs[n++] = static_cast<T *>(a.g_post);
  if (a.gate_kind == 1) outs[n++] = static_cast<T *>(a.g_gate);
  T *out = blockIdx.y == 0 ? outs[0] : blockIdx.y == 1 ? outs[1] : outs[2];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int col = blockIdx.x * 64 + lane;
  const float *p = a.part + static_cast<size_t>(blockIdx.y) * a.blocks * a.d;
  float s = 0.f;
  if (col < a.d)
#pragma unroll 8
    for (int b = wave; b < a.blocks; b += 16) s += p[static_cast<size_t>(b) * a.d + col];
  red[wave][lane] = s;
  __syncthreads();
  if (wave == 0 && col < a.d) {
    s = 0.f;
#pragma unroll
    for (int w = 0; w < 16; ++w) s += red[w][lane];
    out[col] = Elem<T>::from_f32(s);
  }
}

constexpr int kNormBlocks = 2048;

// the smallest workgroup whose threads hold a row of d in one access each, else 1024
// threads with two or four
template <typename T, typename F> void by_width(int d, F f) {
  constexpr int V = kVec<T>;
  if (d <= 64 * V)
    f(std::integral_constant<int, 64>{}, std::integral_constant<int, 1>{});
  else if (d <= 128 * V)
    f(std::integral_constant<int, 128>{}, std::integral_constant<int, 1>{});
  else if (d <= 256 * V)
    f(std::integral_constant<int, 256>{}, std::integral_constant<int, 1>{});
  else if (d <= 512 * V)
    f(std::integral_constant<int, 512>{}, std::integral_constant<int, 1>{});
  else if (d <= 1024 * V)
    f(std::integral_constant<int, 1024>{}, std::integral_constant<int, 1>{});
  else if (d <= 2048 * V)
    f(std::integral_constant<int, 1024>{}, std::integral_constant<int, 2>{});
  else if constexpr (V == 4)
    f(std::integral_constant<int, 1024>{}, std::integral_constant<int, 4>{});
}

template <typename T> void launch_fwd(const NormArgs &a, hipStream_t s) {
  by_width<T>(a.d, [&](auto nt, auto ch) {
    block_norm_kernel<T, nt(), ch()><<<std::min(a.T, kNormBlocks), nt(), 0, s>>>(a);
  });
}

template <typename T> void launch_grad(const NormArgs &a, hipStream_t s) {
  by_width<T>(a.d, [&](auto nt, auto ch) { block_norm_grad_kernel<T, nt(), ch()><<<a.blocks, nt(), 0, s>>>(a); });
  const int n = (a.g_pre != nullptr) + (a.g_post != nullptr) + (a.gate_kind == 1);
  if (n > 0) param_sum_kernel<T><<<dim3((a.d + 63) / 64, n), 1024, 0, s>>>(a);
}

}  // namespace

int block_norm_grad_blocks(int T) { return T < 1 ? 1 : T < 512 ? T : 512; }

hipError_t launch_block_norm(const NormArgs &a, bool bf16, hipStream_t stream) {
  if (a.T <= 0) return hipSuccess;
  bf16 ? launch_fwd<bf16_t>(a, stream) : launch_fwd<float>(a, stream);
  return hipGetLastError();
}

hipError_t launch_block_norm_grad(const NormArgs &a, bool bf16, hipStream_t stream) {
  bf16 ? launch_grad<bf16_t>(a, stream) : launch_grad<float>(a, stream);
  return hipGetLastError();
}

}  // namespace ace
