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
// sums, so every operand is read once and every result written once: the forward is HBM-bound.  All
// arithmetic and every sum is fp32, each result rounded once.
#include <algorithm>
#include <type_traits>

#include "lds_dma.h"

namespace ace {

namespace {

template <typename T> constexpr int kVec = 16 / static_cast<int>(sizeof(T));  // elements of a 16-byte access

template <typename T> __device__ __forceinline__ void unpack(const uint4 &v, float *f) {
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

template <typename T> __device__ __forceinline__ void load_vec(const T *p, float *f) {
  unpack<T>(*reinterpret_cast<const uint4 *>(p), f);
}

template <typename T> __device__ __forceinline__ void store_vec(T *p, const float *f) {
  uint4 v;
  if constexpr (sizeof(T) == 2)
    v = uint4{pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7])};
  else
    v = uint4{__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])};
  *reinterpret_cast<uint4 *>(p) = v;
}

// Sum over a wave in a fixed order, the same in every lane: within rows of 16 lanes by DPP, then across
// the rows (a lane exchange through LDS takes several times as long)
template <int CTRL, int ROWS> __device__ __forceinline__ float dpp_add(float v) {
  return v + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, ROWS, 0xf, true));
}
// over N <= 16 neighbouring lanes rounded up to a power of two, in each of them
template <int N> __device__ __forceinline__ float lanes_sum(float v) {
  if constexpr (N > 1) v = dpp_add<0xb1, 0xf>(v);   // lanes 1 apart
  if constexpr (N > 2) v = dpp_add<0x4e, 0xf>(v);   // 2 apart
  if constexpr (N > 4) v = dpp_add<0x141, 0xf>(v);  // mirrored in 8
  if constexpr (N > 8) v = dpp_add<0x140, 0xf>(v);  // mirrored in 16
  return v;
}
__device__ __forceinline__ float wave_sum(float v) {
  v = lanes_sum<16>(v);
  v = dpp_add<0x142, 0xa>(v);  // rows 1 and 3 add the row before
  v = dpp_add<0x143, 0xc>(v);  // rows 2 and 3 add row 1's: lane 63 holds all
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}

// of N waves' sums in LDS, in every lane
template <int N> __device__ __forceinline__ float waves_sum(const float *sums) {
  constexpr int P = N <= 1 ? 1 : N <= 2 ? 2 : N <= 4 ? 4 : N <= 8 ? 8 : 16;
  const int l = threadIdx.x % P;
  return lanes_sum<N>(l < N ? sums[l] : 0.f);
}

// Sums over the workgroup, the same in every thread, in a fixed order.  Successive calls
// alternate between two LDS slots, so one barrier per call is enough.
template <int NT, int N> struct BlockSum {
  float (*red)[N][NT / 64];
  int par = 0;
  __device__ __forceinline__ void operator()(float (&v)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = wave_sum(v[i]);
    if constexpr (NT > 64) {
      const int wave = threadIdx.x >> 6;
      if ((threadIdx.x & 63) == 0)
#pragma unroll
        for (int i = 0; i < N; ++i) red[par][i][wave] = v[i];
      __syncthreads();
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] = waves_sum<NT / 64>(red[par][i]);
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

// Sums over the NT threads of each of a workgroup's RG rows, the same in each of them, in a fixed
// order; as BlockSum, with one barrier of the workgroup, none where a row is one wave's.
template <int NT, int RG, int N> struct RowSum {
  float (*red)[RG][N][NT / 64];
  int par = 0;
  __device__ __forceinline__ void operator()(float (&v)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = wave_sum(v[i]);
    if constexpr (NT > 64) {
      const int grp = threadIdx.x / NT, wave = (threadIdx.x % NT) >> 6;
      if ((threadIdx.x & 63) == 0)
#pragma unroll
        for (int i = 0; i < N; ++i) red[par][grp][i][wave] = v[i];
      __syncthreads();
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] = waves_sum<NT / 64>(red[par][grp][i]);
      par ^= 1;
    }
  }
};

// A workgroup takes RG rows at a time (NT threads each).  While it works on them, held in registers as
// stored and widened where used, the next ones are copied into LDS (each thread its own 16 bytes of
// each operand, so no barrier is needed for them); weights and a gate per channel lie in LDS too.  As compiled, a
// round's first reads of LDS wait for all of the wave's memory operations, the last row's stores among them
// (the choice between an operand and zeros is made between addresses, so they are flat loads), and a gate per
// token or element, loaded behind the next rows' copies, waits for those.
// The parameter gradients are sums over rows: a thread keeps its columns' sums of its rows in registers,
// the RG rows' are added through LDS at the end, and each workgroup writes one line of part
// [w_pre, w_post, gate [d]][gridDim.x][d], which param_sum_kernel adds in a fixed order (no atomics:
// equal calls give equal bits).  RG rows at a time keep these lines few.
// Not at the memory's rate: 4096 rows of 2048 (bf16) take 28.6 us with a gate per channel, 27.7 per token, 29.9 per
// element, where the memory takes 19.4, 19.4 and 25.8; 4 of them are param_sum_kernel's.  Some 30 fp32 operations
// an element and the waits above stand beside it.  Rows past 8192 elements spill registers (72 in bf16, 83 in
// fp32; from 5128 on 11 in bf16): 2048 rows of 16384 (bf16) take 231 us, the memory 78.
template <typename T, int NT, int CH, int RG>
__global__ __launch_bounds__(NT *RG) void block_norm_grad_kernel(NormArgs a) {
  constexpr int V = kVec<T>;
  constexpr bool AHEAD = CH == 1;  // longer rows would not fit LDS
  __shared__ float red3[2][RG][3][NT / 64], red2[2][RG][2][NT / 64];
  __shared__ f32x4_t join[RG > 1 ? RG - 1 : 1][RG > 1 ? NT * V / 4 : 1];
  __shared__ uint4 params[3][AHEAD ? NT : 1];                    // w_pre, w_post, gate [d]
  __shared__ uint4 ahead[AHEAD ? NT * RG / 64 : 1][4][64];       // a wave's h, dn, y, dh
  RowSum<NT, RG, 3> sum3{red3};
  RowSum<NT, RG, 2> sum2{red2};
  const float inv_d = 1.f / static_cast<float>(a.d);
  const int tid = threadIdx.x % NT, grp = threadIdx.x / NT;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  float pre[CH][V], post[CH][V], gc[CH][V];
#pragma unroll
  for (int c = 0; c < CH; ++c)
#pragma unroll
    for (int i = 0; i < V; ++i) pre[c][i] = post[c][i] = gc[c][i] = 0.f;
  const bool need_y = a.y && (a.w_post || a.gate_kind);
  const void *src[4] = {a.dn ? a.h : nullptr, a.dn, need_y ? a.y : nullptr, a.dh};
  const uint4 zero{0, 0, 0, 0};
  const uint32_t one = sizeof(T) == 2 ? 0x3f803f80u : 0x3f800000u;
  // chunk c of a parameter: ones where there is none
  auto fetch_param = [&](int k, int c) {
    const int col = (c * NT + tid) * V;
    const void *p = k == 0 ? a.w_pre : k == 1 ? a.w_post : a.gate_kind == 1 ? a.gate : nullptr;
    return p && col < a.d ? *reinterpret_cast<const uint4 *>(static_cast<const T *>(p) + col) : uint4{one, one, one, one};
  };
  auto param = [&](int k, int c, float *f) {
    if constexpr (AHEAD)
      unpack<T>(params[k][tid], f);
    else
      unpack<T>(fetch_param(k, c), f);
  };
  const bool wide = tid * V < a.d;
  const uint32_t slot = lds_addr(ahead[AHEAD ? wave : 0]);
  auto copy = [&](int row) {
    if (row < a.T && wide)
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (src[k]) dma16(static_cast<const T *>(src[k]) + static_cast<size_t>(row) * a.d + tid * V, slot + k * 1024);
  };
  const int step = static_cast<int>(gridDim.x) * RG;
  if constexpr (AHEAD) {
    copy(blockIdx.x * RG + grp);
    if (grp == 0)
#pragma unroll
      for (int k = 0; k < 3; ++k) params[k][tid] = fetch_param(k, 0);
    __syncthreads();
  }
  // stores of a wave after the copies that it waits for: at least these (a wave's memory operations finish
  // in order; see above for what is waited for behind it)
  const int behind = 1 + (a.y != nullptr) + (a.gate_kind == 3);
  bool first = true;
  for (int row0 = blockIdx.x * RG; row0 < a.T; row0 += step) {
    const int row = row0 + grp;
    const bool there = row < a.T;
    const size_t ro = static_cast<size_t>(row) * a.d;
    uint4 cur[4][CH];  // h, dn, y, dh
    if constexpr (AHEAD) {
      if (first || !there)
        wait_vmcnt_in<0, 0>(0);
      else
        wait_vmcnt_in<1, 3>(behind);
      first = false;
#pragma unroll
      for (int k = 0; k < 4; ++k) cur[k][0] = there && wide && src[k] ? ahead[wave][k][lane] : zero;
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // read before the next copies overwrite it
#pragma unroll
      for (int k = 0; k < 4; ++k) asm volatile("" : "+v"(cur[k][0].x), "+v"(cur[k][0].y), "+v"(cur[k][0].z), "+v"(cur[k][0].w));
      if (step < a.T - row0) copy(row + step);
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int c = 0; c < CH; ++c) {
          const int col = (c * NT + tid) * V;
          cur[k][c] = there && col < a.d && src[k] ? *reinterpret_cast<const uint4 *>(static_cast<const T *>(src[k]) + ro + col) : zero;
        }
    }
    float s3[3] = {0.f, 0.f, 0.f};  // sum h'^2, sum p h', sum y^2
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      float h[V], p[V], y[V], w[V];
      unpack<T>(cur[0][c], h);
      unpack<T>(cur[1][c], p);
      unpack<T>(cur[2][c], y);
      param(0, c, w);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        s3[0] += h[i] * h[i];
        s3[1] += p[i] * w[i] * h[i];
        s3[2] += y[i] * y[i];
      }
    }
    sum3(s3);
    const float r = 1.f / sqrtf(s3[0] * inv_d + a.eps);
    const float mr = s3[1] * inv_d * r * r * r;
    const float s = a.w_post ? 1.f / sqrtf(s3[2] * inv_d + a.eps) : 1.f;
    const float gt = there ? a.branch_scale * gate_of_row<T>(a, row) : 0.f;
    float q[CH][V];
    float s2[2] = {0.f, 0.f};  // sum q y, sum t u
    // a row that is not there adds nothing to the parameters' sums: its zeros times an infinite parameter would
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      if (!there) break;
      const int col = (c * NT + tid) * V;
      const bool in = col < a.d;
      float h[V], p[V], y[V], t[V], w[V], o[V];
      unpack<T>(cur[0][c], h);
      unpack<T>(cur[1][c], p);
      unpack<T>(cur[2][c], y);
      unpack<T>(cur[3][c], t);
      param(0, c, w);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float pr = p[i] * r;
        pre[c][i] += pr * h[i];
        t[i] += pr * w[i] - h[i] * mr;
        o[i] = a.res_scale * t[i];
      }
      if (in) store_vec(static_cast<T *>(a.g_h) + ro + col, o);
      if (!a.y) continue;
      float g[V];
      param(1, c, w);
      param(2, c, g);
      if (a.gate_kind == 3 && in) load_vec(static_cast<const T *>(a.gate) + ro + col, g);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float tyn = t[i] * (y[i] * s), gg = g[i] * gt;
        o[i] = tyn * w[i];
        gc[c][i] += o[i];
        s2[1] += o[i];
        post[c][i] += tyn * gg;
        q[c][i] = t[i] * gg * w[i];
        s2[0] += q[c][i] * y[i];
      }
      if (a.gate_kind == 3 && in) {
#pragma unroll
        for (int i = 0; i < V; ++i) o[i] *= a.branch_scale;
        store_vec(static_cast<T *>(a.g_gate) + ro + col, o);
      }
    }
    if (!a.y) continue;
    if (a.w_post || a.gate_kind == 2) sum2(s2);
    if (a.gate_kind == 2 && tid == 0 && there)
      static_cast<T *>(a.g_gate)[row] = Elem<T>::from_f32(a.branch_scale * s2[1]);
    const float k = s2[0] * inv_d * s * s * s;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int col = (c * NT + tid) * V;
      if (a.w_post) {  // else dy is q, whatever y is
        float y[V];
        unpack<T>(cur[2][c], y);
#pragma unroll
        for (int i = 0; i < V; ++i) q[c][i] = s * q[c][i] - y[i] * k;
      }
      if (there && col < a.d) store_vec(static_cast<T *>(a.g_y) + ro + col, q[c]);
    }
  }
  float *part = a.part;
  auto put = [&](float (&acc)[CH][V], float scale) {
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      if constexpr (RG > 1) {
        __syncthreads();
        if (grp > 0)
#pragma unroll
          for (int i = 0; i < V; i += 4)
            join[grp - 1][tid * (V / 4) + i / 4] = f32x4_t{acc[c][i], acc[c][i + 1], acc[c][i + 2], acc[c][i + 3]};
        __syncthreads();
      }
      const int col = (c * NT + tid) * V;
      if (grp > 0 || col >= a.d) continue;
      float *o = part + static_cast<size_t>(blockIdx.x) * a.d + col;
#pragma unroll
      for (int i = 0; i < V; i += 4) {
        f32x4_t v = {acc[c][i], acc[c][i + 1], acc[c][i + 2], acc[c][i + 3]};
        if constexpr (RG > 1)
          for (int k = 0; k < RG - 1; ++k) v += join[k][tid * (V / 4) + i / 4];
        *reinterpret_cast<f32x4_t *>(o + i) = v * scale;
      }
    }
    part += static_cast<size_t>(gridDim.x) * a.d;
  };
  if (a.g_pre) put(pre, 1.f);
  if (a.g_post) put(post, 1.f);
  if (a.gate_kind == 1) put(gc, a.branch_scale);
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
constexpr int kGradBlocks = 256;  // a workgroup a CU

// Threads of a gradient workgroup: 1024, or 512 where those would not fill the CUs once (bf16: 117 rows of 384
// 10.8 us with 1024 and 8.4 with 512, 1574 rows of 200 11.6 and 9.8; 4096 rows of 2048 29 and 32, 10819 of 1296 63 and 77;
// of the bf16 kernel's 131 to 135 registers only one such workgroup fits a CU, of the fp32 kernel's 86 to 94 two).
// They come as whole rows' threads.
constexpr int grad_small(int nt) { return nt >= 512 ? nt : 512 / nt * nt; }
constexpr int grad_large(int nt) { return 1024 / nt * nt; }
int grad_threads(int T, int nt) {
  return static_cast<long long>(T) <= static_cast<long long>(kGradBlocks) * (1024 / nt) ? grad_small(nt) : grad_large(nt);
}

// Threads of a row: the fewest of these that hold it in one access each, else 1024 with two or four.  Between the
// powers of two as well: 15927 rows of 1088 (bf16) took the gradient 81 us with 256 threads, of which it uses 136.
constexpr int kRowThreads[] = {64, 128, 192, 256, 320, 512, 640, 1024};
int row_threads(int d, int vec) {
  for (int nt : kRowThreads)
    if (d <= nt * vec) return nt;
  return 1024;
}

template <typename T, typename F> void by_width(int d, F f) {
  constexpr int V = kVec<T>;
  using std::integral_constant;
  const integral_constant<int, 1> one{};
  if (d > 2048 * V) {
    if constexpr (V == 4) f(integral_constant<int, 1024>{}, integral_constant<int, 4>{});
    return;
  }
  if (d > 1024 * V) return f(integral_constant<int, 1024>{}, integral_constant<int, 2>{});
  switch (row_threads(d, V)) {
    case 64: return f(integral_constant<int, 64>{}, one);
    case 128: return f(integral_constant<int, 128>{}, one);
    case 192: return f(integral_constant<int, 192>{}, one);
    case 256: return f(integral_constant<int, 256>{}, one);
    case 320: return f(integral_constant<int, 320>{}, one);
    case 512: return f(integral_constant<int, 512>{}, one);
    case 640: return f(integral_constant<int, 640>{}, one);
    default: return f(integral_constant<int, 1024>{}, one);
  }
}

template <typename T> void launch_fwd(const NormArgs &a, hipStream_t s) {
  by_width<T>(a.d, [&](auto nt, auto ch) {
    block_norm_kernel<T, nt(), ch()><<<std::min(a.T, kNormBlocks), nt(), 0, s>>>(a);
  });
}

template <typename T> void launch_grad(const NormArgs &a, hipStream_t s) {
  by_width<T>(a.d, [&](auto nt, auto ch) {
    constexpr int NT = nt(), SMALL = grad_small(NT), LARGE = grad_large(NT);
    if (grad_threads(a.T, NT) == SMALL)
      block_norm_grad_kernel<T, NT, ch(), SMALL / NT><<<a.blocks, SMALL, 0, s>>>(a);
    else
      block_norm_grad_kernel<T, NT, ch(), LARGE / NT><<<a.blocks, LARGE, 0, s>>>(a);
  });
  const int n = (a.g_pre != nullptr) + (a.g_post != nullptr) + (a.gate_kind == 1);
  if (n > 0) param_sum_kernel<T><<<dim3((a.d + 63) / 64, n), 1024, 0, s>>>(a);
}

}  // namespace

int block_norm_grad_blocks(int T, int d, bool bf16) {
  const int nt = row_threads(d, bf16 ? 8 : 4);
  const int threads = grad_threads(T, nt), rows = threads / nt;  // of a workgroup at a time
  return std::min((std::max(T, 1) - 1) / rows + 1, threads <= 512 ? 2 * kGradBlocks : kGradBlocks);
}

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
