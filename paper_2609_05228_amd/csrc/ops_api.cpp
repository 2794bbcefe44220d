// C ABI of the operators around the layer (grouped matrix products, the norms before and
// after a block, low-rank adapters): host-side validation, then the launches.  Nothing is
// allocated and no call keeps state.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "../../include/ace.h"
#include "ace_internal.h"

namespace {

constexpr int32_t kMaxGroups = 4096;  // groups of rows, requests
constexpr int32_t kMaxWidth = 65536;  // feature sizes
constexpr int32_t kMaxNormWidth = 16384;
constexpr int32_t kMaxRank = 128;
constexpr int32_t kMaxRows = 0x7fffffff - 65536;  // rounding up to a tile, a stage or a grid's rows stays an int

bool is_dtype(int32_t t) { return t == ACE_F32 || t == ACE_BF16; }
size_t elem_bytes(int32_t t) { return t == ACE_BF16 ? 2 : 4; }
// feature sizes are whole 16-byte accesses
bool bad_width(int32_t n, int32_t dtype) { return n % static_cast<int32_t>(16 / elem_bytes(dtype)) != 0; }

bool usable(const void *p, size_t align) { return p && (reinterpret_cast<uintptr_t>(p) & (align - 1)) == 0; }

struct Span {
  const void *p;
  size_t bytes;
};
bool overlap(const Span &a, const Span &b) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a.p), y = reinterpret_cast<uintptr_t>(b.p);
  return a.p && b.p && a.bytes && b.bytes && x < y + b.bytes && y < x + a.bytes;
}

ace_status status_of(hipError_t e) {
  return e == hipSuccess ? ACE_OK : e == hipErrorInvalidValue ? ACE_ERR_UNSUPPORTED : ACE_ERR_HIP;
}

enum class Way { kForward = ACE_GROUPED_FORWARD, kGradX = ACE_GROUPED_GRAD_X, kGradW = ACE_GROUPED_GRAD_W };

ace_status grouped_desc(const ace_grouped_desc *d) {
  if (!d) return ACE_ERR_INVALID_ARG;
  if (d->S < 0 || d->N <= 0 || d->M <= 0 || d->K <= 0 || !is_dtype(d->dtype) ||
      (d->flags & ~static_cast<uint32_t>(ACE_ZERO_REST)))
    return ACE_ERR_INVALID_ARG;
  if (d->S > kMaxRows || d->N > kMaxGroups || d->M > kMaxWidth || d->K > kMaxWidth || bad_width(d->M, d->dtype) ||
      bad_width(d->K, d->dtype))
    return ACE_ERR_UNSUPPORTED;
  return ACE_OK;
}

ace::GroupedArgs grouped_args(const ace_grouped_desc &d) {
  ace::GroupedArgs g{};
  g.S = d.S;
  g.N = d.N;
  g.M = d.M;
  g.K = d.K;
  g.fill = (d.flags & ACE_ZERO_REST) ? 1 : 0;
  return g;
}

size_t grouped_bytes(const ace_grouped_desc &d, Way way) {
  return ace::grouped_workspace_bytes(grouped_args(d), way == Way::kGradW, way == Way::kGradX, d.dtype == ACE_BF16);
}

ace_status grouped(const ace_grouped_desc *d, Way way, const void *rows, const void *other, const int32_t *offsets,
                   void *out, void *workspace, size_t workspace_bytes, void *stream) {
  const ace_status st = grouped_desc(d);
  if (st != ACE_OK) return st;
  const size_t es = elem_bytes(d->dtype), S = d->S, M = d->M, K = d->K, W = static_cast<size_t>(d->N) * M * K * es;
  const size_t xb = S * K * es, yb = S * M * es;
  const bool gw = way == Way::kGradW;
  if (S == 0 && !gw) return ACE_OK;
  if (!usable(offsets, 4) || !usable(out, 16)) return ACE_ERR_INVALID_ARG;
  if (S > 0 && (!usable(rows, 16) || !usable(other, 16))) return ACE_ERR_INVALID_ARG;
  const Span o{out, gw ? W : way == Way::kGradX ? xb : yb};
  const Span in[] = {{rows, way == Way::kForward ? xb : yb}, {other, gw ? xb : W}, {offsets, (d->N + 1u) * size_t{4}}};
  for (const Span &s : in)
    if (overlap(o, s)) return ACE_ERR_INVALID_ARG;
  const size_t need = grouped_bytes(*d, way);
  if (need > 0 && (!usable(workspace, 256) || workspace_bytes < need)) return ACE_ERR_WORKSPACE;
  ace::GroupedArgs g = grouped_args(*d);
  g.rows = rows;
  g.other = other;
  g.out = out;
  g.offsets = offsets;
  g.part = static_cast<float *>(workspace);
  const bool bf16 = d->dtype == ACE_BF16;
  hipStream_t s = static_cast<hipStream_t>(stream);
  return status_of(gw ? ace::launch_grouped_weights(g, bf16, s)
                      : ace::launch_grouped_rows(g, way == Way::kGradX, bf16, s));
}

ace_status norm_desc(const ace_norm_desc *d) {
  if (!d) return ACE_ERR_INVALID_ARG;
  if (d->T < 0 || d->d <= 0 || !is_dtype(d->dtype) || d->gate_kind < ACE_GATE_NONE || d->gate_kind > ACE_GATE_FULL)
    return ACE_ERR_INVALID_ARG;
  if (!std::isfinite(d->res_scale) || !std::isfinite(d->branch_scale) || !std::isfinite(d->eps) || !(d->eps > 0.f))
    return ACE_ERR_INVALID_ARG;
  if (d->T > kMaxRows || d->d > kMaxNormWidth || bad_width(d->d, d->dtype)) return ACE_ERR_UNSUPPORTED;
  return ACE_OK;
}

// inputs that both directions share
ace_status norm_inputs(const ace_norm_desc &d, const ace_norm_inputs &in) {
  if (!in.y && (in.w_post || d.gate_kind != ACE_GATE_NONE || d.res_scale != 1.f)) return ACE_ERR_INVALID_ARG;
  if (!in.y && !in.w_pre) return ACE_ERR_INVALID_ARG;
  if ((d.gate_kind != ACE_GATE_NONE) != (in.gate != nullptr)) return ACE_ERR_INVALID_ARG;
  for (const void *p : {in.h, in.y, in.w_post, in.w_pre})
    if (p && !usable(p, 16)) return ACE_ERR_INVALID_ARG;
  if (in.gate && !usable(in.gate, d.gate_kind == ACE_GATE_TOKEN ? elem_bytes(d.dtype) : 16)) return ACE_ERR_INVALID_ARG;
  return ACE_OK;
}

ace::NormArgs norm_args(const ace_norm_desc &d, const ace_norm_inputs &in) {
  ace::NormArgs a{};
  a.h = in.h;
  a.y = in.y;
  a.w_post = in.w_post;
  a.w_pre = in.w_pre;
  a.gate = in.gate;
  a.gate_kind = d.gate_kind;
  a.T = d.T;
  a.d = d.d;
  a.res_scale = d.res_scale;
  a.branch_scale = d.branch_scale;
  a.eps = d.eps;
  return a;
}

size_t gate_bytes(const ace_norm_desc &d) {
  const size_t es = elem_bytes(d.dtype), T = d.T, w = d.d;
  return es * (d.gate_kind == ACE_GATE_CHANNEL ? w : d.gate_kind == ACE_GATE_TOKEN ? T : d.gate_kind == ACE_GATE_FULL ? T * w : 0);
}

ace_status adapter_desc(const ace_adapter_desc *d) {
  if (!d) return ACE_ERR_INVALID_ARG;
  if (d->S < 0 || d->R < 0 || d->L <= 0 || d->rank <= 0 || d->d_in <= 0 || d->d_out <= 0 || !is_dtype(d->dtype))
    return ACE_ERR_INVALID_ARG;
  if (d->S > kMaxRows || d->R > kMaxGroups || d->rank > kMaxRank || d->d_in > kMaxWidth || d->d_out > kMaxWidth ||
      bad_width(d->rank, d->dtype) || bad_width(d->d_in, d->dtype) || bad_width(d->d_out, d->dtype))
    return ACE_ERR_UNSUPPORTED;
  return ACE_OK;
}

// A result may lie exactly on an input of the same rows (each thread reads its elements of a
// row before it writes them); any other overlap is refused.
bool bad_alias(const Span &out, const Span &in, bool may_equal) {
  return overlap(out, in) && !(may_equal && out.p == in.p && out.bytes == in.bytes);
}

}  // namespace

extern "C" {

size_t ace_grouped_workspace_size(const ace_grouped_desc *desc, int way) {
  if (grouped_desc(desc) != ACE_OK || way < ACE_GROUPED_FORWARD || way > ACE_GROUPED_GRAD_W) return 0;
  return grouped_bytes(*desc, static_cast<Way>(way));
}

ace_status ace_grouped_matmul(const ace_grouped_desc *desc, const void *x, const void *w, const int32_t *offsets,
                              void *y, void *workspace, size_t workspace_bytes, void *stream) {
  return grouped(desc, Way::kForward, x, w, offsets, y, workspace, workspace_bytes, stream);
}

ace_status ace_grouped_matmul_grad_x(const ace_grouped_desc *desc, const void *dy, const void *w,
                                     const int32_t *offsets, void *dx, void *workspace, size_t workspace_bytes,
                                     void *stream) {
  return grouped(desc, Way::kGradX, dy, w, offsets, dx, workspace, workspace_bytes, stream);
}

ace_status ace_grouped_matmul_grad_w(const ace_grouped_desc *desc, const void *dy, const void *x,
                                     const int32_t *offsets, void *dw, void *workspace, size_t workspace_bytes,
                                     void *stream) {
  return grouped(desc, Way::kGradW, dy, x, offsets, dw, workspace, workspace_bytes, stream);
}

ace_status ace_block_norm(const ace_norm_desc *desc, const ace_norm_inputs *in, void *h_out, void *n_out,
                          void *stream) {
  if (!in) return ACE_ERR_INVALID_ARG;
  ace_status st = norm_desc(desc);
  if (st != ACE_OK) return st;
  const ace_norm_desc &d = *desc;
  if (d.T == 0) return ACE_OK;
  st = norm_inputs(d, *in);
  if (st != ACE_OK) return st;
  if (!in->h || (in->y && !usable(h_out, 16)) || (in->w_pre && !usable(n_out, 16))) return ACE_ERR_INVALID_ARG;
  const size_t es = elem_bytes(d.dtype), rows = es * d.T * d.d, vec = es * d.d;
  const Span ho{in->y ? h_out : nullptr, rows}, no{in->w_pre ? n_out : nullptr, rows};
  if (overlap(ho, no)) return ACE_ERR_INVALID_ARG;
  for (const Span &o : {ho, no})
    if (bad_alias(o, {in->h, rows}, true) || bad_alias(o, {in->y, rows}, true) || bad_alias(o, {in->w_post, vec}, false) ||
        bad_alias(o, {in->w_pre, vec}, false) || bad_alias(o, {in->gate, gate_bytes(d)}, false))
      return ACE_ERR_INVALID_ARG;
  ace::NormArgs a = norm_args(d, *in);
  a.out_h = h_out;
  a.out_n = n_out;
  return status_of(ace::launch_block_norm(a, d.dtype == ACE_BF16, static_cast<hipStream_t>(stream)));
}

size_t ace_block_norm_grad_workspace_size(const ace_norm_desc *desc) {
  if (norm_desc(desc) != ACE_OK) return 0;
  return static_cast<size_t>(ace::block_norm_grad_blocks(desc->T, desc->d, desc->dtype == ACE_BF16)) * desc->d * 3 * sizeof(float);
}

ace_status ace_block_norm_grad(const ace_norm_desc *desc, const ace_norm_inputs *in, const void *dh, const void *dn,
                               const ace_norm_grads *out, void *workspace, size_t workspace_bytes, void *stream) {
  if (!in || !out) return ACE_ERR_INVALID_ARG;
  ace_status st = norm_desc(desc);
  if (st != ACE_OK) return st;
  const ace_norm_desc &d = *desc;
  // a gradient for each of the operands there is, no other; dn exactly where there is a pre-norm
  if ((out->w_post != nullptr) != (in->w_post != nullptr) || (out->w_pre != nullptr) != (in->w_pre != nullptr) ||
      (d.gate_kind == ACE_GATE_CHANNEL && !out->gate))
    return ACE_ERR_INVALID_ARG;
  if (d.T > 0) {
    st = norm_inputs(d, *in);
    if (st != ACE_OK) return st;
    if (!usable(out->h, 16) || (in->y != nullptr) != (out->y != nullptr) || (out->gate != nullptr) != (in->gate != nullptr))
      return ACE_ERR_INVALID_ARG;
    if ((dn != nullptr) != (in->w_pre != nullptr) || (!dh && !dn) || (in->w_pre && !in->h)) return ACE_ERR_INVALID_ARG;
  }
  for (const void *p : {dh, dn, static_cast<const void *>(out->y), static_cast<const void *>(out->w_post),
                        static_cast<const void *>(out->w_pre)})
    if (p && !usable(p, 16)) return ACE_ERR_INVALID_ARG;
  if (out->gate && !usable(out->gate, d.gate_kind == ACE_GATE_TOKEN ? elem_bytes(d.dtype) : 16)) return ACE_ERR_INVALID_ARG;
  const size_t es = elem_bytes(d.dtype), rows = es * d.T * d.d, vec = es * d.d, gate = gate_bytes(d);
  const Span outs[] = {{out->h, rows}, {in->y ? out->y : nullptr, rows}, {out->w_post, vec}, {out->w_pre, vec}, {out->gate, gate}};
  const Span ins[] = {{dh, rows}, {dn, rows}, {in->h, rows}, {in->y, rows}, {in->w_post, vec}, {in->w_pre, vec}, {in->gate, gate}};
  for (int i = 0; i < 5; ++i) {
    for (int j = 0; j < 7; ++j)
      if (bad_alias(outs[i], ins[j], i < 2 && j < 4)) return ACE_ERR_INVALID_ARG;
    for (int j = 0; j < i; ++j)
      if (overlap(outs[i], outs[j])) return ACE_ERR_INVALID_ARG;
  }
  if (!usable(workspace, 256) || workspace_bytes < ace_block_norm_grad_workspace_size(desc)) return ACE_ERR_WORKSPACE;
  ace::NormArgs a = norm_args(d, *in);
  a.dh = dh;
  a.dn = dn;
  a.g_h = out->h;
  a.g_y = out->y;
  a.g_post = out->w_post;
  a.g_pre = out->w_pre;
  a.g_gate = out->gate;
  a.part = static_cast<float *>(workspace);
  a.blocks = ace::block_norm_grad_blocks(d.T, d.d, d.dtype == ACE_BF16);
  return status_of(ace::launch_block_norm_grad(a, d.dtype == ACE_BF16, static_cast<hipStream_t>(stream)));
}

size_t ace_adapter_workspace_size(const ace_adapter_desc *desc) {
  if (adapter_desc(desc) != ACE_OK || desc->S == 0) return 0;
  return static_cast<size_t>(ace::adapter_splits(desc->S, desc->R, desc->rank, desc->d_in, desc->d_out, desc->dtype == ACE_BF16)) * desc->S *
         desc->rank * sizeof(float);
}

ace_status ace_adapter_add(const ace_adapter_desc *desc, const void *base, const void *x, const void *a, const void *b,
                           const float *scale, const int32_t *offsets, const int32_t *adapter, void *out,
                           void *workspace, size_t workspace_bytes, void *stream) {
  const ace_status st = adapter_desc(desc);
  if (st != ACE_OK) return st;
  const ace_adapter_desc &d = *desc;
  if (d.S == 0) return ACE_OK;
  for (const void *p : {base, x, a, b, static_cast<const void *>(out)})
    if (!usable(p, 16)) return ACE_ERR_INVALID_ARG;
  if (!usable(offsets, 4) || (d.R > 0 && !usable(adapter, 4)) || (scale && !usable(scale, 4))) return ACE_ERR_INVALID_ARG;
  const size_t es = elem_bytes(d.dtype), S = d.S, L = d.L, r = d.rank;
  const Span o{out, es * S * d.d_out};
  if (bad_alias(o, {base, o.bytes}, true)) return ACE_ERR_INVALID_ARG;
  const Span ins[] = {{x, es * S * d.d_in}, {a, es * L * r * d.d_in}, {b, es * L * d.d_out * r}, {scale, 4 * L},
                      {offsets, 4 * (d.R + size_t{1})}, {adapter, 4 * static_cast<size_t>(d.R)}};
  for (const Span &s : ins)
    if (overlap(o, s)) return ACE_ERR_INVALID_ARG;
  const size_t need = ace_adapter_workspace_size(desc);
  if (need > 0 && (!usable(workspace, 256) || workspace_bytes < need)) return ACE_ERR_WORKSPACE;
  ace::AdapterArgs p{};
  p.base = base;
  p.x = x;
  p.a = a;
  p.b = b;
  p.scale = scale;
  p.offsets = offsets;
  p.adapter = adapter;
  p.out = out;
  p.v = static_cast<float *>(workspace);
  p.S = d.S;
  p.R = d.R;
  p.L = d.L;
  p.r = d.rank;
  p.din = d.d_in;
  p.dout = d.d_out;
  p.splits = ace::adapter_splits(d.S, d.R, d.rank, d.d_in, d.d_out, d.dtype == ACE_BF16);
  return status_of(ace::launch_adapter(p, d.dtype == ACE_BF16, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
