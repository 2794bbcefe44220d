"""torch-facing wrappers of the operators around the layer: matrix products grouped by
expert with ragged sizes, the norms before and after a block fused with its gate and residual
scale, and low-rank adapters of many requests at once.

Like `moe_forward` they marshal device tensors into the C ABI of libace.so and enqueue on the
current HIP stream of the tensors' device.  They record no autograd graph: the gradients are
entry points of their own (`grouped_matmul_grad_x`, `grouped_matmul_grad_w`, `block_norm_grad`),
and inputs that require a gradient are refused while autograd is on, inputs with a forward-mode
tangent always.  Workspaces come from torch's allocator with every call, so captured graphs share
none.
"""
from __future__ import annotations

import torch
from torch.autograd import forward_ad

from . import _lib
from .layer import _DT

# the raw handle of a device's current stream; torch.cuda.current_stream builds a Stream object around
# it, which costs a call more than its checks
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda index: torch.cuda.current_stream(index).cuda_stream)


def _need(ok, msg):
    if not ok:
        raise ValueError(msg)


def _check_all(dev, dtype, named):
    """(name, tensor, shape, dtype or None for the call's): shapes, types, layout, device."""
    grad = torch.is_grad_enabled()
    # asked for each tensor inside a forward-mode level only: that takes as long as the other checks
    if getattr(forward_ad, "_current_level", 0) >= 0:
        for name, t, _, _ in named:
            if forward_ad.unpack_dual(t).tangent is not None:
                raise ValueError(f"{name} has a forward-mode tangent, which the call would lose")
    for name, t, shape, dt in named:
        if (t.shape == shape and t.dtype is (dt or dtype) and t.device == dev and t.is_contiguous()
                and not (grad and t.requires_grad)):
            continue
        if t.shape != shape:
            raise ValueError(f"{name}: shape {tuple(t.shape)} != {tuple(shape)}")
        if t.dtype != (dt or dtype):
            raise ValueError(f"{name}: dtype {t.dtype} != {dt or dtype}")
        if not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous")
        if t.device != dev:
            raise ValueError(f"{name} is on {t.device}, expected {dev}")
        raise ValueError(f"{name} requires a gradient, and no graph is recorded: call under torch.no_grad() (gradients of "
                         "grouped_matmul and block_norm: the *_grad functions; adapter_add has none)")
    if dev.type != "cuda":
        raise ValueError(f"the tensors are on {dev}: a GPU is needed")


def _dtype_of(name, t, dims):
    if not isinstance(t, torch.Tensor) or t.dim() != dims:
        raise ValueError(f"{name} must be a tensor of {dims} dimensions")
    if t.dtype not in _DT:
        raise ValueError(f"{name}: unsupported dtype {t.dtype}")
    return t.dtype


def _sizes(*n):
    """The sizes as the library's 32-bit ones; more would be cut off on the way there."""
    for v in n:
        if v > 0x7fffffff:
            raise ValueError(f"a size of {v}: at most 2^31 - 1")
    return n


def _enqueue(dev, fn, *args):
    """fn(*args, stream) on the current stream of dev, with dev current."""
    index = dev.index
    if index == torch.cuda.current_device():
        st = fn(*args, _raw_stream(index))
    else:
        with torch.cuda.device(dev):
            st = fn(*args, _raw_stream(index))
    if st != _lib.ACE_OK:
        raise _lib.AceError(st, _lib.status_string(st))


def _grouped(way, rows, other, offsets, S, N, M, K, shape, names, shapes, out):
    dtype, dev = rows.dtype, rows.device
    size = _sizes(S, N, M, K)
    named = [(names[0], rows, shapes[0], None), (names[1], other, shapes[1], None),
             ("offsets", offsets, (N + 1,), torch.int32)]
    flags = 0
    if out is not None:
        named.append(("out", out, shape, None))
    _check_all(dev, dtype, named)
    if out is None:
        out = torch.empty(shape, dtype=dtype, device=dev)
        flags = _lib.ACE_ZERO_REST
    desc = _lib.GroupedDesc(*size, _DT[dtype], flags)
    lib = _lib.lib()
    n = lib.ace_grouped_workspace_size(desc, way)
    ws = torch.empty(n, dtype=torch.uint8, device=dev) if n else None
    fn = (lib.ace_grouped_matmul, lib.ace_grouped_matmul_grad_x, lib.ace_grouped_matmul_grad_w)[way]
    _enqueue(dev, fn, desc, rows.data_ptr(), other.data_ptr(), offsets.data_ptr(), out.data_ptr(),
             None if ws is None else ws.data_ptr(), n)
    return out


def _groups_of(offsets):
    _need(isinstance(offsets, torch.Tensor) and offsets.dim() == 1 and offsets.shape[0] >= 2,
          "offsets must hold at least one group: [N + 1] int32")
    return offsets.shape[0] - 1


def grouped_matmul(x, w, offsets, *, out=None):
    """Products grouped by expert: y[r] = w[e] x[r] for the rows r of group e.

    x        [S, K] bf16 or fp32 device tensor, rows in group order
    w        [N, M, K] weights of the groups (nn.Linear layout)
    offsets  [N + 1] int32: group e owns rows offsets[e] .. offsets[e + 1] - 1, ascending
             (the `offsets` of `moe_forward`'s plan)
    out      [S, M] or None.  Rows of no group stay as they are in `out`; a fresh result
             holds zeros there.
    K and M are multiples of 8 (fp32: 4).  Returns y [S, M]."""
    _dtype_of("x", x, 2)
    _dtype_of("w", w, 3)
    N, M, K = w.shape
    S = x.shape[0]
    return _grouped(_lib.GROUPED_FORWARD, x, w, offsets, S, N, M, K, (S, M), ("x", "w"), ((S, K), (N, M, K)),
                    out)


def grouped_matmul_grad_x(dy, w, offsets, *, out=None):
    """Gradient of `grouped_matmul` for its rows: dx[r] = w[e]^T dy[r].  dy [S, M]; the rest, and
    rows of no group, as there.  Returns dx [S, K]."""
    _dtype_of("dy", dy, 2)
    _dtype_of("w", w, 3)
    N, M, K = w.shape
    S = dy.shape[0]
    return _grouped(_lib.GROUPED_GRAD_X, dy, w, offsets, S, N, M, K, (S, K), ("dy", "w"),
                    ((S, M), (N, M, K)), out)


def grouped_matmul_grad_w(dy, x, offsets, *, out=None):
    """Gradient of `grouped_matmul` for its weights: dw[e] = sum of dy[r] x[r]^T over the rows of
    group e (zeros for an empty group).  dy [S, M], x [S, K], offsets [N + 1].  Returns dw [N, M, K]."""
    _dtype_of("dy", dy, 2)
    _dtype_of("x", x, 2)
    N = _groups_of(offsets)
    S, M = dy.shape
    K = x.shape[1]
    return _grouped(_lib.GROUPED_GRAD_W, dy, x, offsets, S, N, M, K, (N, M, K), ("dy", "x"),
                    ((S, M), (S, K)), out)


def _norm_call(lead, dtype, T, d, h, y, w_post, w_pre, gate, res_scale, branch_scale, eps, named):
    """Check a block_norm call's tensors, `named` among them; (desc, inputs)."""
    rows, vec, kind, size = (T, d), (d,), 0, _sizes(T, d)
    if y is not None:
        named.append(("y", y, rows, None))
    elif w_post is not None or gate is not None or res_scale != 1.0:
        raise ValueError("w_post, gate and res_scale need y")
    elif w_pre is None:
        raise ValueError("y or w_pre is required")
    if w_post is not None:
        named.append(("w_post", w_post, vec, None))
    if w_pre is not None:
        named.append(("w_pre", w_pre, vec, None))
    if gate is not None:
        shape = tuple(gate.shape)
        kind = 1 if shape == vec else 2 if shape == (T, 1) else 3 if shape == rows else 0
        if kind == 0:
            raise ValueError(f"gate: shape {shape} is none of [d], [T, 1], [T, d]")
        named.append(("gate", gate, shape, None))
    _check_all(lead.device, dtype, named)
    return (_lib.NormDesc(*size, _DT[dtype], kind, res_scale, branch_scale, eps),
            _lib.NormInputs(h if h is None else h.data_ptr(), y if y is None else y.data_ptr(),
                            w_post if w_post is None else w_post.data_ptr(),
                            w_pre if w_pre is None else w_pre.data_ptr(), gate if gate is None else gate.data_ptr()))


def block_norm(h, y=None, *, w_post=None, w_pre=None, gate=None, res_scale=1.0, branch_scale=1.0, eps=1e-6, out=None):
    """The norms after one block and before the next, with the block's gate and the residual scale:

        u = y / rms(y) * w_post                         (y itself without w_post)
        h' = res_scale * h + branch_scale * gate * u
        n = h' / rms(h') * w_pre                        (not without w_pre)

    h        [T, d] bf16 or fp32: the residual stream
    y        [T, d]: the block's output (`moe_forward`'s y); None for the norm before the first block
    w_post, w_pre  [d] or None
    gate     [d], [T, 1] or [T, d], or None
    out      dict that may hold "h" and "n" [T, d] (h or y themselves are fine; "h" only with y)
    d is a multiple of 8 (fp32: 4), at most 16384; eps > 0.  Returns dict(h=h'[, n]); without y, h' is h."""
    dtype = _dtype_of("h", h, 2)
    T, d = h.shape
    named = [("h", h, h.shape, None)]
    if out is None:
        out = {}
    else:
        out = dict(out)
        if y is None and out.get("h", h).data_ptr() != h.data_ptr():
            raise ValueError("out['h'] needs y: without it h' is h itself")
        named += [(f"out['{k}']", out[k], h.shape, None) for k in ("h", "n") if k in out]
    desc, inp = _norm_call(h, dtype, T, d, h, y, w_post, w_pre, gate, res_scale, branch_scale, eps, named)
    if y is None:
        out["h"] = h
    elif "h" not in out:
        out["h"] = torch.empty_like(h)
    if w_pre is None:
        out.pop("n", None)
    elif "n" not in out:
        out["n"] = torch.empty_like(h)
    _enqueue(h.device, _lib.lib().ace_block_norm, desc, inp, out["h"].data_ptr() if y is not None else None,
             out["n"].data_ptr() if w_pre is not None else None)
    return out


def block_norm_grad(dh, dn, h, y=None, *, w_post=None, w_pre=None, gate=None, res_scale=1.0, branch_scale=1.0,
                    eps=1e-6):
    """Gradients of `block_norm`.

    dh, dn   [T, d]: gradients of the results h' and n (dh None: zero; dn exactly with w_pre)
    h        [T, d]: the forward's result h' (without y: its h); may be None without w_pre
    y, weights, gate and scales as in the forward
    Returns a dict of the gradients of h, and of y, w_post, w_pre and gate where there is one, in their
    shapes and type.  Sums over the rows are fp32 in a fixed order."""
    lead = dh if dh is not None else dn
    _need(lead is not None, "dh or dn is required")
    dtype = _dtype_of("dh" if dh is not None else "dn", lead, 2)
    T, d = lead.shape
    _need((dn is None) == (w_pre is None), "dn and w_pre go together")
    _need(h is not None or w_pre is None, "h is required with w_pre")
    named = [(n, t, lead.shape, None) for n, t in (("dh", dh), ("dn", dn), ("h", h)) if t is not None]
    desc, inp = _norm_call(lead, dtype, T, d, h, y, w_post, w_pre, gate, res_scale, branch_scale, eps, named)
    dev = lead.device
    out = {"h": torch.empty_like(lead)}
    for name, t in (("y", y), ("w_post", w_post), ("w_pre", w_pre), ("gate", gate)):
        if t is not None:
            out[name] = torch.empty_like(t)
    grads = _lib.NormGrads(**{n: t.data_ptr() for n, t in out.items()})
    lib = _lib.lib()
    n = lib.ace_block_norm_grad_workspace_size(desc)
    ws = torch.empty(max(n, 256), dtype=torch.uint8, device=dev)
    _enqueue(dev, lib.ace_block_norm_grad, desc, inp, None if dh is None else dh.data_ptr(),
             None if dn is None else dn.data_ptr(), grads, ws.data_ptr(), ws.numel())
    return out


def adapter_add(base, x, a, b, offsets, adapter, *, scale=None, out=None):
    """Low-rank adapters of many requests beside a shared projection:
    out[r] = base[r] + scale[l] * b[l] (a[l] x[r]), l = adapter[i] for the rows r of request i.

    base     [S, d_out] bf16 or fp32: the shared projection's output
    x        [S, d_in]: its input
    a, b     [L, rank, d_in], [L, d_out, rank]: the adapters (lower ranks padded with zero rows of a)
    offsets  [R + 1] int32: request i owns rows offsets[i] .. offsets[i + 1] - 1, ascending
    adapter  [R] int32: adapter of each request, -1 for none
    scale    [L] fp32 or None
    out      [S, d_out] or None; `base` itself adds in place
    Rows without an adapter, and rows of no request, are base's.  d_in, d_out and the rank (at most 128) are
    multiples of 8 (fp32: 4).  For serving: it has no gradient.  Returns out."""
    dtype = _dtype_of("x", x, 2)
    _dtype_of("a", a, 3)
    _dtype_of("b", b, 3)
    S, d_in = x.shape
    L, rank, _ = a.shape
    d_out = b.shape[1]
    R = (_groups_of(offsets) if isinstance(offsets, torch.Tensor) and offsets.shape != (1,) else 0)
    dev, size = x.device, _sizes(S, R, L, rank, d_in, d_out)
    named = [("x", x, (S, d_in), None), ("base", base, (S, d_out), None), ("a", a, (L, rank, d_in), None),
             ("b", b, (L, d_out, rank), None), ("offsets", offsets, (R + 1,), torch.int32),
             ("adapter", adapter, (R,), torch.int32)]
    if scale is not None:
        named.append(("scale", scale, (L,), torch.float32))
    if out is not None:
        named.append(("out", out, (S, d_out), None))
    _check_all(dev, dtype, named)
    if out is None:
        out = torch.empty_like(base)
    desc = _lib.AdapterDesc(*size, _DT[dtype])
    lib = _lib.lib()
    n = lib.ace_adapter_workspace_size(desc)
    ws = torch.empty(n, dtype=torch.uint8, device=dev) if n else None
    _enqueue(dev, lib.ace_adapter_add, desc, base.data_ptr(), x.data_ptr(), a.data_ptr(), b.data_ptr(),
             None if scale is None else scale.data_ptr(), offsets.data_ptr(), adapter.data_ptr(), out.data_ptr(),
             None if ws is None else ws.data_ptr(), n)
    return out
