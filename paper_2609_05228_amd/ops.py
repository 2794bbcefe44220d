"""torch-facing wrappers of the operators around the layer: matrix products grouped by
expert with ragged sizes, the experts' gated feed-forward block, weights in microscaled 4-bit
floating point for both, the norms before and after a block fused with its gate and residual
scale, and low-rank adapters of many requests at once.

Like `moe_forward` they marshal device tensors into the C ABI of libace.so and enqueue on the
current HIP stream of the tensors' device.  They record no autograd graph: the gradients are
entry points of their own (`grouped_matmul_grad_x`, `grouped_matmul_grad_w`, `grouped_gated_grad`, `block_norm_grad`),
and inputs that require a gradient are refused while autograd is on, inputs with a forward-mode
tangent always.  Workspaces come from torch's allocator with every call, so captured graphs share
none.
"""
from __future__ import annotations

from typing import NamedTuple

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
    try:
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
                             "grouped_matmul, grouped_gated and block_norm: the *_grad functions; adapter_add has none, nor do "
                             "weights in 4 bits)")
    except (AttributeError, TypeError):  # caught, not asked for each tensor: that takes as long as the other checks
        for name, t, _, _ in named:
            if not isinstance(t, torch.Tensor):
                raise ValueError(f"{name} must be a tensor") from None
        raise
    if dev.type != "cuda":
        raise ValueError(f"the tensors are on {dev}: a GPU is needed")


def _dtype_of(name, t, dims):
    if not isinstance(t, torch.Tensor) or t.dim() != dims:
        raise ValueError(f"{name} must be a tensor of {dims} dimensions")
    if t.dtype not in _DT:
        raise ValueError(f"{name}: unsupported dtype {t.dtype}")
    return t.dtype


def _pair(name, v, what):
    """The two that v, asked for as `what`, is made of."""
    try:
        first, second = v
    except (TypeError, ValueError):
        raise ValueError(f"{name}: {what} is needed") from None
    return first, second


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


class Mx4(NamedTuple):
    """Numbers [..., K] in microscaled 4-bit floating point, blocks of 32 along the last dimension (K a multiple of 32):

    codes   [..., K / 2] uint8, two numbers a byte, the even one in the low half: a sign (8) and 0, .5, 1, 1.5, 2, 3, 4, 6
    scales  [..., 4 ceil(K / 128)] uint8: 2^(byte - 127) for each block, 255: the block stands for NaN; the bytes
            from K / 32 on mean nothing"""
    codes: torch.Tensor
    scales: torch.Tensor


_BLOCK = 32


def _scale_bytes(K):
    return (K + 127) // 128 * 4


def _mx4_of(name, q, dims):
    """K of an Mx4 with `dims` dimensions (None: any)."""
    if not isinstance(q, Mx4):
        raise ValueError(f"{name} must be an Mx4")
    codes = q.codes
    if not (isinstance(codes, torch.Tensor) and isinstance(q.scales, torch.Tensor)):
        raise ValueError(f"{name} must hold tensors")
    if codes.dim() != dims if dims is not None else codes.dim() < 1:
        raise ValueError(f"{name} must hold tensors of {'1 dimension or more' if dims is None else f'{dims} dimensions'}")
    return 2 * codes.shape[-1]


# names of the tensors of an Mx4 argument, for `_check_all`
_PARTS = {n: (n + ".codes", n + ".scales") for n in ("x", "q", "w", "w_gate", "w_up")}


def _mx4_named(name, q, lead, K):
    """What `_check_all` has to find for an Mx4 of numbers [*lead, K]."""
    codes, scales = _PARTS[name]
    return ((codes, q.codes, (*lead, K // 2), torch.uint8), (scales, q.scales, (*lead, _scale_bytes(K)), torch.uint8))


def _whole_blocks(K):
    if K <= 0 or K % _BLOCK != 0:
        raise ValueError(f"the last dimension, {K}, is not a multiple of {_BLOCK}")


def mx4_quantize(x):
    """x [..., K] bf16 or fp32 in microscaled 4-bit floating point: per block of 32 a scale 2^e with e = floor(log2 of
    the largest magnitude) - 2, at least -127; each number over it to the nearest of 0, .5, 1, 1.5, 2, 3, 4, 6 with its sign (ties
    to the even code, above 6 to 6).  A block that holds a NaN or an infinity stands for NaN.  Returns an `Mx4`."""
    _need(isinstance(x, torch.Tensor) and x.dim() >= 1, "x must be a tensor of 1 dimension or more")
    dtype, K = _dtype_of("x", x, x.dim()), x.shape[-1]
    _whole_blocks(K)
    dev = x.device
    _sizes(K)
    _check_all(dev, dtype, [("x", x, x.shape, None)])
    lead = x.shape[:-1]
    q = Mx4(x.new_empty((*lead, K // 2), dtype=torch.uint8), x.new_empty((*lead, _scale_bytes(K)), dtype=torch.uint8))
    _enqueue(dev, _lib.lib().ace_mx4_quantize, x.numel() // K, K, _DT[dtype], x.data_ptr(), q.codes.data_ptr(),
             q.scales.data_ptr())
    return q


def mx4_dequantize(q, dtype=torch.bfloat16):
    """The numbers [..., K] that an `Mx4` stands for, as bf16 or fp32: exactly, infinite from 2^128 on, which scales of
    253 and 254 reach."""
    K = _mx4_of("q", q, None)
    if dtype not in _DT:
        raise ValueError(f"unsupported dtype {dtype}")
    _whole_blocks(K)
    dev, lead = q.codes.device, q.codes.shape[:-1]
    _sizes(K)
    _check_all(dev, torch.uint8, _mx4_named("q", q, lead, K))
    out = q.codes.new_empty((*lead, K), dtype=dtype)
    _enqueue(dev, _lib.lib().ace_mx4_dequantize, out.numel() // K, K, _DT[dtype], q.codes.data_ptr(), q.scales.data_ptr(),
             out.data_ptr())
    return out


def _mx4_call(x, weights, offsets, out, act, names):
    """y = w x, or with two weights the gated block, on weights in 4 bits."""
    K = _mx4_of(names[0], weights[0], 3)
    N, M = weights[0].codes.shape[:2]
    if isinstance(x, Mx4):
        _mx4_of("x", x, 2)
        lead, scales = x
        S = lead.shape[0]
        named = [*_mx4_named("x", x, (S,), K)]
    else:
        if _dtype_of("x", x, 2) is not torch.bfloat16:
            raise ValueError("x: bf16 or Mx4 with weights in 4 bits")
        S, lead, scales = x.shape[0], x, None
        named = [("x", x, (S, K), torch.bfloat16)]
    _whole_blocks(K)
    size = _sizes(S, N, M, K)
    for name, w in zip(names, weights):
        if w is not weights[0]:
            _mx4_of(name, w, 3)
        named += _mx4_named(name, w, (N, M), K)
    named.append(("offsets", offsets, (N + 1,), torch.int32))
    flags = 0
    if out is not None:
        named.append(("out", out, (S, M), torch.bfloat16))
    dev = lead.device
    _check_all(dev, torch.bfloat16, named)
    if out is None:
        out = torch.empty((S, M), dtype=torch.bfloat16, device=dev)
        flags = _lib.ACE_ZERO_REST
    desc = _lib.Mx4Desc(*size, act, flags)
    lib = _lib.lib()
    gated = len(weights) == 2
    n = lib.ace_grouped_mx4_workspace_size(desc, gated)
    ws = _scratch(n, dev)
    w = [_lib.Mx4Ptr(q.codes.data_ptr(), q.scales.data_ptr()) for q in weights]
    _enqueue(dev, lib.ace_grouped_gated_mx4 if gated else lib.ace_grouped_matmul_mx4, desc, lead.data_ptr(), _ptr(scales), *w,
             offsets.data_ptr(), out.data_ptr(), _ptr(ws), n)
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
    K and M are multiples of 8 (fp32: 4).  Returns y [S, M].
    w may be an `Mx4` of [N, M, K]; then x is bf16 or an `Mx4` of [S, K], y and out are bf16, and there is no gradient.
    bf16 rows meet the weights as `mx4_dequantize` gives them."""
    if isinstance(w, Mx4):
        return _mx4_call(x, (w,), offsets, out, 0, ("w",))
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


def _activation(name):
    if not isinstance(name, str) or name not in _lib.ACTIVATIONS:
        raise ValueError(f"activation {name!r} is none of {', '.join(_lib.ACTIVATIONS)}")
    return _lib.ACTIVATIONS[name]


def _scratch(n, dev):
    return torch.empty(n, dtype=torch.uint8, device=dev) if n else None


def _ptr(t):
    return None if t is None else t.data_ptr()


def grouped_gated(x, w_gate, w_up, offsets, *, activation="silu", keep=False, out=None):
    """The gated feed-forward block of the experts: a[r] = act(g[r]) * u[r] with g[r] = w_gate[e] x[r] and
    u[r] = w_up[e] x[r] for the rows r of group e, in one kernel (where a few tiles have a long reduction, in parts and a
    second launch that adds them up).

    x        [S, K] bf16 or fp32 device tensor, rows in group order
    w_gate, w_up  [N, M, K] weights of the groups (nn.Linear layout)
    offsets  [N + 1] int32: group e owns rows offsets[e] .. offsets[e + 1] - 1, ascending
             (the `offsets` of `moe_forward`'s plan; [0, S] for one block that takes every row)
    activation  "silu", or "gelu" with the normal distribution's integral (not its tanh approximation)
    keep     also return g and u, for `grouped_gated_grad`
    out      None, or tensors in the shape of the result (with keep (a, (g, u))).  Rows of no group stay as they are in them; a fresh
             result holds zeros there.
    K and M are multiples of 8 (fp32: 4).  Returns a [S, M], with keep (a, (g, u)).
    Both weights may be an `Mx4` of [N, M, K]; then x is bf16 or an `Mx4` of [S, K] (see `grouped_matmul`), a and out are
    bf16, and there is no gradient, so nothing to keep."""
    if isinstance(w_gate, Mx4) or isinstance(w_up, Mx4):
        _need(not keep, "keep: weights in 4 bits have no gradient")
        return _mx4_call(x, (w_gate, w_up), offsets, out, _activation(activation), ("w_gate", "w_up"))
    dtype = _dtype_of("x", x, 2)
    _dtype_of("w_gate", w_gate, 3)
    act = _activation(activation)
    N, M, K = w_gate.shape
    S = x.shape[0]
    dev, size = x.device, _sizes(S, N, M, K)
    named = [("x", x, (S, K), None), ("w_gate", w_gate, (N, M, K), None), ("w_up", w_up, (N, M, K), None),
             ("offsets", offsets, (N + 1,), torch.int32)]
    flags = 0
    a, g, u = out, None, None
    if out is not None:
        if keep:
            a, gu = _pair("out", out, "(a, (g, u))")
            g, u = _pair("out", gu, "(a, (g, u))")
            named += [("out's g", g, (S, M), None), ("out's u", u, (S, M), None)]
        named.append(("out", a, (S, M), None))
    _check_all(dev, dtype, named)
    if out is None:
        a, g, u = (torch.empty((S, M), dtype=dtype, device=dev) if i == 0 or keep else None for i in range(3))
        flags = _lib.ACE_ZERO_REST
    desc = _lib.GatedDesc(*size, _DT[dtype], act, flags)
    lib = _lib.lib()
    n = lib.ace_grouped_gated_workspace_size(desc)
    ws = _scratch(n, dev)
    _enqueue(dev, lib.ace_grouped_gated, desc, x.data_ptr(), w_gate.data_ptr(), w_up.data_ptr(), offsets.data_ptr(),
             a.data_ptr(), _ptr(g), _ptr(u), _ptr(ws), n)
    return (a, (g, u)) if keep else a


def grouped_gated_grad(da, x, w_gate, w_up, offsets, *, kept=None, activation="silu", weights=True):
    """Gradients of `grouped_gated`.

    da       [S, M]: gradient of the result a
    x, w_gate, w_up, offsets, activation  as in the forward
    kept     the forward's (g, u), or None: both projections are computed again, which takes as long as the
             forward and no memory between the passes
    weights  False: the weights are frozen, only x's gradient is computed (x may be None with kept)
    Returns a dict of the gradients of x [S, K] (zeros in rows of no group) and, with weights, of w_gate and w_up
    [N, M, K] (zeros for an empty group).  The gradients of g and u are rounded to the tensors' type between the
    products; sums are fp32 in a fixed order."""
    dtype = _dtype_of("da", da, 2)
    _dtype_of("w_gate", w_gate, 3)
    act = _activation(activation)
    N, M, K = w_gate.shape
    S = da.shape[0]
    dev, size = da.device, _sizes(S, N, M, K)
    g, u = (None, None) if kept is None else _pair("kept", kept, "(g, u)")
    _need(x is not None or (kept is not None and not weights), "x is required with weights or without kept")
    named = [("da", da, (S, M), None), ("w_gate", w_gate, (N, M, K), None), ("w_up", w_up, (N, M, K), None),
             ("offsets", offsets, (N + 1,), torch.int32)]
    if x is not None:
        named.append(("x", x, (S, K), None))
    if kept is not None:
        named += [("kept's g", g, (S, M), None), ("kept's u", u, (S, M), None)]
    _check_all(dev, dtype, named)
    out = {"x": torch.empty((S, K), dtype=dtype, device=dev)}
    if weights:
        out["w_gate"], out["w_up"] = torch.empty_like(w_gate), torch.empty_like(w_up)
    desc = _lib.GatedDesc(*size, _DT[dtype], act, _lib.ACE_ZERO_REST)
    lib = _lib.lib()
    n = lib.ace_grouped_gated_grad_workspace_size(desc, kept is not None, weights)
    ws = _scratch(n, dev)
    _enqueue(dev, lib.ace_grouped_gated_grad, desc, da.data_ptr(), _ptr(x), w_gate.data_ptr(), w_up.data_ptr(),
             offsets.data_ptr(), _ptr(g), _ptr(u), out["x"].data_ptr(), _ptr(out.get("w_gate")), _ptr(out.get("w_up")),
             _ptr(ws), n)
    return out


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
