"""Refusals of the operators around the layer, on the CPU: the C ABI returns before any launch,
the wrappers raise before they call it."""
import ctypes
import inspect

import pytest
import torch

import paper_2609_05228_amd as ace
from paper_2609_05228_amd import _lib

# aligned, never dereferenced, far apart: every call below returns before any launch
P = [0x100000000000 + (i << 40) for i in range(16)]
BIG = (1 << 31) - 1
BAD, UNS, WSP = _lib.ACE_ERR_INVALID_ARG, _lib.ACE_ERR_UNSUPPORTED, _lib.ACE_ERR_WORKSPACE


def _grouped(fn="ace_grouped_matmul", rows=P[0], other=P[1], offsets=P[2], out=P[3], null=False, ws=P[15], ws_bytes=1 << 40,
             **kw):
    d = dict(S=64, N=4, M=64, K=64, dtype=_lib.ACE_BF16, flags=0)
    d.update(kw)
    desc = None if null else ctypes.byref(_lib.GroupedDesc(*[d[n] for n in ("S", "N", "M", "K", "dtype", "flags")]))
    return getattr(ace.lib(), fn)(desc, rows, other, offsets, out, ws, ws_bytes, None)


FNS = ("ace_grouped_matmul", "ace_grouped_matmul_grad_x", "ace_grouped_matmul_grad_w")


@pytest.mark.parametrize("fn", FNS)
def test_grouped_refusals(fn):
    for kw in (dict(S=-1), dict(N=0), dict(M=0), dict(K=-8), dict(dtype=7), dict(flags=2), dict(null=True), dict(rows=0),
               dict(other=0), dict(offsets=0), dict(out=0), dict(rows=P[0] + 8), dict(out=P[3] + 4), dict(offsets=P[2] + 2),
               dict(out=P[0]), dict(out=P[1] + 64), dict(out=P[2])):
        assert _grouped(fn, **kw) == BAD, kw
    for kw in (dict(S=BIG), dict(N=4097), dict(M=65544), dict(K=65544), dict(M=12), dict(K=4), dict(dtype=_lib.ACE_F32, K=6)):
        assert _grouped(fn, **kw) == UNS, kw


def test_grouped_workspace():
    """Few tiles with a long reduction take partial sums; enough tiles none."""
    size = ace.lib().ace_grouped_workspace_size
    for way, fn in enumerate(FNS):
        few = dict(S=64, N=2, M=4096, K=128) if way == 1 else dict(S=64, N=2, M=128, K=4096) if way == 0 else dict(
            S=40000, N=2, M=128, K=128)
        n = size(_lib.GroupedDesc(*few.values(), _lib.ACE_BF16, 0), way)
        assert n > 0 and n % 4 == 0
        for kw in (dict(ws=0), dict(ws=P[15] + 16), dict(ws_bytes=n - 1)):
            assert _grouped(fn, **few, **kw) == WSP, kw
        many = _lib.GroupedDesc(32768, 128, 768, 2048, _lib.ACE_BF16, 0)
        # the weights' gradient keeps room for the parts of groups of more than four times the mean
        assert size(many, way) == 0 if way < 2 else 0 < size(many, way) <= 2 * 128 * 768 * 2048
        assert size(_lib.GroupedDesc(64, 0, 64, 64, _lib.ACE_BF16, 0), way) == 0
    assert size(many, 3) == 0 and size(many, -1) == 0


def test_grouped_empty_rows():
    assert _grouped(FNS[0], S=0, rows=0, out=0) == _lib.ACE_OK
    assert _grouped(FNS[1], S=0, rows=0, out=0) == _lib.ACE_OK
    assert _grouped(FNS[2], S=0, rows=0, other=0, out=0) == BAD  # it has zeros to write


def _norm_desc(**kw):
    d = dict(T=4, d=64, dtype=_lib.ACE_BF16, gate_kind=0, res_scale=1.0, branch_scale=1.0, eps=1e-6)
    d.update(kw)
    return _lib.NormDesc(*d.values())


def _norm(inp=None, ho=P[5], no=P[6], **kw):
    i = dict(h=P[0], y=P[1], w_post=P[2], w_pre=P[3], gate=None)
    i.update(inp or {})
    return ace.lib().ace_block_norm(ctypes.byref(_norm_desc(**kw)), ctypes.byref(_lib.NormInputs(*i.values())), ho, no, None)


def test_block_norm_refusals():
    inf, nan = float("inf"), float("nan")
    for kw in (dict(T=-1), dict(d=0), dict(dtype=9), dict(gate_kind=4), dict(gate_kind=-1), dict(res_scale=inf),
               dict(branch_scale=nan), dict(eps=0.0), dict(eps=-1e-6), dict(eps=nan), dict(eps=inf), dict(gate_kind=1),
               dict(inp=dict(gate=P[4])), dict(inp=dict(h=None)), dict(inp=dict(y=None)),
               dict(inp=dict(y=None, w_post=None, w_pre=None)), dict(inp=dict(y=None, w_post=None), res_scale=0.5),
               dict(ho=None), dict(no=None), dict(ho=P[5] + 2), dict(inp=dict(w_pre=P[3] + 8)), dict(no=P[5]),
               dict(ho=P[0] + 16), dict(no=P[1] + 16), dict(ho=P[2]), dict(no=P[3]),
               dict(inp=dict(gate=P[4]), gate_kind=3, ho=P[4])):
        assert _norm(**kw) == BAD, kw
    for kw in (dict(T=BIG, inp=dict(y=P[12]), ho=P[13], no=P[14]), dict(d=16392), dict(d=60), dict(d=6, dtype=_lib.ACE_F32)):
        assert _norm(**kw) == UNS, kw
    assert _norm(T=0, inp=dict(h=None, y=None), ho=None, no=None) == _lib.ACE_OK


def _norm_grad(inp=None, out=None, dh=P[7], dn=P[8], ws=P[15], need=0, **kw):
    i = dict(h=P[0], y=P[1], w_post=P[2], w_pre=P[3], gate=None)
    i.update(inp or {})
    o = dict(h=P[9], y=P[10], w_post=P[11], w_pre=P[12], gate=None)
    o.update(out or {})
    desc = _norm_desc(**kw)
    n = ace.lib().ace_block_norm_grad_workspace_size(ctypes.byref(desc))
    return ace.lib().ace_block_norm_grad(ctypes.byref(desc), ctypes.byref(_lib.NormInputs(*i.values())), dh, dn,
                                         ctypes.byref(_lib.NormGrads(*o.values())), ws, n + need, None)


def test_block_norm_grad_refusals():
    for kw in (dict(T=-1), dict(eps=0.0), dict(dn=None), dict(inp=dict(w_pre=None)), dict(out=dict(w_post=None)),
               dict(out=dict(y=None)), dict(inp=dict(y=None, w_post=None), out=dict(w_post=None)), dict(out=dict(h=None)),
               dict(inp=dict(h=None)), dict(gate_kind=1, inp=dict(gate=P[4])), dict(out=dict(gate=P[13])),
               dict(out=dict(h=P[0] + 16)), dict(out=dict(w_pre=P[3])), dict(out=dict(h=P[10])), dict(dh=P[7] + 2),
               dict(out=dict(y=P[2])), dict(dh=None, dn=None, inp=dict(w_pre=None, h=None), out=dict(w_pre=None)),
               dict(gate_kind=3, inp=dict(gate=P[4]), out=dict(gate=P[4]))):
        assert _norm_grad(**kw) == BAD, kw
    assert _norm_grad(d=16400) == UNS
    for kw in (dict(ws=None), dict(ws=P[15] + 16), dict(need=-1)):
        assert _norm_grad(**kw) == WSP, kw


def _adapter(base=P[0], x=P[1], a=P[2], b=P[3], scale=P[4], offsets=P[5], ids=P[6], out=P[7], ws=P[15], need=0, **kw):
    d = dict(S=8, R=3, L=2, rank=16, d_in=64, d_out=64, dtype=_lib.ACE_BF16)
    d.update(kw)
    desc = _lib.AdapterDesc(*d.values())
    n = ace.lib().ace_adapter_workspace_size(ctypes.byref(desc))
    return ace.lib().ace_adapter_add(ctypes.byref(desc), base, x, a, b, scale, offsets, ids, out, ws, n + need, None)


def test_adapter_refusals():
    for kw in (dict(S=-1), dict(R=-1), dict(L=0), dict(rank=0), dict(d_in=0), dict(d_out=-8), dict(dtype=2), dict(base=None),
               dict(x=None), dict(a=None), dict(b=None), dict(offsets=None), dict(ids=None), dict(out=None),
               dict(x=P[1] + 8), dict(scale=P[4] + 2), dict(out=P[0] + 16), dict(out=P[1]), dict(out=P[2]), dict(out=P[3]),
               dict(out=P[4] - 16), dict(out=P[6])):
        assert _adapter(**kw) == BAD, kw
    for kw in (dict(S=BIG), dict(R=4097), dict(rank=136), dict(rank=12), dict(d_in=65544), dict(d_out=65544), dict(d_in=60),
               dict(d_out=4)):
        assert _adapter(**kw) == UNS, kw
    for kw in (dict(ws=None), dict(ws=P[15] + 16), dict(need=-1)):
        assert _adapter(S=8192, **kw) == WSP, kw
    assert _adapter(S=0, base=None, x=None, out=None) == _lib.ACE_OK


def _z(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype)


def _o(*v):
    return torch.tensor(v, dtype=torch.int32)


def test_wrappers_refuse():
    x, w, dy, o = _z(6, 16), _z(2, 8, 16), _z(6, 8), _o(0, 2, 6)
    bad = [
        (lambda: ace.grouped_matmul(x, w, o), "GPU"),
        (lambda: ace.grouped_matmul(x[0], w, o), "2 dimensions"),
        (lambda: ace.grouped_matmul(x.half(), w, o), "dtype"),
        (lambda: ace.grouped_matmul(x, w.float(), o), "dtype"),
        (lambda: ace.grouped_matmul(x, _z(2, 8, 24), o), "shape"),
        (lambda: ace.grouped_matmul(x, w, o.long()), "offsets: dtype"),
        (lambda: ace.grouped_matmul(x, w, _o(0, 6)), "offsets: shape"),
        (lambda: ace.grouped_matmul(_z(16, 6).t(), w, o), "contiguous"),
        (lambda: ace.grouped_matmul(x, w, o, out=_z(6, 16)), "out: shape"),
        (lambda: ace.grouped_matmul(x.clone().requires_grad_(), w, o), "no_grad"),
        (lambda: ace.grouped_matmul_grad_x(x, w, o), "dy: shape"),
        (lambda: ace.grouped_matmul_grad_w(dy, _z(5, 16), o), "x: shape"),
        (lambda: ace.grouped_matmul_grad_w(dy, x, _o(0)), "at least one group"),
        (lambda: ace.block_norm(x, dy), "y: shape"),
        (lambda: ace.block_norm(x), "y or w_pre"),
        (lambda: ace.block_norm(x, w_pre=_z(16), w_post=_z(16)), "need y"),
        (lambda: ace.block_norm(x, x, gate=_z(6)), "gate: shape"),
        (lambda: ace.block_norm(x, x, w_pre=_z(16, dtype=torch.float32)), "w_pre: dtype"),
        (lambda: ace.block_norm(x, x, out={"n": _z(5, 16)}), r"out\['n'\]: shape"),
        (lambda: ace.block_norm(x, x), "GPU"),
        (lambda: ace.block_norm_grad(None, None, x), "dh or dn"),
        (lambda: ace.block_norm_grad(x, x, x, x), "go together"),
        (lambda: ace.block_norm_grad(x, x, None, x, w_pre=_z(16)), "h is required"),
        (lambda: ace.adapter_add(dy, x, _z(2, 8, 16), _z(2, 8, 8), o, _o(0)), "adapter: shape"),
        (lambda: ace.adapter_add(dy, x, _z(2, 8, 16), _z(2, 8, 16), o, _o(0, -1)), "b: shape"),
        (lambda: ace.adapter_add(dy, x, _z(2, 8, 16), _z(2, 8, 8), o, _o(0, -1), scale=_z(2)), "scale: dtype"),
        (lambda: ace.adapter_add(dy, x, _z(2, 8, 16), _z(2, 8, 8), o, _o(0, -1)), "GPU"),
    ]
    for i, (call, match) in enumerate(bad):
        with pytest.raises(ValueError, match=match):
            print(i, inspect.getsource(call).strip())
            call()


def test_sizes_past_32_bits_are_refused():
    """2^32 + 5 rows or columns are not 5."""
    n = (1 << 32) + 5

    def m(*shape):
        return torch.empty(shape, dtype=torch.bfloat16, device="meta")

    o, i = torch.empty(3, dtype=torch.int32, device="meta"), torch.empty(2, dtype=torch.int32, device="meta")
    for call in (lambda: ace.grouped_matmul(m(n, 16), m(2, 8, 16), o), lambda: ace.grouped_matmul(m(1, n), m(2, 8, n), o),
                 lambda: ace.grouped_matmul_grad_x(m(n, 8), m(2, 8, 16), o),
                 lambda: ace.grouped_matmul_grad_w(m(n, 8), m(n, 16), o), lambda: ace.block_norm(m(n, 8), m(n, 8)),
                 lambda: ace.block_norm_grad(m(n, 8), None, None, m(n, 8)),
                 lambda: ace.adapter_add(m(n, 8), m(n, 16), m(2, 8, 16), m(2, 8, 8), o, i),
                 lambda: ace.adapter_add(m(6, 8), m(6, 16), m(n, 8, 16), m(n, 8, 8), o, i)):
        with pytest.raises(ValueError, match="size of"):
            call()


def test_workspace_sizes_of_refused_calls():
    assert ace.lib().ace_block_norm_grad_workspace_size(_lib.NormDesc(BIG, 64, _lib.ACE_BF16, 0, 1.0, 1.0, 1e-6)) == 0
    assert ace.lib().ace_block_norm_grad_workspace_size(_lib.NormDesc(64, 64, 7, 0, 1.0, 1.0, 1e-6)) == 0
    assert ace.lib().ace_adapter_workspace_size(_lib.AdapterDesc(BIG, 4, 2, 16, 64, 64, _lib.ACE_BF16)) == 0
    assert ace.lib().ace_adapter_workspace_size(_lib.AdapterDesc(8192, 4, 2, 12, 64, 64, _lib.ACE_BF16)) == 0
