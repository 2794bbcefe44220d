"""Refusals of the experts' operators, on the CPU: the C ABI returns before any launch, the wrappers raise before
they call it."""
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


def _gated_desc(kw):
    d = dict(S=64, N=4, M=64, K=64, dtype=_lib.ACE_BF16, activation=0, flags=0)
    d.update({k: kw.pop(k) for k in list(kw) if k in d})
    return _lib.GatedDesc(*d.values())


def _gated(x=P[0], wg=P[1], wu=P[2], offsets=P[3], a=P[4], g=P[5], u=P[6], null=False, ws=P[15], ws_bytes=1 << 40, **kw):
    desc = _gated_desc(kw)
    assert not kw
    return ace.lib().ace_grouped_gated(None if null else ctypes.byref(desc), x, wg, wu, offsets, a, g, u, ws, ws_bytes, None)


def _grad(da=P[0], x=P[1], wg=P[2], wu=P[3], offsets=P[4], g=P[5], u=P[6], dx=P[7], dwg=P[8], dwu=P[9], null=False, ws=P[15],
          ws_bytes=1 << 40, **kw):
    desc = _gated_desc(kw)
    assert not kw
    return ace.lib().ace_grouped_gated_grad(None if null else ctypes.byref(desc), da, x, wg, wu, offsets, g, u, dx, dwg, dwu,
                                            ws, ws_bytes, None)


SIZES_BAD = (dict(S=-1), dict(N=0), dict(M=0), dict(K=-8), dict(dtype=7), dict(flags=2), dict(activation=2),
             dict(activation=-1), dict(null=True))
SIZES_UNS = (dict(S=BIG), dict(N=4097), dict(M=65544), dict(K=65544), dict(M=12), dict(K=4), dict(dtype=_lib.ACE_F32, K=6))


def test_gated_refusals():
    for kw in SIZES_BAD + (dict(x=0), dict(wg=0), dict(wu=0), dict(offsets=0), dict(a=0), dict(g=0), dict(u=0), dict(x=P[0] + 8),
                           dict(wu=P[2] + 8), dict(a=P[4] + 4), dict(g=P[5] + 8), dict(offsets=P[3] + 2), dict(a=P[0]),
                           dict(a=P[1] + 64), dict(g=P[2]), dict(u=P[3]), dict(g=P[4]), dict(u=P[5] + 16)):
        assert _gated(**kw) == BAD, kw
    for kw in SIZES_UNS:
        assert _gated(**kw) == UNS, kw
    few = dict(S=64, N=2, M=128, K=4096, dtype=_lib.ACE_F32)
    n = ace.lib().ace_grouped_gated_workspace_size(_gated_desc(dict(few)))
    assert n > 0 and n % (2 * 64 * 128 * 4) == 0
    for kw in (dict(ws=0), dict(ws=P[15] + 16), dict(ws_bytes=n - 1)):
        assert _gated(**few, **kw) == WSP, kw
    assert _gated(S=0, x=0, a=0, g=0, u=0) == _lib.ACE_OK
    size = ace.lib().ace_grouped_gated_workspace_size
    assert size(_gated_desc(dict(S=32768, N=128, M=768, K=2048))) == 0
    for kw in (dict(S=BIG), dict(dtype=9), dict(activation=5), dict(S=0)):
        assert size(_gated_desc(kw)) == 0


def test_gated_grad_refusals():
    for kw in SIZES_BAD + (dict(da=0), dict(x=0), dict(g=0, u=0, x=0), dict(wg=0), dict(wu=0), dict(offsets=0), dict(dx=0),
                           dict(g=0), dict(u=0), dict(dwg=0), dict(dwu=0), dict(da=P[0] + 8), dict(x=P[1] + 8),
                           dict(dx=P[7] + 8), dict(dwu=P[9] + 8), dict(offsets=P[4] + 1), dict(g=P[5] + 4), dict(dx=P[0]),
                           dict(dx=P[1]), dict(dx=P[5]), dict(dwg=P[2]), dict(dwu=P[3] + 64), dict(dwu=P[8]), dict(dx=P[8]),
                           dict(dx=P[4])):
        assert _grad(**kw) == BAD, kw
    for kw in SIZES_UNS:
        assert _grad(**kw) == UNS, kw
    size = ace.lib().ace_grouped_gated_grad_workspace_size
    for gu in (dict(), dict(g=0, u=0)):
        for dw in (dict(), dict(dwg=0, dwu=0)):
            n = size(_gated_desc({}), int(not gu), int(not dw))
            assert n >= 2 * 64 * 64 * 2
            for kw in (dict(ws=0), dict(ws=P[15] + 16), dict(ws_bytes=n - 1)):
                assert _grad(**gu, **dw, **kw) == WSP, kw
    # more to add up where more is asked for
    d = _gated_desc(dict(S=40000, N=2, M=128, K=128))
    assert size(d, 1, 1) > size(d, 1, 0) and size(d, 0, 0) >= size(d, 1, 0)
    assert size(_gated_desc(dict(S=BIG)), 0, 1) == 0
    assert _grad(S=0, da=0, x=0, dx=0, g=0, u=0, dwg=0, dwu=0) == _lib.ACE_OK
    assert _grad(S=0, dwg=0) == BAD and _grad(S=0, dwg=P[8] + 2) == BAD


def _z(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype)


def _o(*v):
    return torch.tensor(v, dtype=torch.int32)


def refused(bad):
    for i, (call, match) in enumerate(bad):
        with pytest.raises(ValueError, match=match):
            print(i, inspect.getsource(call).strip())
            call()


def test_gated_wrappers_refuse():
    x, w, da, o = _z(6, 16), _z(2, 8, 16), _z(6, 8), _o(0, 2, 6)
    refused([
        (lambda: ace.grouped_gated(x, w, w, o), "GPU"),
        (lambda: ace.grouped_gated(x[0], w, w, o), "2 dimensions"),
        (lambda: ace.grouped_gated(x, w[0], w, o), "3 dimensions"),
        (lambda: ace.grouped_gated(x.half(), w, w, o), "dtype"),
        (lambda: ace.grouped_gated(x, w, w.float(), o), "w_up: dtype"),
        (lambda: ace.grouped_gated(x, w, _z(2, 16, 16), o), "w_up: shape"),
        (lambda: ace.grouped_gated(x, w, w, o.long()), "offsets: dtype"),
        (lambda: ace.grouped_gated(x, w, w, _o(0, 6)), "offsets: shape"),
        (lambda: ace.grouped_gated(_z(16, 6).t(), w, w, o), "contiguous"),
        (lambda: ace.grouped_gated(x, w, w, o, activation="relu"), "activation"),
        (lambda: ace.grouped_gated(x, w, w, o, out=_z(6, 16)), "out: shape"),
        (lambda: ace.grouped_gated(x, w, w, o, keep=True, out=(da, (da, _z(6, 16)))), "out's u: shape"),
        (lambda: ace.grouped_gated(x.clone().requires_grad_(), w, w, o), "no_grad"),
        (lambda: ace.grouped_gated_grad(x, x, w, w, o), "da: shape"),
        (lambda: ace.grouped_gated_grad(da, da, w, w, o), "x: shape"),
        (lambda: ace.grouped_gated_grad(da, None, w, w, o), "x is required"),
        (lambda: ace.grouped_gated_grad(da, None, w, w, o, kept=(da, da)), "x is required"),
        (lambda: ace.grouped_gated_grad(da, x, w, w, o, kept=(da, x)), "kept's u: shape"),
        (lambda: ace.grouped_gated_grad(da, x, w, w, o, activation=1), "activation"),
        (lambda: ace.grouped_gated_grad(da, x, w, w, o), "GPU"),
    ])


def test_gated_sizes_past_32_bits_are_refused():
    n = (1 << 32) + 5

    def m(*shape):
        return torch.empty(shape, dtype=torch.bfloat16, device="meta")

    o, w = torch.empty(3, dtype=torch.int32, device="meta"), m(2, 8, 16)
    for call in (lambda: ace.grouped_gated(m(n, 16), w, w, o), lambda: ace.grouped_gated(m(1, n), m(2, 8, n), m(2, 8, n), o),
                 lambda: ace.grouped_gated_grad(m(n, 8), m(n, 16), w, w, o)):
        with pytest.raises(ValueError, match="size of"):
            call()


def _convert(back=False, rows=64, K=64, dtype=_lib.ACE_BF16, x=P[0], codes=P[1], scales=P[2]):
    if back:
        return ace.lib().ace_mx4_dequantize(rows, K, dtype, codes, scales, x, None)
    return ace.lib().ace_mx4_quantize(rows, K, dtype, x, codes, scales, None)


@pytest.mark.parametrize("back", [False, True])
def test_mx4_conversion_refusals(back):
    for kw in (dict(rows=-1), dict(K=0), dict(K=-32), dict(dtype=5), dict(x=0), dict(codes=0), dict(scales=0), dict(x=P[0] + 8),
               dict(codes=P[1] + 8), dict(scales=P[2] + 2), dict(codes=P[0]), dict(scales=P[0] + 64)):
        assert _convert(back, **kw) == BAD, kw
    assert _convert(scales=P[1]) == BAD  # both are results
    for kw in (dict(K=48), dict(K=65568), dict(rows=1 << 31), dict(rows=1 << 30, K=256), dict(rows=1 << 62)):
        assert _convert(back, **kw) == UNS, kw
    assert _convert(back, rows=0, x=0, codes=0, scales=0) == _lib.ACE_OK


def _mx4(gated=False, x=P[0], xs=P[1], wc=P[2], wsc=P[3], uc=P[4], usc=P[5], offsets=P[6], out=P[7], null=False, ws=P[15],
         ws_bytes=1 << 40, **kw):
    d = dict(S=64, N=4, M=64, K=64, activation=0, flags=0)
    d.update(kw)
    desc = None if null else ctypes.byref(_lib.Mx4Desc(*d.values()))
    w, u = (None if c is None else ctypes.byref(_lib.Mx4Ptr(c, s)) for c, s in ((wc, wsc), (uc, usc)))
    if gated:
        return ace.lib().ace_grouped_gated_mx4(desc, x, xs, w, u, offsets, out, ws, ws_bytes, None)
    return ace.lib().ace_grouped_matmul_mx4(desc, x, xs, w, offsets, out, ws, ws_bytes, None)


@pytest.mark.parametrize("gated", [False, True])
def test_mx4_product_refusals(gated):
    bad = [dict(S=-1), dict(N=0), dict(M=0), dict(K=-32), dict(flags=2), dict(null=True), dict(x=0), dict(wc=None), dict(wc=0),
           dict(wsc=0), dict(offsets=0), dict(out=0), dict(x=P[0] + 8), dict(xs=P[1] + 2), dict(wc=P[2] + 4), dict(wsc=P[3] + 1),
           dict(offsets=P[6] + 2), dict(out=P[7] + 8), dict(out=P[0]), dict(out=P[1]), dict(out=P[2] + 64), dict(out=P[3]),
           dict(out=P[6])]
    if gated:
        bad += [dict(activation=2), dict(activation=-1), dict(uc=None), dict(uc=0), dict(usc=0), dict(uc=P[4] + 8), dict(out=P[4]),
                dict(out=P[5])]
    for kw in bad:
        assert _mx4(gated, **kw) == BAD, kw
    for kw in (dict(S=BIG), dict(N=4097), dict(M=65544), dict(K=65568), dict(M=12), dict(K=48), dict(K=8)):
        assert _mx4(gated, **kw) == UNS, kw
    few = dict(S=512, N=1, M=512, K=4096)
    size = ace.lib().ace_grouped_mx4_workspace_size
    n = size(_lib.Mx4Desc(*few.values(), 0, 0), int(gated))
    assert n > 0 and n % (512 * 512 * 4 * (2 if gated else 1)) == 0
    for kw in (dict(ws=0), dict(ws=P[15] + 16), dict(ws_bytes=n - 1)):
        assert _mx4(gated, **few, **kw) == WSP, kw
    assert size(_lib.Mx4Desc(32768, 128, 768, 2048, 0, 0), int(gated)) == 0
    assert size(_lib.Mx4Desc(64, 4, 64, 48, 0, 0), int(gated)) == 0
    assert _mx4(gated, S=0, x=0, xs=0, wc=None, uc=None, out=0, offsets=0) == _lib.ACE_OK


def test_mx4_wrappers_refuse():
    u8 = torch.uint8
    x, o = _z(6, 64), _o(0, 2, 6)
    w = ace.Mx4(_z(2, 8, 32, dtype=u8), _z(2, 8, 4, dtype=u8))
    q = ace.Mx4(_z(6, 32, dtype=u8), _z(6, 4, dtype=u8))
    refused([
        (lambda: ace.mx4_quantize(x), "GPU"),
        (lambda: ace.mx4_quantize(_z(6, 48)), "multiple of 32"),
        (lambda: ace.mx4_quantize(_z(6, 0)), "multiple of 32"),
        (lambda: ace.mx4_quantize(torch.zeros(())), "1 dimension"),
        (lambda: ace.mx4_quantize(x.half()), "dtype"),
        (lambda: ace.mx4_quantize(_z(64, 6).t()), "contiguous"),
        (lambda: ace.mx4_quantize(x.clone().requires_grad_()), "no_grad"),
        (lambda: ace.mx4_dequantize(q), "GPU"),
        (lambda: ace.mx4_dequantize(x), "Mx4"),
        (lambda: ace.mx4_dequantize(q, torch.float16), "dtype"),
        (lambda: ace.mx4_dequantize(ace.Mx4(q.codes, q.scales[:, :2])), "q.scales: shape"),
        (lambda: ace.mx4_dequantize(ace.Mx4(q.codes.int(), q.scales)), "q.codes: dtype"),
        (lambda: ace.mx4_dequantize(ace.Mx4(q.codes[:, :24], q.scales)), "multiple of 32"),
        (lambda: ace.grouped_matmul(x, w, o), "GPU"),
        (lambda: ace.grouped_matmul(q, w, o), "GPU"),
        (lambda: ace.grouped_matmul(x.float(), w, o), "bf16 or Mx4"),
        (lambda: ace.grouped_matmul(_z(6, 96), w, o), "x: shape"),
        (lambda: ace.grouped_matmul(q, _z(2, 8, 64), o), "2 dimensions"),
        (lambda: ace.grouped_matmul(ace.Mx4(q.codes[0], q.scales[0]), w, o), "2 dimensions"),
        (lambda: ace.grouped_matmul(x, ace.Mx4(w.codes[0], w.scales[0]), o), "3 dimensions"),
        (lambda: ace.grouped_matmul(x, w, _o(0, 6)), "offsets: shape"),
        (lambda: ace.grouped_matmul(x, w, o, out=_z(6, 8, dtype=torch.float32)), "out: dtype"),
        (lambda: ace.grouped_matmul_grad_x(_z(6, 8), w, o), "3 dimensions"),
        (lambda: ace.grouped_gated(x, w, _z(2, 8, 64), o), "w_up must be an Mx4"),
        (lambda: ace.grouped_gated(x, _z(2, 8, 64), w, o), "w_gate must be an Mx4"),
        (lambda: ace.grouped_gated(x, w, w, o, keep=True), "no gradient"),
        (lambda: ace.grouped_gated(x, w, w, o, activation="tanh"), "activation"),
        (lambda: ace.grouped_gated(x, w, ace.Mx4(w.codes[:, :4], w.scales[:, :4]), o), "w_up.codes: shape"),
        (lambda: ace.grouped_gated(x, w, w, o), "GPU"),
        (lambda: ace.grouped_gated_grad(_z(6, 8), x, w, w, o), "3 dimensions"),
    ])
