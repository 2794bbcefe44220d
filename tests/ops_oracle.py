"""The operators around the layer in 64 bits, as their definitions say, on the CPU: what the
GPU tests compare with.  Every function also returns `mag`, the sum of the absolute values of
the terms of each result, which rounding errors of sums are relative to."""
from __future__ import annotations

import torch

F32 = 2.0 ** -24
HALF = {torch.bfloat16: torch.finfo(torch.bfloat16).eps / 2, torch.float32: F32}


def close(got, ref, mag, dtype, terms, name=""):
    """|got - ref| within the rounding of the result and `terms` fp32 operations on its terms.  The matrix
    cores may round a sum toward zero: a whole fp32 step, 2 F32, for each operation."""
    got = got.detach().cpu().double()
    assert got.shape == ref.shape, (name, got.shape, ref.shape)
    err = terms * 2 * F32 * mag
    tol = HALF[dtype] * (ref.abs() + err) + err + 1e-37
    bad = ~((got - ref).abs() <= tol)
    if bad.any():
        i = tuple(torch.nonzero(bad)[0].tolist())
        raise AssertionError(f"{name}: {int(bad.sum())} of {bad.numel()} off, first at {i}: {got[i]} for {ref[i]} "
                             f"(tolerance {tol[i]})")


def groups(offsets):
    o = [int(v) for v in offsets]
    return [(e, o[e], o[e + 1]) for e in range(len(o) - 1)]


def grouped(x, w, offsets):
    y = torch.zeros((x.shape[0], w.shape[1]), dtype=torch.float64)
    mag = torch.zeros_like(y)
    for e, lo, hi in groups(offsets):
        if hi > lo:
            y[lo:hi] = x[lo:hi].double() @ w[e].double().t()
            mag[lo:hi] = x[lo:hi].double().abs() @ w[e].double().abs().t()
    return y, mag


def grouped_grad_w(dy, x, offsets):
    out = torch.zeros((len(offsets) - 1, dy.shape[1], x.shape[1]), dtype=torch.float64)
    mag = torch.zeros_like(out)
    for e, lo, hi in groups(offsets):
        if hi > lo:
            out[e] = dy[lo:hi].double().t() @ x[lo:hi].double()
            mag[e] = dy[lo:hi].double().abs().t() @ x[lo:hi].double().abs()
    return out, mag


def rms(v, eps):
    return (v.square().mean(dim=1, keepdim=True) + eps).sqrt()


def block_norm(h, y=None, w_post=None, w_pre=None, gate=None, res_scale=1.0, branch_scale=1.0, eps=1e-6):
    """(dict of results, dict of mags); differentiable."""
    h = h.double()
    if y is None:
        hp, mag = h, h.abs()
    else:
        u = y.double()
        if w_post is not None:
            u = u / rms(u, eps) * w_post.double()
        if gate is not None:
            u = gate.double() * u
        hp = res_scale * h + branch_scale * u
        mag = (res_scale * h).abs() + (branch_scale * u).abs()
    out, mags = {"h": hp}, {"h": mag}
    if w_pre is not None:
        k = w_pre.double() / rms(hp, eps)
        out["n"], mags["n"] = hp * k, mag * k.abs()
    return out, mags


def block_norm_grad(dh, dn, h, y=None, w_post=None, w_pre=None, gate=None, res_scale=1.0, branch_scale=1.0, eps=1e-6):
    """Gradients at the stored h', and the absolute values of their terms."""
    d = (dh if dh is not None else dn).shape[1]
    t = torch.zeros_like((dh if dh is not None else dn).double()) if dh is None else dh.double()
    mt = t.abs()
    out, mag = {}, {}
    if w_pre is not None:
        hd, p = h.double(), dn.double() * w_pre.double()
        r = rms(hd, eps)
        t = t + p / r - hd * ((p * hd).sum(1, keepdim=True) / (d * r ** 3))
        mt = mt + p.abs() / r + hd.abs() * ((p * hd).abs().sum(1, keepdim=True) / (d * r ** 3))
        term = dn.double() * hd / r
        out["w_pre"], mag["w_pre"] = term.sum(0), term.abs().sum(0)
    out["h"], mag["h"] = res_scale * t, abs(res_scale) * mt
    if y is None:
        return out, mag
    yd = y.double()
    s = rms(yd, eps) if w_post is not None else torch.ones((), dtype=torch.float64)
    wp = w_post.double() if w_post is not None else torch.ones((), dtype=torch.float64)
    yn = yd / s
    db, mdb = branch_scale * t, abs(branch_scale) * mt
    g = torch.ones((), dtype=torch.float64) if gate is None else gate.double()
    if gate is not None:
        term, mterm = db * (yn * wp), mdb * (yn * wp).abs()
        if gate.shape == (d,):
            out["gate"], mag["gate"] = term.sum(0), mterm.sum(0)
        elif gate.shape[1] == 1 and d != 1:
            out["gate"], mag["gate"] = term.sum(1, keepdim=True), mterm.sum(1, keepdim=True)
        else:
            out["gate"], mag["gate"] = term, mterm
    q, mq = db * g, mdb * g.abs()
    if w_post is not None:
        out["w_post"], mag["w_post"] = (q * yn).sum(0), (mq * yn.abs()).sum(0)
        q, mq = q * wp, mq * wp.abs()
        out["y"] = q / s - yd * ((q * yd).sum(1, keepdim=True) / (d * s ** 3))
        mag["y"] = mq / s + yd.abs() * ((mq * yd.abs()).sum(1, keepdim=True) / (d * s ** 3))
    else:
        out["y"], mag["y"] = q, mq
    return out, mag


def adapter_add(base, x, a, b, offsets, adapter, scale=None):
    out, mag = base.double(), base.double().abs()
    L = a.shape[0]
    for i, lo, hi in groups(offsets):
        l = int(adapter[i])
        if hi > lo and 0 <= l < L:
            sc = 1.0 if scale is None else float(scale[l])
            v, mv = x[lo:hi].double() @ a[l].double().t(), x[lo:hi].double().abs() @ a[l].double().abs().t()
            out[lo:hi] += sc * (v @ b[l].double().t())
            mag[lo:hi] += abs(sc) * (mv @ b[l].double().abs().t())
    return out, mag
