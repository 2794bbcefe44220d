"""The experts' operators in 64 bits, as their definitions say, on the CPU, with how far results may be off:
what the GPU tests compare with."""
from __future__ import annotations

import math

import torch

from ops_oracle import F32, HALF, groups


def act(g, name):
    """act(g), act'(g)."""
    if name == "silu":
        s = torch.sigmoid(g)
        return g * s, s * (1 + g * (1 - s))
    p = torch.special.ndtr(g)
    return g * p, p + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)


def within(got, ref, err, dtype, name=""):
    """|got - ref| within err and the rounding of the result."""
    got = got.detach().cpu().double()
    assert got.shape == ref.shape, (name, got.shape, ref.shape)
    tol = HALF[dtype] * (ref.abs() + err) + err + 1e-37
    bad = ~((got - ref).abs() <= tol)
    if bad.any():
        i = tuple(torch.nonzero(bad)[0].tolist())
        raise AssertionError(f"{name}: {int(bad.sum())} of {bad.numel()} off, first at {i}: {got[i]} for {ref[i]} "
                             f"(tolerance {tol[i]})")


def both(x, w, offsets):
    """y[r] = w[e] x[r] and the error of its fp32 sum: a whole step for each of the K products (see ops_oracle.close)."""
    y = torch.zeros((x.shape[0], w.shape[1]), dtype=torch.float64)
    err = torch.zeros_like(y)
    for e, lo, hi in groups(offsets):
        if hi > lo:
            y[lo:hi] = x[lo:hi].double() @ w[e].double().t()
            err[lo:hi] = x[lo:hi].double().abs() @ w[e].double().abs().t()
    return y, 2 * F32 * x.shape[1] * err


def gated(x, w_gate, w_up, offsets, name):
    """dict of a, g, u, and of their errors.  |act'| <= 1.13, and act is computed to some steps of 32 bits; where its
    exponential is formed from |g| in 32 bits, to as many more as |g|."""
    g, eg = both(x, w_gate, offsets)
    u, eu = both(x, w_up, offsets)
    f, _ = act(g, name)
    a = f * u
    ea = 1.13 * eg * (u.abs() + eu) + f.abs() * eu + (16 + 4 * g.abs()) * F32 * a.abs()
    return dict(a=a, g=g, u=u), dict(a=ea, g=eg, u=eu)


def gated_grad(da, x, w_gate, w_up, offsets, name, kept=None, dtype=torch.float32):
    """dict of the gradients of x, w_gate, w_up, and of their errors: those of act' (its own derivative is at most 0.8),
    of dg and du rounded to dtype, and of the sums."""
    if kept is None:
        g, eg = both(x, w_gate, offsets)
        u, eu = both(x, w_up, offsets)
    else:
        g, u = (t.double() for t in kept)
        eg = eu = torch.zeros_like(g)
    d = da.double()
    f, s = act(g, name)
    dg, du = d * u * s, d * f
    some = (32 + 8 * g.abs()) * F32
    edg = d.abs() * ((u.abs() + eu) * 0.8 * eg + 1.13 * eu + some * u.abs() * (s.abs() + g.abs().clamp_max(1)))
    edu = d.abs() * (1.13 * eg + some * f.abs())
    edg, edu = (e + HALF[dtype] * (v.abs() + e) for e, v in ((edg, dg), (edu, du)))
    S, K, M = da.shape[0], w_gate.shape[2], da.shape[1]
    out = {"x": torch.zeros((S, K), dtype=torch.float64)}
    out.update({n: torch.zeros(w_gate.shape, dtype=torch.float64) for n in ("w_gate", "w_up")})
    err = {n: torch.zeros_like(t) for n, t in out.items()}
    for e, lo, hi in groups(offsets):
        if hi <= lo:
            continue
        for n, w, v, ev in (("w_gate", w_gate, dg, edg), ("w_up", w_up, du, edu)):
            wd, vd, evd = w[e].double(), v[lo:hi], ev[lo:hi]
            out["x"][lo:hi] += vd @ wd
            err["x"][lo:hi] += (evd + 2 * F32 * 2 * M * (vd.abs() + evd)) @ wd.abs()
            if x is not None:
                xd = x[lo:hi].double()
                out[n][e] = vd.t() @ xd
                err[n][e] = (evd + 2 * F32 * (hi - lo) * (vd.abs() + evd)).t() @ xd.abs()
    return out, err
