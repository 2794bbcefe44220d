"""Microscaled 4-bit floating point number by number, in 64 bits, as the format defines it: what the GPU tests
compare with."""
from __future__ import annotations

import torch

GRID = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)


def scale_bytes(K):
    return 4 * ((K + 127) // 128)


def quantize(x):
    """codes and scales of x [..., K]: the nearest magnitude by its distance to all eight, the even code on a tie."""
    K = x.shape[-1]
    v = x.double().reshape(-1, K // 32, 32)
    ok = v.isfinite().all(dim=2)
    v = torch.where(ok[..., None], v, torch.zeros((), dtype=torch.float64))
    top = v.abs().amax(dim=2)
    e = (torch.frexp(top)[1] - 3).clamp_min(-127)  # frexp's mantissa lies in [1/2, 1)
    e = torch.where(top == 0, torch.full_like(e, -127), e)
    a = v.abs() / torch.ldexp(torch.ones((), dtype=torch.float64), e)[..., None]
    dist = (a.clamp_max(6.0)[..., None] - GRID).abs()
    best = dist.amin(dim=-1, keepdim=True)
    cand = dist == best
    even = cand & (torch.arange(8) % 2 == 0)
    pick = torch.where(even.any(dim=-1, keepdim=True), even, cand)
    code = pick.int().argmax(dim=-1) + 8 * torch.signbit(v).int()
    code = torch.where(ok[..., None], code, torch.zeros_like(code)).reshape(-1, K)
    s = torch.where(ok, e + 127, torch.full_like(e, 255))
    scales = torch.zeros((code.shape[0], scale_bytes(K)), dtype=torch.uint8)
    scales[:, :K // 32] = s.to(torch.uint8)
    codes = (code[:, 0::2] + 16 * code[:, 1::2]).to(torch.uint8)
    return codes.reshape(*x.shape[:-1], K // 2), scales.reshape(*x.shape[:-1], scale_bytes(K))


def values(codes, scales):
    """The numbers in 64 bits."""
    c = torch.stack([codes % 16, codes // 16], dim=-1).flatten(-2).long()
    v = torch.cat([GRID, -GRID])[c]
    nb = c.shape[-1] // 32
    e = scales[..., :nb].int() - 127
    k = torch.ldexp(torch.ones((), dtype=torch.float64), e)
    k = torch.where(e == 128, torch.full_like(k, float("nan")), k)
    return (v.unflatten(-1, (nb, 32)) * k[..., None]).flatten(-2)
