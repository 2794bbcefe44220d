"""The operators around the ACE MoE layer that this framework is timed on: what a decoder
that contains the layer calls next to it, in serving and in fine-tuning.

Three families, each through the package's public entry points (`own`) or as elementary
torch operations in 32 bits:
  grouped  matrix products grouped by expert with ragged sizes: forward ("fwd"), gradient of
           the rows ("grad_x") and of the weights ("grad_w")
  norm     the norms after one block and before the next, fused with the block's gate and the
           residual scale: forward ("fwd") and gradients ("grad")
  adapter  low-rank adapters of many requests at once beside a shared projection

dtype is the type of every activation, weight and output.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
EPS = 1e-6
_DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _grouped(**kw):
    case = dict(kind="grouped", way="fwd", S=256, N=128, K=2048, M=768, dtype="bf16", zipf=0.0)
    case.update(kw)
    return case


def _norm(**kw):
    case = dict(kind="norm", way="fwd", T=1, d=2048, dtype="bf16", post=True, pre=True, gate="channel",
                res_scale=1.0, branch_scale=1.0)
    case.update(kw)
    return case


def _adapter(**kw):
    case = dict(kind="adapter", T=32, R=32, L=16, rank=16, d_in=2048, d_out=2048, dtype="bf16")
    case.update(kw)
    return case


def listed():
    return [
        # a decode batch of 32 tokens, eight slots each: a few rows per expert, weight streaming
        _grouped(name="grouped_decode", S=256),
        # the up projection of a 4096-token prompt with every slot kept
        _grouped(name="grouped_prefill", S=32768),
        # the wider pool under a skewed router: experts from a handful of rows to thousands
        _grouped(name="grouped_zipf", S=65536, N=256, M=512, zipf=1.1),
        # fine-tuning on 2048 tokens: rows' gradient of a down projection
        _grouped(name="grouped_grad_x", way="grad_x", S=16384, K=768, M=2048),
        # fine-tuning on 2048 tokens: the experts' gradients of an up projection
        _grouped(name="grouped_grad_w", way="grad_w", S=16384),
        # an fp32 model on a ragged batch
        _grouped(name="grouped_f32", S=2069, N=32, K=1024, M=512, dtype="f32"),
        # one new token through the norms between two blocks
        _norm(name="norm_1"),
        # the same for a prompt of 8192 tokens
        _norm(name="norm_8192", T=8192),
        # the gradients of the norms, the gate and the residual stream for 4096 tokens
        _norm(name="norm_grad_4096", way="grad", T=4096, res_scale=0.9, branch_scale=0.5),
        # an fp32 model, one gate per token, on a ragged batch
        _norm(name="norm_grad_f32", way="grad", T=517, d=1024, dtype="f32", gate="token"),
        # 32 requests decoding one token each with 16 adapters among them
        _adapter(name="adapter_decode"),
        # 7 prompts of uneven lengths with wider adapters
        _adapter(name="adapter_prefill", T=4096, R=7, L=5, rank=64),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["grouped", "grouped", "norm", "adapter"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    if kind == "grouped":
        while True:
            case = _grouped(way=rng.choice(["fwd", "grad_x", "grad_w"]), S=_log_int(rng, 1, 65536),
                            N=_log_int(rng, 2, 256), K=8 * _log_int(rng, 8, 512), M=8 * _log_int(rng, 8, 512),
                            dtype=dtype, zipf=rng.choice([0.0, 0.0, 1.1]))
            flops = case["S"] * case["K"] * case["M"] * (16 if dtype == "f32" else 1)
            if flops <= 65536 * 2048 * 512 and case["N"] * case["K"] * case["M"] <= 256 * 2048 * 512:
                return case
    if kind == "norm":
        while True:
            case = _norm(way=rng.choice(["fwd", "grad"]), T=_log_int(rng, 1, 65536), d=8 * _log_int(rng, 16, 1024),
                         dtype=dtype, post=rng.random() < 0.7, pre=rng.random() < 0.8,
                         gate=rng.choice(["none", "channel", "token", "full"]),
                         res_scale=rng.choice([1.0, round(rng.uniform(0.5, 1.5), 3)]),
                         branch_scale=rng.choice([1.0, round(rng.uniform(0.1, 1.0), 3)]))
            if case["T"] * case["d"] * (2 if dtype == "f32" else 1) <= 32768 * 2048:
                return case
    T = _log_int(rng, 1, 16384)
    while True:
        case = _adapter(T=T, R=_log_int(rng, 1, min(T, 512)), L=_log_int(rng, 1, 64), rank=8 * _log_int(rng, 1, 16),
                        d_in=8 * _log_int(rng, 16, 512), d_out=8 * _log_int(rng, 16, 512), dtype=dtype)
        if T * (case["d_in"] + case["d_out"]) * (2 if dtype == "f32" else 1) <= 16384 * 4096:
            return case


# ---------------------------------------------------------------- inputs

def _normal(gen, shape, std, mean, dtype):
    return torch.empty(shape, dtype=dtype, device=DEV).normal_(mean, std, generator=gen)


def _sizes(gen, total, parts, zipf):
    """Ragged sizes of `parts` groups: a draw of `total` rows over equal or skewed shares."""
    share = torch.ones(parts, dtype=torch.float64)
    if zipf > 0:
        share = (torch.arange(parts, dtype=torch.float64) + 1) ** -zipf
        share = share[torch.randperm(parts, generator=gen)]
    pick = torch.multinomial(share, total, replacement=True, generator=gen)
    return torch.bincount(pick, minlength=parts).tolist()


def _offsets(sizes):
    return [0] + torch.tensor(sizes, dtype=torch.int64).cumsum(0).tolist()


def _device_ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _grouped_inputs(case, seed):
    """Rows N(0, 1), expert weights N(0, 0.02), gradients of the outputs N(0, 1)."""
    host = torch.Generator().manual_seed(seed)
    gen = torch.Generator(device=DEV).manual_seed(seed)
    S, N, K, M, dt = case["S"], case["N"], case["K"], case["M"], _DT[case["dtype"]]
    offs = _offsets(_sizes(host, S, N, case["zipf"]))
    t = {}
    if case["way"] != "grad_x":
        t["x"] = _normal(gen, (S, K), 1.0, 0.0, dt)
    if case["way"] != "grad_w":
        t["w"] = _normal(gen, (N, M, K), 0.02, 0.0, dt)
    if case["way"] != "fwd":
        t["dy"] = _normal(gen, (S, M), 1.0, 0.0, dt)
    return t, offs


def _norm_inputs(case, seed):
    """A residual stream that has grown over some blocks, a block's output, norm weights near
    one, gates of either sign, gradients as large as a mean loss over the batch leaves them."""
    gen = torch.Generator(device=DEV).manual_seed(seed)
    T, d, dt = case["T"], case["d"], _DT[case["dtype"]]
    t = {"h": _normal(gen, (T, d), 2.0, 0.0, dt), "y": _normal(gen, (T, d), 0.7, 0.0, dt), "w_post": None,
         "w_pre": None, "gate": None, "dh": None, "dn": None}
    if case["post"]:
        t["w_post"] = _normal(gen, (d,), 0.1, 1.0, dt)
    if case["pre"]:
        t["w_pre"] = _normal(gen, (d,), 0.1, 1.0, dt)
    shape = {"channel": (d,), "token": (T, 1), "full": (T, d)}.get(case["gate"])
    if shape:
        t["gate"] = _normal(gen, shape, 0.5, 0.5, dt)
    if case["way"] == "grad":
        t["dh"] = _normal(gen, (T, d), 1e-2, 0.0, dt)
        if case["pre"]:
            t["dn"] = _normal(gen, (T, d), 1e-2, 0.0, dt)
    return t


def _adapter_inputs(case, seed):
    """Requests of uneven lengths; about one in eight has no adapter."""
    host = torch.Generator().manual_seed(seed)
    gen = torch.Generator(device=DEV).manual_seed(seed)
    T, R, L, r, dt = case["T"], case["R"], case["L"], case["rank"], _DT[case["dtype"]]
    sizes = [1] * R if T == R else _sizes(host, T, R, 0.7)
    ids = torch.randint(0, L, (R,), generator=host)
    ids[torch.rand(R, generator=host) < 0.125] = -1
    t = {"base": _normal(gen, (T, case["d_out"]), 1.0, 0.0, dt), "x": _normal(gen, (T, case["d_in"]), 1.0, 0.0, dt),
         "a": _normal(gen, (L, r, case["d_in"]), case["d_in"] ** -0.5, 0.0, dt),
         "b": _normal(gen, (L, case["d_out"], r), 0.1, 0.0, dt),
         "scale": _normal(gen, (L,), 0.2, 1.0, torch.float32)}
    return t, _offsets(sizes), ids.tolist()


def prepare(case, seed):
    """The tensors of a call; the offsets and adapter numbers on the host too, where the plain
    forms split their products by them."""
    if case["kind"] == "grouped":
        t, offs = _grouped_inputs(case, seed)
        return dict(case=case, t=t, offs=offs, offsets=_device_ints(offs))
    if case["kind"] == "norm":
        return dict(case=case, t=_norm_inputs(case, seed))
    t, offs, ids = _adapter_inputs(case, seed)
    return dict(case=case, t=t, offs=offs, ids=ids, offsets=_device_ints(offs), adapter=_device_ints(ids))


# ---------------------------------------------------------------- one pass

def run(state):
    if own:
        return _run_own(state)
    return {"grouped": _plain_grouped, "norm": _plain_norm, "adapter": _plain_adapter}[state["case"]["kind"]](state)


def _run_own(state):
    import paper_2609_05228_amd as ace

    case, t = state["case"], state["t"]
    if case["kind"] == "grouped":
        if case["way"] == "fwd":
            return ace.grouped_matmul(t["x"], t["w"], state["offsets"])
        if case["way"] == "grad_x":
            return ace.grouped_matmul_grad_x(t["dy"], t["w"], state["offsets"])
        return ace.grouped_matmul_grad_w(t["dy"], t["x"], state["offsets"])
    if case["kind"] == "norm":
        kw = dict(w_post=t["w_post"], w_pre=t["w_pre"], gate=t["gate"], res_scale=case["res_scale"],
                  branch_scale=case["branch_scale"], eps=EPS)
        if case["way"] == "fwd":
            return ace.block_norm(t["h"], t["y"], **kw)
        return ace.block_norm_grad(t["dh"], t["dn"], t["h"], t["y"], **kw)
    return ace.adapter_add(t["base"], t["x"], t["a"], t["b"], state["offsets"], state["adapter"], scale=t["scale"])


def _groups(offs):
    return [(e, offs[e], offs[e + 1]) for e in range(len(offs) - 1) if offs[e + 1] > offs[e]]


def _plain_grouped(state):
    case, t = state["case"], state["t"]
    dt = _DT[case["dtype"]]
    if case["way"] == "grad_w":
        dw = torch.zeros((case["N"], case["M"], case["K"]), dtype=dt, device=DEV)
        for e, lo, hi in _groups(state["offs"]):
            dw[e] = t["dy"][lo:hi].float().t() @ t["x"][lo:hi].float()
        return dw
    rows = t["x"] if case["way"] == "fwd" else t["dy"]
    out = torch.empty((case["S"], case["M"] if case["way"] == "fwd" else case["K"]), dtype=dt, device=DEV)
    for e, lo, hi in _groups(state["offs"]):
        w = t["w"][e].float()
        out[lo:hi] = rows[lo:hi].float() @ (w.t() if case["way"] == "fwd" else w)
    return out


def _rms(v):
    return torch.rsqrt((v * v).mean(dim=1, keepdim=True) + EPS)


def _plain_norm(state):
    case, t = state["case"], state["t"]
    dt = _DT[case["dtype"]]
    f = {k: (None if v is None else v.float()) for k, v in t.items()}
    a, b = case["res_scale"], case["branch_scale"]
    gate = 1.0 if f["gate"] is None else f["gate"]
    y = f["y"]
    if case["post"]:
        s = _rms(y)
        yn = y * s
        u = yn * f["w_post"]
    else:
        u = y
    if case["way"] == "fwd":
        h = a * f["h"] + b * (gate * u)
        out = {"h": h.to(dt)}
        if case["pre"]:
            out["n"] = (h * _rms(h) * f["w_pre"]).to(dt)
        return out
    out = {}
    g = f["dh"]
    if case["pre"]:
        r = _rms(f["h"])
        hn = f["h"] * r
        p = f["dn"] * f["w_pre"]
        g = g + r * (p - hn * (p * hn).mean(dim=1, keepdim=True))
        out["w_pre"] = (f["dn"] * hn).sum(dim=0).to(dt)
    out["h"] = (a * g).to(dt)
    g = b * g
    if case["gate"] != "none":
        dg = g * u
        dg = dg.sum(dim=0) if case["gate"] == "channel" else dg.sum(dim=1, keepdim=True) if case["gate"] == "token" else dg
        out["gate"] = dg.to(dt)
    g = g * gate
    if case["post"]:
        out["w_post"] = (g * yn).sum(dim=0).to(dt)
        p = g * f["w_post"]
        g = s * (p - yn * (p * yn).mean(dim=1, keepdim=True))
    out["y"] = g.to(dt)
    return out


def _plain_adapter(state):
    case, t = state["case"], state["t"]
    out = t["base"].clone()
    for (lo, hi), ad in zip(zip(state["offs"], state["offs"][1:]), state["ids"]):
        if hi > lo and ad >= 0:
            v = t["x"][lo:hi].float() @ t["a"][ad].float().t()
            d = (v @ t["b"][ad].float().t()) * t["scale"][ad]
            out[lo:hi] = (t["base"][lo:hi].float() + d).to(_DT[case["dtype"]])
    return out


# ---------------------------------------------------------------- work

def _expected_active(S, N, zipf):
    """Groups that a draw of S rows is expected to reach."""
    share = [(i + 1) ** -zipf for i in range(N)]
    tot = sum(share)
    return sum(1 - (1 - s / tot) ** S for s in share)


def work(case):
    es = 2 if case["dtype"] == "bf16" else 4
    if case["kind"] == "grouped":
        S, N, K, M = case["S"], case["N"], case["K"], case["M"]
        # the gradient of the weights writes the groups without rows too
        n = N if case["way"] == "grad_w" else _expected_active(S, N, case["zipf"])
        return {"bytes": int(es * (S * K + S * M + n * K * M)) + 4 * (N + 1), "flops": 2 * S * K * M}
    if case["kind"] == "norm":
        T, d = case["T"], case["d"]
        gate = {"none": 0, "channel": d, "token": T, "full": T * d}[case["gate"]]
        par = d * (case["post"] + case["pre"])
        if case["way"] == "fwd":
            full = 3 + case["pre"]  # h, y -> h'[, n]
            return {"bytes": es * (full * T * d + par + gate), "flops": T * d * (4 + 3 * case["post"] + 4 * case["pre"])}
        # dh, y [, dn, h'] -> dh, dy; the block's output only where its norm or gate needs it
        full = 3 + 2 * case["pre"] + (case["post"] or case["gate"] != "none")
        return {"bytes": es * (full * T * d + 2 * par + 2 * gate),
                "flops": T * d * (4 + 10 * case["post"] + 10 * case["pre"])}
    T, r, di, do = case["T"], case["rank"], case["d_in"], case["d_out"]
    used = 0.875
    n = case["L"] * (1 - (1 - 1 / case["L"]) ** (used * case["R"]))
    return {"bytes": int(es * (used * T * di + 2 * T * do + n * r * (di + do))), "flops": int(used * 2 * T * r * (di + do))}


# ---------------------------------------------------------------- in 64 bits

def exact(case, seed):
    if case["kind"] == "grouped":
        return _exact_grouped(case, *_grouped_inputs(case, seed))
    if case["kind"] == "norm":
        return _exact_norm(case, _norm_inputs(case, seed))
    return _exact_adapter(case, *_adapter_inputs(case, seed))


def _exact_grouped(case, t, offs):
    if case["way"] == "grad_w":
        out = torch.zeros((case["N"], case["M"], case["K"]), dtype=torch.float64, device=DEV)
        for e in range(case["N"]):
            rows = slice(offs[e], offs[e + 1])
            out[e].addmm_(t["dy"][rows].double().t().contiguous(), t["x"][rows].double())
        return out
    cols = case["M"] if case["way"] == "fwd" else case["K"]
    out = torch.zeros((case["S"], cols), dtype=torch.float64, device=DEV)
    for e in range(case["N"]):
        rows = slice(offs[e], offs[e + 1])
        if case["way"] == "fwd":
            out[rows] = torch.mm(t["w"][e].double(), t["x"][rows].double().t()).t()
        else:
            out[rows] = torch.mm(t["w"][e].double().t(), t["dy"][rows].double().t()).t()
    return out


def _exact_norm(case, t):
    """By the chain rule on row vectors: the Jacobian of v -> v / rms(v) is (I - v v^T / (d rms^2)) / rms."""
    d = case["d"]
    v = {k: (None if x is None else x.double()) for k, x in t.items()}
    ones = torch.ones((), dtype=torch.float64, device=DEV)
    gate = ones if v["gate"] is None else v["gate"]
    w_post = ones if v["w_post"] is None else v["w_post"]

    def rms(x):
        return (x.square().sum(dim=1, keepdim=True) / d + EPS).sqrt()

    def jac(x, g):
        m = rms(x)
        return g / m - x * ((g * x).sum(dim=1, keepdim=True) / (d * m ** 3))

    ybar = v["y"] / rms(v["y"]) if case["post"] else v["y"]
    if case["way"] == "fwd":
        h = case["res_scale"] * v["h"] + case["branch_scale"] * gate * ybar * w_post
        out = {"h": h}
        if case["pre"]:
            out["n"] = h / rms(h) * v["w_pre"]
        return out
    out = {}
    g = v["dh"]
    if case["pre"]:
        g = g + jac(v["h"], v["dn"] * v["w_pre"])
        out["w_pre"] = torch.einsum("td,td->d", v["dn"], v["h"] / rms(v["h"]))
    out["h"] = case["res_scale"] * g
    g = case["branch_scale"] * g
    if v["gate"] is not None:
        full = g * ybar * w_post
        out["gate"] = {"channel": lambda: full.sum(0), "token": lambda: full.sum(1, keepdim=True), "full": lambda: full}[case["gate"]]()
    if case["post"]:
        out["w_post"] = (g * gate * ybar).sum(0)
        out["y"] = jac(v["y"], g * gate * w_post)
    else:
        out["y"] = g * gate
    return out


def _exact_adapter(case, t, offs, ids):
    out = t["base"].double()
    for i, ad in enumerate(ids):
        if ad < 0 or offs[i + 1] == offs[i]:
            continue
        rows = slice(offs[i], offs[i + 1])
        ba = torch.mm(t["b"][ad].double(), t["a"][ad].double())
        out[rows] += t["scale"][ad].double() * torch.mm(t["x"][rows].double(), ba.t().contiguous())
    return out
