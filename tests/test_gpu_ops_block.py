"""The operators together, as a decoder block that contains the layer uses them: the layer's experts
rebuilt from its plan, a training step through the block, and a decode step captured in a graph."""
import pytest
import torch

import oracle
import paper_2609_05228_amd as ace
import synth
from gpu_helpers import DEV, TDT, device_layer, rel_l2

pytestmark = pytest.mark.gpu


def plan_of(o):
    """Rows of the plan: their tokens, their experts, their gates."""
    n = int(o["offsets"][-1])
    tok = o["perm"][:n].long()
    exp = torch.repeat_interleave(torch.arange(o["counts"].numel(), device=tok.device), o["counts"].long())
    slot = (o["topk_idx"].long()[tok] == exp[:, None]).float().argmax(dim=1)
    return tok, exp, o["gates"][tok, slot]


def layer_of(dtype, T=300, d=256, N=16, k=4, m=192, seed=11):
    L = synth.make_layer(synth.config("prefill_4096", T=T, d=d, N=N, k=k, m=m, dtype=dtype, seed=seed))
    tb = oracle.tables.build_tables(L)
    D = device_layer(L)
    tabs = [torch.from_numpy(tb[n]).to(DEV) for n in ("a_gsp", "a_rcr")]
    return L, D, tabs


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [3, 300])
def test_experts_from_the_plan(T, dtype):
    """Norm, gather, three grouped products and the gates give moe_forward's y, to the bars that its own
    tests hold it to (bf16: gate and up projections are rounded here, which the layer does not do)."""
    L, D, tabs = layer_of(dtype, T=T)
    o = ace.moe_forward(D["x"], D, *tabs, k=4, tau=0.2, want_plan=True)
    tok, exp, gates = plan_of(o)
    assert T <= len(tok) <= 4 * T
    rows = ace.block_norm(D["x"], w_pre=D["gamma"])["n"][tok]
    g, u = (ace.grouped_matmul(rows, D[n], o["offsets"]) for n in ("w_gate", "w_up"))
    H = (torch.nn.functional.silu(g.float()) * u.float()).to(g.dtype)
    Y = ace.grouped_matmul(H, D["w_down"], o["offsets"])
    y = torch.zeros((T, 256), device=DEV).index_add_(0, tok, Y.float() * gates[:, None])
    a, b = y.cpu().double().numpy(), o["y"].float().cpu().double().numpy()
    assert rel_l2(a, b) <= (1e-5 if dtype == "f32" else 1e-2)


def test_a_training_step():
    """Gradients of a block (norm, experts, gates, post-norm, gate, residual, next norm) by the operators'
    gradients, against autograd in 64 bits with the same routing."""
    L, D, tabs = layer_of("f32")
    T, d, m, N = 300, 256, 192, 16
    o = ace.moe_forward(D["x"], D, *tabs, k=4, tau=0.2, want_plan=True)
    tok, exp, gates = plan_of(o)
    offs = o["offsets"]
    gen = torch.Generator(device=DEV).manual_seed(3)
    w_post, w_pre, gate = (1 + 0.2 * torch.randn(d, generator=gen, device=DEV) for _ in range(3))
    dh, dn = (torch.randn((T, d), generator=gen, device=DEV) for _ in range(2))
    kw = dict(res_scale=0.9, branch_scale=0.7)
    silu = torch.nn.functional.silu
    # forward
    x = D["x"]
    rows = ace.block_norm(x, w_pre=D["gamma"])["n"][tok]
    g, u = (ace.grouped_matmul(rows, D[n], offs) for n in ("w_gate", "w_up"))
    H = silu(g) * u
    Y = ace.grouped_matmul(H, D["w_down"], offs)
    y = torch.zeros((T, d), device=DEV).index_add_(0, tok, Y * gates[:, None])
    out = ace.block_norm(x, y, w_post=w_post, w_pre=w_pre, gate=gate, **kw)
    # backward
    gr = ace.block_norm_grad(dh, dn, out["h"], y, w_post=w_post, w_pre=w_pre, gate=gate, **kw)
    dY = (gr["y"][tok] * gates[:, None]).contiguous()
    dH = ace.grouped_matmul_grad_x(dY, D["w_down"], offs)
    s = torch.sigmoid(g)
    dg, du = (dH * u * s * (1 + g * (1 - s))).contiguous(), (dH * silu(g)).contiguous()
    drows = ace.grouped_matmul_grad_x(dg, D["w_gate"], offs) + ace.grouped_matmul_grad_x(du, D["w_up"], offs)
    dxn = torch.zeros((T, d), device=DEV).index_add_(0, tok, drows)
    first = ace.block_norm_grad(None, dxn, x, w_pre=D["gamma"])
    got = dict(x=gr["h"] + first["h"], gamma=first["w_pre"], w_post=gr["w_post"], w_pre=gr["w_pre"], gate=gr["gate"],
               w_gate=ace.grouped_matmul_grad_w(dg, rows, offs), w_up=ace.grouped_matmul_grad_w(du, rows, offs),
               w_down=ace.grouped_matmul_grad_w(dY, H, offs))
    # 64 bits
    p = {n: D[n].cpu().double().requires_grad_() for n in ("x", "gamma", "w_gate", "w_up", "w_down")}
    p.update({n: v.cpu().double().requires_grad_() for n, v in (("w_post", w_post), ("w_pre", w_pre), ("gate", gate))})
    tc, ec, gc = tok.cpu(), exp.cpu(), gates.cpu().double()

    def norm(v, w):
        return v / (v.square().mean(1, keepdim=True) + 1e-6).sqrt() * w

    r = norm(p["x"], p["gamma"])[tc]
    hh = silu(torch.einsum("rd,rmd->rm", r, p["w_gate"][ec])) * torch.einsum("rd,rmd->rm", r, p["w_up"][ec])
    yy = torch.zeros((T, d), dtype=torch.float64).index_add(0, tc, torch.einsum("rm,rdm->rd", hh, p["w_down"][ec]) * gc[:, None])
    h2 = 0.9 * p["x"] + 0.7 * p["gate"] * norm(yy, p["w_post"])
    (h2 * dh.cpu().double()).sum().add((norm(h2, p["w_pre"]) * dn.cpu().double()).sum()).backward()
    for n, v in got.items():
        # chains of up to eight fp32 operations, each within some 1e-7 of its result, as the layer's own bar
        assert rel_l2(v.cpu().double().numpy(), p[n].grad.numpy()) <= 1e-5, n


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_captured_decode_step(dtype):
    """Norm, shared projection with adapters, the layer, and the norm behind it in one graph: every replay
    gives the eager call's bits on the tokens then in the buffers."""
    L, D, tabs = layer_of(dtype, T=12)
    T, d = 12, 256
    gen = torch.Generator(device=DEV).manual_seed(9)
    dt = TDT[dtype]

    def n(*shape, std=1.0, mean=0.0):
        return (torch.randn(shape, generator=gen, device=DEV) * std + mean).to(dt)

    w1, w2, gate = (n(d, std=0.1, mean=1.0) for _ in range(3))
    proj, a, b = n(1, d, d, std=d ** -0.5), n(3, 16, d, std=d ** -0.5), n(3, d, 16, std=0.1)
    whole = torch.tensor([0, T], dtype=torch.int32, device=DEV)
    offs = torch.tensor([0, 1, 2, 5, 5, 12], dtype=torch.int32, device=DEV)
    ids = torch.tensor([2, -1, 0, 1, 2], dtype=torch.int32, device=DEV)
    h = D["x"].clone()

    def step():
        xn = ace.block_norm(h, w_pre=w1)["n"]
        mixed = ace.adapter_add(ace.grouped_matmul(xn, proj, whole), xn, a, b, offs, ids)
        mid = ace.block_norm(h, mixed, w_post=w2)["h"]
        y = ace.moe_forward(mid, D, *tabs, k=4, tau=0.2)["y"]
        return ace.block_norm(mid, y, w_pre=w2, gate=gate, branch_scale=0.5)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = step()
    for i in range(4):
        h.copy_(n(T, d))
        want = step()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out["h"], want["h"]) and torch.equal(out["n"], want["n"]), i
        assert bool(out["h"].isfinite().all())
