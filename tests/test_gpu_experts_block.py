"""The experts' operators together, as a layer that is trained or served in 4 bits uses them: on the plan that the layer
returns, with the rows that it leaves unused behind the last expert."""
import pytest
import torch

import oracle
import paper_2609_05228_amd as ace
import synth
from gpu_helpers import DEV, device_layer, rel_l2

pytestmark = pytest.mark.gpu

T, D, N, K, M = 300, 256, 16, 4, 192


def layer_of(dtype, tokens=T):
    L = synth.make_layer(synth.config("prefill_4096", T=tokens, d=D, N=N, k=K, m=M, dtype=dtype, seed=12))
    tb = oracle.tables.build_tables(L)
    return device_layer(L), [torch.from_numpy(tb[n]).to(DEV) for n in ("a_gsp", "a_rcr")]


def routed(x, L, tabs, weights=None):
    """The layer's call; token, expert and gate of all T k rows: those past the plan name token 0 with gate 0."""
    o = ace.moe_forward(x, L if weights is None else {**L, **weights}, *tabs, k=K, tau=0.2, want_plan=True)
    rows = torch.arange(x.shape[0] * K, device=DEV)
    used = rows < o["offsets"][-1]
    tok = torch.where(used, o["perm"].long(), 0).clamp(0, x.shape[0] - 1)
    exp = torch.searchsorted(o["offsets"][1:].long(), rows, right=True).clamp(max=N - 1)
    slot = (o["topk_idx"].long()[tok] == exp[:, None]).float().argmax(dim=1)
    return o, tok, torch.where(used, o["gates"][tok, slot], 0.0)


def combined(Y, tok, gates, tokens):
    # the rows of no expert hold zeros; their gate is zero too
    return torch.zeros((tokens, D), device=DEV).index_add_(0, tok, Y.float() * gates[:, None])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tokens", [1, 3, T])
def test_the_layer_from_the_gated_block(tokens, dtype):
    """Norm, gather, gated block, down projection and gates give moe_forward's y, to the bars of its own tests."""
    L, tabs = layer_of(dtype, tokens)
    o, tok, gates = routed(L["x"], L, tabs)
    rows = ace.block_norm(L["x"], w_pre=L["gamma"])["n"][tok]
    H = ace.grouped_gated(rows, L["w_gate"], L["w_up"], o["offsets"])
    y = combined(ace.grouped_matmul(H, L["w_down"], o["offsets"]), tok, gates, tokens)
    a, b = y.cpu().double().numpy(), o["y"].float().cpu().double().numpy()
    assert rel_l2(a, b) <= (1e-5 if dtype == "f32" else 1e-2)


@pytest.mark.parametrize("again", [False, True], ids=["kept", "again"])
def test_a_training_step(again):
    """Gradients of the experts and their input through both products, against autograd in 64 bits."""
    L, tabs = layer_of("f32")
    o, tok, gates = routed(L["x"], L, tabs)
    offs = o["offsets"]
    n = int(offs[-1])
    gen = torch.Generator(device=DEV).manual_seed(4)
    dy = torch.randn((T, D), generator=gen, device=DEV)
    rows = ace.block_norm(L["x"], w_pre=L["gamma"])["n"][tok]
    H, kept = ace.grouped_gated(rows, L["w_gate"], L["w_up"], offs, keep=True)
    # backward of y = sum of gates * down(H)
    dY = (dy[tok] * gates[:, None]).contiguous()
    dH = ace.grouped_matmul_grad_x(dY, L["w_down"], offs)
    g = ace.grouped_gated_grad(dH, rows, L["w_gate"], L["w_up"], offs, kept=None if again else kept)
    dxn = torch.zeros((T, D), device=DEV).index_add_(0, tok, g["x"])
    first = ace.block_norm_grad(None, dxn, L["x"], w_pre=L["gamma"])
    got = dict(x=first["h"], gamma=first["w_pre"], w_gate=g["w_gate"], w_up=g["w_up"],
               w_down=ace.grouped_matmul_grad_w(dY, H, offs))
    p = {k: L[k].cpu().double().requires_grad_() for k in ("x", "gamma", "w_gate", "w_up", "w_down")}
    tc, gc = tok[:n].cpu(), gates[:n].cpu().double()
    ec = torch.repeat_interleave(torch.arange(N), o["counts"].cpu().long())
    x = p["x"]
    r = (x / (x.square().mean(1, keepdim=True) + 1e-6).sqrt() * p["gamma"])[tc]
    hh = torch.nn.functional.silu(torch.einsum("rd,rmd->rm", r, p["w_gate"][ec])) * torch.einsum("rd,rmd->rm", r, p["w_up"][ec])
    yy = torch.zeros((T, D), dtype=torch.float64).index_add(0, tc, torch.einsum("rm,rdm->rd", hh, p["w_down"][ec]) * gc[:, None])
    (yy * dy.cpu().double()).sum().backward()
    for k, v in got.items():
        # chains of up to six fp32 operations, each within some 1e-7 of its result, as the layer's own bar
        assert rel_l2(v.cpu().double().numpy(), p[k].grad.numpy()) <= 1e-5, k


def quantized(L):
    q = {k: ace.mx4_quantize(L[k]) for k in ("w_gate", "w_up", "w_down")}
    return q, {k: ace.mx4_dequantize(v) for k, v in q.items()}


@pytest.mark.parametrize("tokens", [1, 3, T])
def test_the_layer_on_weights_in_4_bits(tokens):
    """The layer on the values that the 4-bit weights stand for, and its experts from the 4-bit operators."""
    L, tabs = layer_of("bf16", tokens)
    q, values = quantized(L)
    o, tok, gates = routed(L["x"], L, tabs, values)
    rows = ace.block_norm(L["x"], w_pre=L["gamma"])["n"][tok]
    H = ace.grouped_gated(rows, q["w_gate"], q["w_up"], o["offsets"])
    y = combined(ace.grouped_matmul(H, q["w_down"], o["offsets"]), tok, gates, tokens)
    assert rel_l2(y.cpu().double().numpy(), o["y"].float().cpu().double().numpy()) <= 1e-2


def test_rows_in_4_bits_too():
    """Both products on rows that are quantised in between, against the same products of the values in bf16."""
    L, tabs = layer_of("bf16")
    q, values = quantized(L)
    o, tok, _ = routed(L["x"], L, tabs, values)
    offs, n = o["offsets"], int(o["offsets"][-1])
    rows = ace.mx4_quantize(ace.block_norm(L["x"], w_pre=L["gamma"])["n"][tok])
    H = ace.grouped_gated(rows, q["w_gate"], q["w_up"], offs)
    Y = ace.grouped_matmul(ace.mx4_quantize(H), q["w_down"], offs)
    H2 = ace.grouped_gated(ace.mx4_dequantize(rows), values["w_gate"], values["w_up"], offs)
    # exact products, fp32 sums and one rounding on both sides
    assert rel_l2(H[:n].float().cpu().numpy(), H2[:n].float().cpu().numpy()) <= 2.0 ** -8
    Y2 = ace.grouped_matmul(ace.mx4_dequantize(ace.mx4_quantize(H)), values["w_down"], offs)
    assert rel_l2(Y[:n].float().cpu().numpy(), Y2[:n].float().cpu().numpy()) <= 2.0 ** -8
    assert not Y[n:].any() and not H[n:].any()


def test_a_captured_decode_step_in_4_bits():
    """Norm, routing, gather, both 4-bit products and the sum over slots in one graph: every replay gives the eager
    call's bits on the tokens then in the buffer, however many rows the plan then holds."""
    L, tabs = layer_of("bf16", 12)
    q, _ = quantized(L)
    x = L["x"].clone()

    def step():
        o, tok, gates = routed(x, L, tabs)
        rows = ace.block_norm(x, w_pre=L["gamma"])["n"][tok]
        H = ace.grouped_gated(rows, q["w_gate"], q["w_up"], o["offsets"])
        return ace.grouped_matmul(H, q["w_down"], o["offsets"]), H, o["offsets"]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = step()
    gen = torch.Generator(device=DEV).manual_seed(9)
    for i in range(4):
        x.copy_(torch.randn(x.shape, generator=gen, device=DEV) * (0.1 + i))
        want = step()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)), i
        assert bool(out[0].isfinite().all()) and bool(out[0].any())
