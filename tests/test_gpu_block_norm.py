"""The norms before and after a block, and their gradients, against the definition in 64 bits."""
import itertools

import pytest
import torch

import ops_oracle as ref
import paper_2609_05228_amd as ace

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
# fp32 operations on a result's terms: a sum over a row is at most 26 deep (16 elements in a
# thread, 6 steps in a wave, 4 over the waves), one over the rows of these cases at most 50 (2 rows of a
# thread, 16 of a workgroup, 16 lines of a wave, 16 waves), and some 10 more form a result from them
TERMS = 64

SIZES = [(1, 8), (1, 2048), (3, 64), (7, 520), (5, 1032), (2, 4096), (3, 4104), (2, 8192), (2, 16384), (515, 264), (9, 1288), (70, 2200), (5, 4888), (40, 648)]


def make(T, d, dtype, gate="channel", post=True, pre=True, seed=0):
    gen = torch.Generator().manual_seed(seed + T + d)

    def n(shape, std=1.0, mean=0.0):
        return (torch.randn(shape, generator=gen) * std + mean).to(DT[dtype])

    t = dict(h=n((T, d), 2.0), y=n((T, d), 0.7), w_post=n((d,), 0.1, 1.0) if post else None,
             w_pre=n((d,), 0.1, 1.0) if pre else None, gate=None)
    if gate != "none":
        t["gate"] = n({"channel": (d,), "token": (T, 1), "full": (T, d)}[gate], 0.5, 0.5)
    return t, n((T, d)), n((T, d)) if pre else None


def dev(t):
    return {k: None if v is None else v.to(DEV) for k, v in t.items()}


def check(got, want, mag, dtype, name):
    assert set(got) == set(want), name
    for k in want:
        ref.close(got[k], want[k], mag[k], DT[dtype], TERMS, f"{name} {k}")


def both(t, dh, dn, dtype, **kw):
    g = dev(t)
    out = ace.block_norm(**g, **kw)
    want, mag = ref.block_norm(**t, **kw)
    torch.cuda.synchronize()
    check(out, want, mag, dtype, "forward")
    stored = out["h"].cpu()
    got = ace.block_norm_grad(None if dh is None else dh.to(DEV), None if dn is None else dn.to(DEV),
                              **dict(g, h=out["h"]), **kw)
    torch.cuda.synchronize()
    want, mag = ref.block_norm_grad(dh, dn, **dict(t, h=stored), **kw)
    check(got, want, mag, dtype, "gradient")
    return out, got


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,d", SIZES)
def test_sizes(T, d, dtype):
    t, dh, dn = make(T, d, dtype)
    both(t, dh, dn, dtype, res_scale=0.75, branch_scale=0.3)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("post,pre,gate", list(itertools.product([True, False], [True, False],
                                                                 ["none", "channel", "token", "full"])))
def test_forms(post, pre, gate, dtype):
    t, dh, dn = make(9, 136, dtype, gate, post, pre)
    both(t, dh, dn, dtype, eps=1e-5)
    if pre:
        both(t, None, dn, dtype, branch_scale=-2.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,d", [(4200, 72), (1100, 1032), (530, 4104), (300, 8192), (1500, 1288), (800, 2320), (2700, 648)])
def test_more_rows_than_one_round(T, d, dtype):
    """Workgroups that take several rows one after the other, the next ones copied ahead."""
    t, dh, dn = make(T, d, dtype)
    both(t, dh, dn, dtype, res_scale=1.25, branch_scale=-0.5)


@pytest.mark.parametrize("post,pre,gate", list(itertools.product([True, False], [True, False],
                                                                 ["none", "channel", "token", "full"])))
def test_forms_of_several_rows(post, pre, gate):
    """The gradients of each form store differently many results behind the copies they wait for."""
    t, dh, dn = make(9000, 40, "bf16", gate, post, pre)
    both(t, dh, dn, "bf16")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_norm_before_the_first_block(dtype):
    t, dh, dn = make(11, 264, dtype)
    t = dict(h=t["h"], y=None, w_post=None, w_pre=t["w_pre"], gate=None)
    out, _ = both(t, dh, dn, dtype)
    h = t["h"].to(DEV)
    out = ace.block_norm(h, w_pre=t["w_pre"].to(DEV))
    assert out["h"] is h and torch.equal(h.cpu(), t["h"])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_of_zeros_and_of_extremes(dtype):
    """A row of zeros, a tiny one and a large one: the statistics stay finite."""
    t, dh, dn = make(6, 72, dtype)
    for k in ("h", "y"):
        t[k][0] = 0
        t[k][1] *= 1e-12
        t[k][2] *= 1e15
    dh[3] = 0
    dn[3] = 0
    both(t, dh, dn, dtype)


def test_a_nan_stays_in_its_row():
    t, dh, dn = make(8, 64, "f32", "token")
    t["y"][5, 3] = float("nan")
    out = ace.block_norm(**dev(t))
    g = ace.block_norm_grad(dh.to(DEV), dn.to(DEV), **dict(dev(t), h=out["h"]))
    for v in (out["h"], out["n"], g["h"], g["y"]):
        assert bool(v[5].isnan().any()) and not bool(v[torch.arange(8) != 5].isnan().any())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_results_on_their_inputs(dtype):
    t, dh, dn = make(33, 264, dtype, "full")
    want = ace.block_norm(**dev(t))
    g = dev(t)
    out = ace.block_norm(**g, out={"h": g["h"], "n": g["y"]})
    assert out["h"] is g["h"] and out["n"] is g["y"]
    assert torch.equal(out["h"], want["h"]) and torch.equal(out["n"], want["n"])


def test_no_rows():
    t, dh, dn = make(0, 64, "bf16")
    out = ace.block_norm(**dev(t))
    assert out["h"].shape == (0, 64) and out["n"].shape == (0, 64)
    for gate in ("channel", "token", "full", "none"):
        t, dh, dn = make(0, 64, "bf16", gate)
        g = ace.block_norm_grad(dh.to(DEV), dn.to(DEV), **dev(t))
        torch.cuda.synchronize()
        assert not g["w_post"].any() and not g["w_pre"].any() and g["y"].shape == (0, 64)
        if gate == "channel":
            assert not g["gate"].any()


def test_rows_past_four_gib():
    """T d of 2^31 elements and some: the last rows, and sums over all of them."""
    T, d = (1 << 20) + 5, 2048
    h = torch.zeros((T, d), dtype=torch.bfloat16, device=DEV)
    y = torch.zeros_like(h)
    gen = torch.Generator(device=DEV).manual_seed(2)
    h[-7:] = torch.randn((7, d), generator=gen, device=DEV).bfloat16()
    y[-7:] = torch.randn((7, d), generator=gen, device=DEV).bfloat16()
    w = torch.ones(d, dtype=torch.bfloat16, device=DEV)
    out = ace.block_norm(h, y, w_post=w, w_pre=w)
    g = ace.block_norm_grad(h, y, out["h"], y, w_post=w, w_pre=w)
    torch.cuda.synchronize()
    hs, ys, ws = h[-7:].cpu(), y[-7:].cpu(), w.cpu()
    want, mag = ref.block_norm(hs, ys, ws, ws)
    check({k: v[-7:] for k, v in out.items()}, want, mag, "bf16", "forward")
    want, mag = ref.block_norm_grad(hs, ys, out["h"][-7:].cpu(), ys, ws, ws)
    check({k: v[-7:] if v.dim() == 2 else v for k, v in g.items()}, want, mag, "bf16", "gradient")
    assert not out["h"][:-7].any() and not g["y"][:-7].any()


@pytest.mark.parametrize("gate", ["channel", "token", "full"])
def test_gradients_against_differences(gate):
    """Central differences of the definition along random directions."""
    t, dh, dn = make(6, 40, "f32", gate)
    kw = dict(res_scale=0.8, branch_scale=0.6)
    t = {k: v.double() for k, v in t.items()}
    x32 = {k: v.float().to(DEV) for k, v in t.items()}
    h1 = ref.block_norm(**t, **kw)[0]["h"]
    got = ace.block_norm_grad(dh.to(DEV), dn.to(DEV), **dict(x32, h=h1.float().to(DEV)), **kw)
    gen = torch.Generator().manual_seed(5)
    for name in ("h", "y", "w_post", "w_pre", "gate"):
        v = torch.randn(t[name].shape, generator=gen, dtype=torch.float64)

        def loss(s):
            o = ref.block_norm(**dict(t, **{name: t[name] + s * v}), **kw)[0]
            return float((o["h"] * dh.double()).sum() + (o["n"] * dn.double()).sum())

        e = 1e-5  # the difference is off by some e^2 and 1e-16 / e, relative
        diff = (loss(e) - loss(-e)) / (2 * e)
        grad = got[name].cpu().double()
        # and the gradient by TERMS fp32 operations on terms that cancel by no more than 100 here
        tol = 100 * TERMS * 2 * ref.F32 * float((grad * v).abs().sum()) + 1e-7
        assert abs(diff - float((grad * v).sum())) <= tol, (name, diff, float((grad * v).sum()))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_streams_graphs_and_repeats(dtype):
    t, dh, dn = make(700, 520, dtype)
    g, dh, dn = dev(t), dh.to(DEV), dn.to(DEV)

    def step():
        out = ace.block_norm(**g)
        return {**out, **{"d" + k: v for k, v in ace.block_norm_grad(dh, dn, **dict(g, h=out["h"])).items()}}

    want = step()
    torch.cuda.synchronize()

    def same(got):
        torch.cuda.synchronize()
        for k in want:
            assert torch.equal(got[k], want[k]), k

    same(step())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = step()
    same(got)
    graphs = []
    for _ in range(2):  # two graphs, replayed at once on two streams
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            got = step()
        graphs.append((gr, got))
    for _ in range(3):
        for _, got in graphs:
            for v in got.values():
                v.fill_(3)
        torch.cuda.synchronize()
        streams = [torch.cuda.Stream() for _ in graphs]
        for (gr, _), s in zip(graphs, streams):
            with torch.cuda.stream(s):
                gr.replay()
        for _, got in graphs:
            same(got)
        same(step())
