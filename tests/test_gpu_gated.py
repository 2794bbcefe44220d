"""The gated feed-forward block and its gradient against the definition in 64 bits: ragged and empty
groups, rows of no group, NaN wherever nothing may be read, offsets past 2^31, streams and graphs."""
import pytest
import torch

import experts_oracle as ref
import paper_2609_05228_amd as ace

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
NAN = float("nan")

# group sizes, rows before the first and behind the last group, M, K
SHAPES = [
    ([1], 0, 0, 8, 8),
    ([1, 1, 1], 0, 1, 64, 64),
    ([0, 3, 0, 0, 5, 0], 2, 4, 72, 136),
    ([16, 17, 15, 33], 0, 0, 128, 64),
    ([0, 0], 3, 0, 40, 24),
    ([65, 1, 0, 130, 63], 1, 70, 136, 200),
    ([257, 3, 256, 255], 0, 9, 264, 72),
    ([300], 0, 0, 520, 328),
    ([5] * 70 + [0] * 60 + [2] * 5, 0, 3, 48, 88),
    ([700, 0, 1, 90], 0, 0, 32, 1032),
    ([2, 0, 1], 0, 0, 1032, 2056),
    ([100] * 9 + [220] * 5, 0, 0, 1096, 72),
    ([37] * 40, 0, 0, 456, 40),
    ([40], 0, 2, 72, 4104),  # the reduction in parts
    # the large shapes by their heights, whole lines and not; of the rows' gradient
    ([150] * 14, 0, 3, 2056, 72),
    ([150] * 12 + [200, 256], 1, 0, 2048, 72),
    ([310] * 9 + [17], 0, 2, 2056, 40),
    ([130] * 20, 2, 0, 40, 2056),
]


def make(sizes, head, tail, M, K, dtype, seed=0):
    """x, w_gate, w_up, da, offsets; NaN and infinities in the rows of no group and the weights of empty groups."""
    gen = torch.Generator().manual_seed(seed + M + K + len(sizes))
    S = head + sum(sizes) + tail
    offs = [head]
    for n in sizes:
        offs.append(offs[-1] + n)
    x, da = (torch.randn((S, n), generator=gen).to(DT[dtype]) for n in (K, M))
    # projections of some size, so that the activation bends
    wg, wu = (torch.randn((len(sizes), M, K), generator=gen).mul(2 * K ** -0.5).to(DT[dtype]) for _ in range(2))
    for t in (x, da):
        t[:head] = NAN
        t[offs[-1]:] = float("inf")
    for e, n in enumerate(sizes):
        if n == 0:
            wg[e] = wu[e] = NAN
    return x, wg, wu, da, torch.tensor(offs, dtype=torch.int32)


def rest(offs, S):
    m = torch.ones(S, dtype=torch.bool)
    m[int(offs[0]):int(offs[-1])] = False
    return m


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: f"{len(s[0])}g_{sum(s[0])}r_{s[3]}x{s[4]}")
def test_forward(shape, dtype, act):
    x, wg, wu, _, offs = make(*shape, dtype)
    d = [t.to(DEV) for t in (x, wg, wu, offs)]
    gap = rest(offs, x.shape[0])
    a = ace.grouped_gated(*d, activation=act)
    a2, (g, u) = ace.grouped_gated(*d, activation=act, keep=True)
    torch.cuda.synchronize()
    want, err = ref.gated(x, wg, wu, offs, act)
    for n, t in (("g", g), ("u", u), ("a", a)):
        ref.within(t[~gap], want[n][~gap], err[n][~gap], DT[dtype], n)
        assert not t[gap].any(), n
    assert torch.equal(a, a2)
    # into given buffers: rows of no group stay, the rest is the same bits
    buf = [torch.full_like(a, 7) for _ in range(3)]
    got = ace.grouped_gated(*d, activation=act, keep=True, out=(buf[0], (buf[1], buf[2])))
    torch.cuda.synchronize()
    assert got[0] is buf[0] and got[1][0] is buf[1] and got[1][1] is buf[2]
    for t, b in zip((a, g, u), buf):
        assert bool((b[gap] == 7).all()) and torch.equal(b[~gap], t[~gap])


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kept", [True, False], ids=["kept", "again"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: f"{len(s[0])}g_{sum(s[0])}r_{s[3]}x{s[4]}")
def test_gradient(shape, kept, dtype, act):
    x, wg, wu, da, offs = make(*shape, dtype)
    gap = rest(offs, x.shape[0])
    keep = None
    if kept:  # as a forward pass leaves them
        want, _ = ref.gated(x, wg, wu, offs, act)
        keep = tuple(want[n].to(DT[dtype]) for n in ("g", "u"))
        for t in keep:
            t[gap] = NAN
    d = [t.to(DEV) for t in (da, x, wg, wu, offs)]
    dk = None if keep is None else tuple(t.to(DEV) for t in keep)
    got = ace.grouped_gated_grad(*d, kept=dk, activation=act)
    only = ace.grouped_gated_grad(d[0], None if kept else d[1], *d[2:], kept=dk, activation=act, weights=False)
    torch.cuda.synchronize()
    assert set(got) == {"x", "w_gate", "w_up"} and set(only) == {"x"}
    want, err = ref.gated_grad(da, x, wg, wu, offs, act, keep, DT[dtype])
    ref.within(got["x"][~gap], want["x"][~gap], err["x"][~gap], DT[dtype], "x")
    assert not got["x"][gap].any()
    for n in ("w_gate", "w_up"):
        ref.within(got[n], want[n], err[n], DT[dtype], n)
    assert torch.equal(got["x"], only["x"])


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("shape", [([3, 0, 40], 1, 2, 12, 20), ([33], 0, 0, 4, 4), ([7] * 30, 0, 1, 68, 132)],
                         ids=lambda s: f"{len(s[0])}g_{s[3]}x{s[4]}")
def test_fp32_in_fours(shape, act):
    """fp32 features come in multiples of four."""
    x, wg, wu, da, offs = make(*shape, "f32")
    gap = rest(offs, x.shape[0])
    d = [t.to(DEV) for t in (x, wg, wu, offs)]
    a, kept = ace.grouped_gated(*d, activation=act, keep=True)
    want, err = ref.gated(x, wg, wu, offs, act)
    for n, t in (("a", a), ("g", kept[0]), ("u", kept[1])):
        ref.within(t[~gap], want[n][~gap], err[n][~gap], torch.float32, n)
    for k in (None, kept):
        got = ace.grouped_gated_grad(da.to(DEV), *d, kept=k, activation=act)
        want, err = ref.gated_grad(da, x, wg, wu, offs, act, None if k is None else tuple(v.cpu() for v in k))
        ref.within(got["x"][~gap], want["x"][~gap], err["x"][~gap], torch.float32, "x")
        for n in ("w_gate", "w_up"):
            ref.within(got[n], want[n], err[n], torch.float32, n)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_no_rows(dtype):
    x, wg, wu, da, offs = make([0, 0, 0], 0, 0, 16, 24, dtype)
    d = [t.to(DEV) for t in (x, wg, wu, da, offs)]
    a, (g, u) = ace.grouped_gated(d[0], d[1], d[2], d[4], keep=True)
    assert a.shape == g.shape == u.shape == (0, 16)
    for kept in (None, (g, u)):
        got = ace.grouped_gated_grad(d[3], d[0], d[1], d[2], d[4], kept=kept)
        torch.cuda.synchronize()
        assert got["x"].shape == (0, 24) and not got["w_gate"].any() and not got["w_up"].any()


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_far_from_zero(dtype, act):
    """Projections from -300 to 300, where the exponentials end: the definition's values, no NaN; slopes 0 and 1 there."""
    S, K = 256, 8
    x = torch.zeros((S, K))
    x[:, 0] = torch.linspace(-300, 300, S)
    x[:, 1] = 1
    x = x.to(DT[dtype])
    wg, wu = torch.zeros((1, 8, K), dtype=DT[dtype]), torch.zeros((1, 8, K), dtype=DT[dtype])
    wg[0, :, 0] = torch.tensor([1, 0.25, 0.0625, 0.03125, -1, 0.1, 0.05, 0.01])
    wu[0, :, 1] = 3
    offs = torch.tensor([0, S], dtype=torch.int32)
    da = torch.ones((S, 8), dtype=DT[dtype])
    d = [t.to(DEV) for t in (x, wg, wu, offs)]
    a = ace.grouped_gated(*d, activation=act)
    got = ace.grouped_gated_grad(da.to(DEV), *d, activation=act)
    want, err = ref.gated(x, wg, wu, offs, act)
    ref.within(a, want["a"], err["a"], DT[dtype], "a")
    want, err = ref.gated_grad(da, x, wg, wu, offs, act, None, DT[dtype])
    for n in want:
        ref.within(got[n], want[n], err[n], DT[dtype], n)


def test_infinities_and_nan_stay_in_their_rows():
    x, wg, wu, da, offs = make([40, 30], 0, 0, 64, 64, "bf16")
    x[3, 5], x[50, 7] = float("inf"), NAN
    d = [t.to(DEV) for t in (x, wg, wu, offs)]
    a = ace.grouped_gated(*d).cpu()
    ok = torch.ones(70, dtype=torch.bool)
    ok[3] = ok[50] = False
    want, err = ref.gated(x, wg, wu, offs, "silu")
    ref.within(a[ok], want["a"][ok], err["a"][ok], torch.bfloat16, "a")
    assert bool(a[50].isnan().all()) and not a[3].isfinite().any()
    got = ace.grouped_gated_grad(da.to(DEV), *d)
    want, err = ref.gated_grad(da, x, wg, wu, offs, "silu", None, torch.bfloat16)
    ref.within(got["x"][ok.to(DEV)], want["x"][ok], err["x"][ok], torch.bfloat16, "dx")


@pytest.mark.parametrize("offs", [[0, 9, 4, 40], [-5, 3, 90, 200], [40, 20, 10, 0], [7, 7, 7, 2 ** 31 - 1],
                                  [-2 ** 31, 2 ** 31 - 1, -2 ** 31, 2 ** 31 - 1]])
def test_bad_offsets_stay_inside(offs):
    """Offsets that do not ascend or leave the array: unspecified results, no write outside."""
    S, M, K, pad = 40, 24, 16, 64
    x, wg, wu, _, _ = make([S, 0, 0], 0, 0, M, K, "bf16")
    wg[1:] = wu[1:] = 0
    o = torch.tensor(offs, dtype=torch.int32, device=DEV)
    d = [t.to(DEV) for t in (x, wg, wu)]
    buf = [torch.full((S * M + 2 * pad,), 5.0, dtype=torch.bfloat16, device=DEV) for _ in range(3)]
    a, g, u = (b[pad:-pad].view(S, M) for b in buf)
    ace.grouped_gated(*d, o, keep=True, out=(a, (g, u)))
    for kept in (None, (g, u)):
        ace.grouped_gated_grad(a, *d, o, kept=kept)
    torch.cuda.synchronize()
    for b in buf:
        assert bool((b[:pad] == 5).all()) and bool((b[-pad:] == 5).all())


def test_offsets_that_go_back_and_forth():
    """2048 groups that each claim the whole array or nothing: no more work than the array is worth."""
    S, N, M, K = 3000, 2048, 24, 16
    gen = torch.Generator(device=DEV).manual_seed(1)
    x, da = (torch.randn((S, n), generator=gen, device=DEV).bfloat16() for n in (K, M))
    wg, wu = (torch.randn((N, M, K), generator=gen, device=DEV).bfloat16() for _ in range(2))
    o = torch.tensor([0, S] * (N // 2) + [0], dtype=torch.int32, device=DEV)
    a, kept = ace.grouped_gated(x, wg, wu, o, keep=True)
    got = ace.grouped_gated_grad(da, x, wg, wu, o, kept=kept)
    torch.cuda.synchronize()
    assert a.shape == (S, M) and got["w_up"].shape == (N, M, K)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_past_two_gib(dtype):
    """Rows whose byte offsets pass 2^32 (and element offsets 2^31), in x and in a, g and u: the last rows are right."""
    n = 300
    gen = torch.Generator(device=DEV).manual_seed(1)
    for K, M in ((2048, 8), (8, 2048)):
        S = (1 << 20) + (1 << 19) + 37
        x = torch.zeros((S, K), dtype=DT[dtype], device=DEV)
        x[-n:], x[:n] = (torch.randn((n, K), generator=gen, device=DEV).to(DT[dtype]) for _ in range(2))
        wg, wu = (torch.randn((2, M, K), generator=gen, device=DEV).mul(K ** -0.5).to(DT[dtype]) for _ in range(2))
        offs = torch.tensor([0, S - 200, S], dtype=torch.int32, device=DEV)
        a, kept = ace.grouped_gated(x, wg, wu, offs, keep=True)
        da = torch.zeros_like(a)
        da[-n:], da[:n] = (torch.randn((n, M), generator=gen, device=DEV).to(DT[dtype]) for _ in range(2))
        got = ace.grouped_gated_grad(da, x, wg, wu, offs, kept=kept)
        torch.cuda.synchronize()
        # the rows that are not zero: n first ones and n last ones, of which 200 are the second group's
        cut = torch.tensor([0, 2 * n - 200, 2 * n], dtype=torch.int32)

        def ends(t):
            return torch.cat([t[:n], t[-n:]]).cpu()

        args = (ends(x), wg.cpu(), wu.cpu(), cut, "silu")
        want, err = ref.gated(*args)
        for name, t in (("a", a), ("g", kept[0]), ("u", kept[1])):
            ref.within(ends(t), want[name], err[name], DT[dtype], name)
            assert not t[n:-n].any(), name
        want, err = ref.gated_grad(ends(da), *args, tuple(ends(t) for t in kept), DT[dtype])
        ref.within(ends(got["x"]), want["x"], err["x"], DT[dtype], "dx")
        assert not got["x"][n:-n].any()
        for name in ("w_gate", "w_up"):
            # the sums run over S rows, zeros but for 2 n of them: as many steps at most
            ref.within(got[name], want[name], err[name], DT[dtype], name)
        del x, a, kept, da, got


def test_gradients_against_differences():
    """<da, a> along a line through the inputs changes as the gradients say (fp32): the slope of the definition in
    64 bits by differences of second order in h, against the kernel's gradients."""
    x, wg, wu, da, offs = make([33, 0, 70, 9], 0, 0, 40, 96, "f32", seed=3)
    wg, wu = torch.nan_to_num(wg), torch.nan_to_num(wu)
    gen = torch.Generator().manual_seed(8)
    dirs = [torch.randn(t.shape, generator=gen).double() for t in (x, wg, wu)]
    d = [t.to(DEV) for t in (x, wg, wu, offs)]
    for act in ("silu", "gelu"):
        kept = ace.grouped_gated(*d, activation=act, keep=True)[1]
        for k in (None, kept):
            got = ace.grouped_gated_grad(da.to(DEV), *d, kept=k, activation=act)
            want, err = ref.gated_grad(da, x, wg, wu, offs, act, None if k is None else tuple(t.cpu() for t in k))
            for i, name in enumerate(("x", "w_gate", "w_up")):
                def loss(h):
                    t = [v.double() + (h * dirs[j] if j == i else 0) for j, v in enumerate((x, wg, wu))]
                    return float((da.double() * ref.gated(*t, offs, act)[0]["a"]).sum())

                h = 2.0 ** -12
                # the fourth-order formula: what it leaves is h^4 / 30 of the fifth derivative
                diff = (8 * (loss(h) - loss(-h)) - (loss(2 * h) - loss(-2 * h))) / (12 * h)
                slope = float((got[name].cpu().double() * dirs[i]).sum())
                # each gradient element within its error and rounding (kept g and u: 2^-24 of them, as much as some sums)
                tol = float(((err[name] + ref.F32 * want[name].abs()) * dirs[i].abs()).sum()) * 2
                assert abs(diff - slope) <= tol, (act, name, diff, slope, tol)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kept", [True, False], ids=["kept", "again"])
def test_streams_graphs_and_repeats(kept, dtype):
    """Equal bits twice, on another stream, and from a captured graph over changed inputs, with eager work between the
    replays; two graphs at once do not disturb each other."""
    x, wg, wu, da, offs = make([30, 0, 5, 200], 0, 3, 72, 520, dtype)
    x[-3:] = 0
    da[-3:] = 0
    d = [t.to(DEV) for t in (x, wg, wu, offs)]
    dd = da.to(DEV)

    def step():
        a, k = ace.grouped_gated(*d, keep=True)
        g = ace.grouped_gated_grad(dd, *d, kept=k if kept else None)
        return [a, *k, g["x"], g["w_gate"], g["w_up"]]

    first = step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        second = step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(first, second))
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = step()
        graphs.append((g, out))
    for i in range(3):
        d[0].mul_(-0.75)
        want = step()
        torch.cuda.synchronize()
        for g, _ in graphs:
            g.replay()
        side.wait_stream(torch.cuda.current_stream())
        torch.cuda.synchronize()
        for _, out in graphs:
            assert all(torch.equal(p, q) for p, q in zip(out, want)), i
