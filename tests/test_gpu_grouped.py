"""Grouped matrix products and their gradients against the definition in 64 bits: ragged and
empty groups, rows of no group, NaN wherever nothing may be read, offsets past 2^31."""
import pytest
import torch

import ops_oracle as ref
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
]


def make(sizes, head, tail, M, K, dtype, seed=0):
    """x, w, dy, offsets; NaN in the rows of no group and the weights of empty groups."""
    gen = torch.Generator().manual_seed(seed + M + K + len(sizes))
    S = head + sum(sizes) + tail
    offs = [head]
    for n in sizes:
        offs.append(offs[-1] + n)
    x = torch.randn((S, K), generator=gen).to(DT[dtype])
    w = (torch.randn((len(sizes), M, K), generator=gen) * K ** -0.5).to(DT[dtype])
    dy = torch.randn((S, M), generator=gen).to(DT[dtype])
    for t in (x, dy):
        t[:head] = NAN
        t[offs[-1]:] = float("inf")
    for e, n in enumerate(sizes):
        if n == 0:
            w[e] = NAN
    return x, w, dy, torch.tensor(offs, dtype=torch.int32)


def rest(offs, S):
    m = torch.ones(S, dtype=torch.bool)
    m[int(offs[0]):int(offs[-1])] = False
    return m


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: f"{len(s[0])}g_{sum(s[0])}r_{s[3]}x{s[4]}")
def test_against_the_definition(shape, dtype):
    x, w, dy, offs = make(*shape, dtype)
    S, M, K = x.shape[0], w.shape[1], w.shape[2]
    gap = rest(offs, S)
    d = [t.to(DEV) for t in (x, w, dy, offs)]
    y = ace.grouped_matmul(d[0], d[1], d[3])
    dx = ace.grouped_matmul_grad_x(d[2], d[1], d[3])
    dw = ace.grouped_matmul_grad_w(d[2], d[0], d[3])
    torch.cuda.synchronize()
    want, mag = ref.grouped(x, w, offs)
    ref.close(y, want, mag, DT[dtype], K, "y")
    want, mag = ref.grouped(dy, w.transpose(1, 2), offs)
    ref.close(dx, want, mag, DT[dtype], M, "dx")
    want, mag = ref.grouped_grad_w(dy, x, offs)
    ref.close(dw, want, mag, DT[dtype], max(max(shape[0]), 1), "dw")
    assert not y[gap].any() and not dx[gap].any()
    # into given buffers: rows of no group stay, the rest is the same bits
    y2, dx2, dw2 = torch.full_like(y, 7), torch.full_like(dx, 7), torch.full_like(dw, NAN)
    assert ace.grouped_matmul(d[0], d[1], d[3], out=y2) is y2
    ace.grouped_matmul_grad_x(d[2], d[1], d[3], out=dx2)
    ace.grouped_matmul_grad_w(d[2], d[0], d[3], out=dw2)
    torch.cuda.synchronize()
    assert bool((y2[gap] == 7).all()) and bool((dx2[gap] == 7).all())
    assert torch.equal(y2[~gap], y[~gap]) and torch.equal(dx2[~gap], dx[~gap]) and torch.equal(dw2, dw)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_no_rows(dtype):
    x, w, dy, offs = make([0, 0, 0], 0, 0, 16, 24, dtype)
    d = [t.to(DEV) for t in (x, w, dy, offs)]
    assert ace.grouped_matmul(d[0], d[1], d[3]).shape == (0, 16)
    assert ace.grouped_matmul_grad_x(d[2], d[1], d[3]).shape == (0, 24)
    dw = ace.grouped_matmul_grad_w(d[2], d[0], d[3], out=torch.full((3, 16, 24), NAN, dtype=DT[dtype], device=DEV))
    torch.cuda.synchronize()
    assert not dw.any()


def test_infinities_stay_in_their_rows():
    """An infinity in a row reaches that row's products (and its group's gradient) alone."""
    x, w, dy, offs = make([40, 30], 0, 0, 64, 64, "bf16")
    x[3, 5] = float("inf")
    d = [t.to(DEV) for t in (x, w, dy, offs)]
    y = ace.grouped_matmul(d[0], d[1], d[3]).cpu()
    dw = ace.grouped_matmul_grad_w(d[2], d[0], d[3]).cpu()
    want, mag = ref.grouped(x, w, offs)
    keep = torch.arange(70) != 3
    ref.close(y[keep], want[keep], mag[keep], torch.bfloat16, 64, "y")
    assert torch.equal(y[3].isinf(), want[3].isinf())
    want, mag = ref.grouped_grad_w(dy, x, offs)
    cols = torch.arange(64) != 5
    ref.close(dw[:, :, cols], want[:, :, cols], mag[:, :, cols], torch.bfloat16, 40, "dw")
    ref.close(dw[1], want[1], mag[1], torch.bfloat16, 40, "dw of the other group")


@pytest.mark.parametrize("offs", [[0, 9, 4, 40], [-5, 3, 90, 200], [40, 20, 10, 0], [7, 7, 7, 2 ** 31 - 1],
                                  [-2 ** 31, 2 ** 31 - 1, -2 ** 31, 2 ** 31 - 1]])
def test_bad_offsets_stay_inside(offs):
    """Offsets that do not ascend or leave the array: unspecified results, no write outside."""
    S, M, K = 40, 24, 16
    x, w, dy, _ = make([S, 0, 0], 0, 0, M, K, "bf16")
    w[1:] = 0
    o = torch.tensor(offs, dtype=torch.int32, device=DEV)
    d = [t.to(DEV) for t in (x, w, dy)]
    pad = 64
    for fn, a, b, shape in ((ace.grouped_matmul, d[0], d[1], (S, M)), (ace.grouped_matmul_grad_x, d[2], d[1], (S, K)),
                            (ace.grouped_matmul_grad_w, d[2], d[0], (3, M, K))):
        n = torch.Size(shape).numel()
        buf = torch.full((n + 2 * pad,), 5.0, dtype=torch.bfloat16, device=DEV)
        fn(a, b, o, out=buf[pad:pad + n].view(shape))
        torch.cuda.synchronize()
        assert bool((buf[:pad] == 5).all()) and bool((buf[-pad:] == 5).all())


def test_offsets_that_go_back_and_forth():
    """4096 groups that each claim the whole array or nothing: no more work than the array is worth."""
    S, N, M, K = 3000, 4096, 24, 16
    gen = torch.Generator(device=DEV).manual_seed(1)
    x = torch.randn((S, K), generator=gen, device=DEV).bfloat16()
    w = torch.randn((N, M, K), generator=gen, device=DEV).bfloat16()
    dy = torch.randn((S, M), generator=gen, device=DEV).bfloat16()
    o = torch.tensor([0, S] * (N // 2) + [0], dtype=torch.int32, device=DEV)
    assert ace.grouped_matmul(x, w, o).shape == (S, M)
    assert ace.grouped_matmul_grad_x(dy, w, o).shape == (S, K)
    assert ace.grouped_matmul_grad_w(dy, x, o).shape == (N, M, K)
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_past_two_gib(dtype):
    """Rows whose byte offsets pass 2^32 (and element offsets 2^31): the last rows are right."""
    K, M = 2048, 8
    S = (1 << 20) + (1 << 19) + 37  # 1.6M rows x 2048
    x = torch.zeros((S, K), dtype=DT[dtype], device=DEV)
    gen = torch.Generator(device=DEV).manual_seed(1)
    n = 300
    x[-n:] = torch.randn((n, K), generator=gen, device=DEV).to(DT[dtype])
    x[:n] = torch.randn((n, K), generator=gen, device=DEV).to(DT[dtype])
    w = torch.randn((2, M, K), generator=gen, device=DEV).to(DT[dtype])
    offs = torch.tensor([0, S - 200, S], dtype=torch.int32, device=DEV)
    y = ace.grouped_matmul(x, w, offs)
    dy = torch.zeros((S, M), dtype=DT[dtype], device=DEV)
    dy[-n:] = y[-n:]
    dy[:n] = y[:n]
    dx = ace.grouped_matmul_grad_x(dy, w, offs)
    dw = ace.grouped_matmul_grad_w(dy, x, offs)
    torch.cuda.synchronize()
    # the rows that are not zero: n first ones and n last ones, of which 200 are the second group's
    cut = torch.tensor([0, 2 * n - 200, 2 * n], dtype=torch.int32)
    xs, dys = torch.cat([x[:n], x[-n:]]).cpu(), torch.cat([dy[:n], dy[-n:]]).cpu()
    want, mag = ref.grouped(xs, w.cpu(), cut)
    ref.close(torch.cat([y[:n], y[-n:]]), want, mag, DT[dtype], K, "y")
    assert not y[n:-n].any() and not dx[n:-n].any()
    want, mag = ref.grouped(dys, w.cpu().transpose(1, 2), cut)
    ref.close(torch.cat([dx[:n], dx[-n:]]), want, mag, DT[dtype], M, "dx")
    want, mag = ref.grouped_grad_w(dys, xs, cut)
    ref.close(dw, want, mag, DT[dtype], 2 * n, "dw")


def test_gradients_against_differences():
    """<dy, y(x + t v)> changes with t as <dx, v> says, and the same for the weights (fp32; the
    function is linear in each, so the difference is exact up to the operator's own rounding)."""
    x, w, dy, offs = make([33, 0, 70, 9], 0, 0, 40, 96, "f32", seed=3)
    w = torch.nan_to_num(w)
    gen = torch.Generator().manual_seed(8)
    v, u = torch.randn(x.shape, generator=gen), torch.randn(w.shape, generator=gen)
    d = [t.to(DEV) for t in (x, w, dy, offs)]
    dx = ace.grouped_matmul_grad_x(d[2], d[1], d[3]).cpu().double()
    dw = ace.grouped_matmul_grad_w(d[2], d[0], d[3]).cpu().double()

    def loss(a, b):
        return float((dy.double() * ref.grouped(a, b, offs)[0]).sum())

    h = 2.0 ** -10
    for grad, dirn, f in ((dx, v, lambda s: loss(x.double() + s * v.double(), w)), (dw, u, lambda s: loss(x, w.double() + s * u.double()))):
        diff = (f(h) - f(-h)) / (2 * h)
        want = float((grad * dirn.double()).sum())
        # each gradient element is off by at most 96 fp32 operations on its terms
        tol = 2 * 96 * ref.F32 * float((grad.abs() * dirn.double().abs()).sum()) * 40
        assert abs(diff - want) <= tol, (diff, want, tol)


@pytest.mark.parametrize("fn", ["fwd", "grad_x", "grad_w"])
def test_streams_graphs_and_repeats(fn):
    """The same bits again, on another stream, and from a graph replayed between eager work."""
    x, w, dy, offs = make([70, 0, 3, 200], 0, 5, 136, 264, "bf16")
    x, dy = torch.nan_to_num(x, 0, 0, 0), torch.nan_to_num(dy, 0, 0, 0)
    d = [t.to(DEV) for t in (x, torch.nan_to_num(w), dy, offs)]
    a, b, f = {"fwd": (d[0], d[1], ace.grouped_matmul), "grad_x": (d[2], d[1], ace.grouped_matmul_grad_x),
               "grad_w": (d[2], d[0], ace.grouped_matmul_grad_w)}[fn]
    want = f(a, b, d[3])
    torch.cuda.synchronize()
    assert torch.equal(f(a, b, d[3]), want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = f(a, b, d[3])
    side.synchronize()
    assert torch.equal(got, want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = f(a, b, d[3])
    for _ in range(3):
        got.fill_(9)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want)
        assert torch.equal(f(a, b, d[3]), want)


def check_all(sizes, tail, M, K, dtype="bf16", seed=0, ways=("fwd", "grad_x", "grad_w")):
    """The ways against the definition in 64 bits, on the GPU (larger cases)."""
    x, w, dy, offs = make(sizes, 0, tail, M, K, dtype, seed)
    d = [t.to(DEV) for t in (x, w, dy, offs)]
    n = int(offs[-1])
    gap = rest(offs, x.shape[0])
    calls = {"fwd": (ace.grouped_matmul, d[0], d[1], K), "grad_x": (ace.grouped_matmul_grad_x, d[2], d[1], M),
             "grad_w": (ace.grouped_matmul_grad_w, d[2], d[0], max(max(sizes), 1))}
    for way in ways:
        fn, a, b, terms = calls[way]
        got = fn(a, b, d[3])
        torch.cuda.synchronize()
        if way == "grad_w":
            want, mag = ref.grouped_grad_w(dy, x, offs)
        else:
            want, mag = ref.grouped(a.cpu(), w if way == "fwd" else w.transpose(1, 2), offs)
            assert not got[gap].any()
        ref.close(got, want, mag, DT[dtype], terms, way)
        assert torch.equal(fn(a, b, d[3]), got)
    return n


def shape_of(sizes, cols):
    """The tile shape that the large kernel takes, by its documented costs."""
    def cost(rows, width, stage):
        items = sum(-(-n // rows) for n in sizes) * -(-cols // width)
        return -(-items // 256) * stage
    costs = {"256": cost(256, 256, 42), "320": cost(320, 192, 41), "192": cost(192, 192, 28), "192w": cost(192, 256, 35)}
    return min(costs, key=costs.get)


LARGE = {"192": (64, 185, 1032), "192w": (40, 180, 1288), "256": (64, 250, 776), "320": (40, 250, 2056)}


@pytest.mark.parametrize("shape", LARGE)
def test_large_shapes(shape):
    """Every tile shape of the large kernel (many rows a group), forward and rows' gradient."""
    N, r, cols = LARGE[shape]
    sizes = [r + (i * 7) % 11 - 5 for i in range(N)]
    assert shape_of(sizes, cols) == shape and sum(sizes) > 80 * N
    check_all(sizes, 0, cols, 72, ways=("fwd",))
    check_all(sizes, 0, 72, cols, ways=("grad_x",))


def test_large_with_a_skewed_plan():
    """Groups of none to thousands of rows, rows of no group behind them."""
    sizes = [3000, 0, 1, 700, 15, 16, 17, 0, 1100, 256, 257, 90] * 2
    assert sum(sizes) > 80 * len(sizes)
    check_all(sizes, 130, 1544, 136, ways=("fwd",))
    check_all(sizes, 130, 136, 1544, ways=("grad_x",))


@pytest.mark.parametrize("sizes,M,K", [([20] * 40, 1544, 104), ([50] * 40, 1544, 136), ([9, 0, 40] * 30, 1160, 200)])
def test_middle_shapes(sizes, M, K):
    """64 x 128 and 128 x 128 tiles: enough of them, few rows a group."""
    check_all(sizes, 3, M, K, ways=("fwd",))
    check_all(sizes, 3, K, M, ways=("grad_x",))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("sizes,M,K", [([3, 2], 64, 4168), ([700, 900], 72, 136), ([2000], 8, 8), ([0, 5000, 1], 40, 200)])
def test_split_reductions(sizes, M, K, dtype):
    """Few tiles with a long reduction: its parts are joined in order, rows of no group stay zero."""
    size = ace.lib().ace_grouped_workspace_size
    from paper_2609_05228_amd import _lib
    code = _lib.ACE_BF16 if dtype == "bf16" else _lib.ACE_F32
    desc = _lib.GroupedDesc(sum(sizes) + 4, len(sizes), M, K, code, 0)
    # two groups of some 800 rows are summed whole: their parts would cost more than they save
    assert (size(desc, 0 if K > 1000 else 2) > 0) == (sizes != [700, 900] or dtype == "f32")
    check_all(sizes, 4, M, K, dtype)
    check_all(sizes, 4, K, M, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("sizes,M,K", [([9000, 5, 0, 2049, 3, 0, 4097, 2048] + [1] * 40, 136, 200),
                                       ([0, 7000] + [3] * 200 + [2500], 264, 72), ([2047, 2049, 0, 1], 520, 520)])
def test_weight_gradient_of_long_groups(sizes, M, K, dtype):
    """Groups of several times the mean are summed in parts, among short and empty ones."""
    check_all(sizes, 77, M, K, dtype, ways=("grad_w",))


@pytest.mark.parametrize("sizes,M,K", [([65, 0, 3, 130, 1] * 14, 264, 520), ([30] * 16, 520, 520)])
def test_weight_gradient_shapes(sizes, M, K):
    """256 x 256 and 128 x 128 tiles of the weights' gradient."""
    check_all(sizes, 1, M, K, ways=("grad_w",))


def test_more_tiles_than_one_list():
    """Work past 64 tiles a workgroup, done in several lists."""
    sizes = [(i * 5) % 4 for i in range(4096)]
    check_all(sizes, 2, 1160, 8, ways=("fwd",))
    gen = torch.Generator(device=DEV).manual_seed(3)
    N, S, M, K = 4096, 8192, 264, 520
    offs = torch.arange(N + 1, device=DEV, dtype=torch.int32) * 2
    dy = torch.randn((S, M), generator=gen, device=DEV).bfloat16()
    x = torch.randn((S, K), generator=gen, device=DEV).bfloat16()
    dw = ace.grouped_matmul_grad_w(dy, x, offs)
    for i in range(0, N, 512):
        a, b = dy[2 * i:2 * i + 1024].double().view(512, 2, M, 1), x[2 * i:2 * i + 1024].double().view(512, 2, 1, K)
        want, mag = (a * b).sum(1), (a * b).abs().sum(1)
        # two products and a sum, then one rounding
        tol = ref.HALF[torch.bfloat16] * want.abs() + 1.01 * 3 * 2 * ref.F32 * mag
        assert bool(((dw[i:i + 512].double() - want).abs() <= tol).all()), i
