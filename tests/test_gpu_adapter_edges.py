"""Low-rank adapters where a factor is infinite or leaves bf16's range: the definition's infinity, no NaN."""
import pytest
import torch

import ops_oracle as ref
import paper_2609_05228_amd as ace
from test_gpu_adapter import check, make

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
INF = float("inf")


def run(args, scale):
    got = ace.adapter_add(*[t.to(DEV) for t in args], scale=None if scale is None else scale.to(DEV))
    torch.cuda.synchronize()
    return got


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [5, 4200])  # one launch, two
@pytest.mark.parametrize("rank", [8, 64])
def test_an_infinite_b_reaches_its_columns(rank, rows, dtype):
    """b infinite in two places: those columns are infinite, with the sign of b times the inner product (which
    is far from zero: a's row is positive, x of either sign row by row); the others are as without."""
    *args, scale = make([rows], [0], 0, 0, 1, rank, 136, 72, dtype)
    base, x, a, b, offs, ids = args
    sign = torch.where(torch.arange(rows) % 3 == 1, -1.0, 1.0)
    x.copy_(x.abs() * sign[:, None].to(x.dtype))
    a[0, 3] = a[0, 3].abs() + 0.01
    b[0, 9, 3], b[0, 70, 3] = INF, -INF
    got = run(args, scale).cpu()
    assert torch.equal(got[:, 9].double(), (sign * INF).double())
    assert torch.equal(got[:, 70].double(), (-sign * INF).double())
    keep = [c for c in range(72) if c not in (9, 70)]
    check(got[:, keep], [base[:, keep], x, a, b[:, keep], offs, ids], scale, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [5, 4200])
def test_an_inner_product_between_bf16_s_largest_value_and_fp32_s(rows, dtype):
    """181^2 / 2^14 2^127: finite in fp32, nearer to 2^128 than to bf16's largest value."""
    *args, _ = make([rows], [0], 0, 0, 1, 8, 136, 72, dtype)
    base, x, a, b, offs, ids = args
    x[2], x[:, 40], a[0, 5], a[0, :, 40], b[0, :, 5] = 0, 0, 0, 0, 2.0 ** -126
    x[2, 40], a[0, 5, 40] = 181 * 2.0 ** 56, 181 * 2.0 ** 57
    got = run(args, None)
    check(got, args, None, dtype)
    assert bool(((got[2].float().cpu() - base[2].float()).abs() > 3.9).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [5, 4200])
def test_a_product_past_fp32_is_infinite(rows, dtype):
    """b v far past fp32, v's lower bits rounded up: infinite with its sign, not the difference of two infinities."""
    *args, _ = make([rows], [0], 0, 0, 1, 8, 136, 72, dtype)
    base, x, a, b, offs, ids = args
    x[:, 40] = 0
    a[0, :, 40] = 0
    # v = 32761 2^16 or -25159 2^16 and small terms, whose nearest bf16 values are 7 and 57 2^16 further from zero
    x[1, 40], x[3, 40] = 181 * 2.0 ** 8, -139 * 2.0 ** 8
    a[0, 5, 40] = 181 * 2.0 ** 8
    b[0, 7] = 0
    b[0, 7, 5] = 3 * 2.0 ** 126
    b[0, 8] = -b[0, 7]
    got = run(args, None).cpu()
    assert got[1, 7] == INF and got[1, 8] == -INF and got[3, 7] == -INF and got[3, 8] == INF


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [5, 4200])
def test_an_infinite_scale_and_an_adapter_of_lower_rank(rows, dtype):
    """Ranks past the adapter's own have zeros in a, anything in b: infinity times the product is infinite."""
    *args, scale = make([rows], [0], 0, 0, 1, 16, 136, 72, dtype)
    base, x, a, b, offs, ids = args
    for t in (x, a, b):
        t.copy_(t.abs() + 0.01)
    a[0, 8:] = 0
    b[0, :, 11] *= -1
    for sign in (INF, -INF):
        scale[0] = sign
        assert bool((run(args, scale).cpu() == sign).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [5, 4200])
def test_a_large_scale_of_a_small_product(rows, dtype):
    """The inner product, some 2^50, times the scale alone would pass fp32; with b it does not."""
    *args, scale = make([rows], [0], 0, 0, 1, 8, 136, 72, dtype)
    args[1].mul_(2.0 ** 25)
    args[2].mul_(2.0 ** 25)
    args[3].mul_(2.0 ** -100)
    scale[0] = 2.0 ** 80
    check(run(args, scale), args, scale, dtype)
