"""4-bit weights where a reduction in parts ends short of a whole panel of scales, and scales at both ends of the byte."""
import pytest
import torch

import experts_oracle as ref
import mx4_oracle as fmt
import paper_2609_05228_amd as ace
from test_gpu_mx4 import BF16, DEV, dev, make, rows_of

pytestmark = pytest.mark.gpu


# groups of few rows, whose reduction the four waves of a workgroup share, and a launch in parts (K = 1824)
@pytest.mark.parametrize("rows", ["bf16", "mx4"])
@pytest.mark.parametrize("sizes,M,K", [([2, 0, 1, 5], 72, K) for K in (32, 160, 384, 512, 640, 768, 1024, 1056, 1536)] +
                         [([300], 520, 1824), ([150, 3], 520, 1824)], ids=str)
def test_parts_of_panels(sizes, M, K, rows):
    x, xv, ws, offs = make(sizes, 0, 0, M, K, rows)
    xd, o, w = rows_of(x), offs.to(DEV), [dev(q) for q in ws]
    wv = [fmt.values(*q) for q in ws]
    y = ace.grouped_matmul(xd, w[0], o)
    want, err = ref.both(xv, wv[0], offs)
    ref.within(y, want, err, BF16, "y")
    a = ace.grouped_gated(xd, *w, o)
    want, err = ref.gated(xv, *wv, offs, "silu")
    ref.within(a, want["a"], err["a"], BF16, "a")


# few rows, 64-row tiles, the large ones
SIZES = [([20, 3], 40, 96), ([40, 0, 90], 136, 224), ([150] * 12, 2056, 160)]


def scaled(x, xv, rows, e):
    """The rows times 2^e."""
    if rows == "bf16":
        return (x.double() * 2.0 ** e).to(BF16), xv * 2.0 ** e
    s = x[1].int() + e
    assert 0 < int(s[:, :xv.shape[1] // 32].min()) and int(s[:, :xv.shape[1] // 32].max()) < 255
    return (x[0], s.to(torch.uint8)), xv * 2.0 ** e


def with_scales(q, K, lo, hi):
    codes, scales = q[0], q[1].clone()
    blocks = scales[..., :K // 32]
    blocks[blocks != 255] = torch.randint(lo, hi, blocks.shape, generator=torch.Generator().manual_seed(lo)).to(torch.uint8)[
        blocks != 255]
    return codes, scales


@pytest.mark.parametrize("rows", ["bf16", "mx4"])
@pytest.mark.parametrize("sizes,M,K", SIZES, ids=str)
def test_least_scales(sizes, M, K, rows):
    """Weights from 2^-128 on, below the least normal number of bf16, count exactly: rows large enough that the products
    are normal numbers."""
    x, xv, ws, offs = make(sizes, 0, 0, M, K, rows)
    x, xv = scaled(x, xv, rows, 100)
    q = with_scales(ws[0], K, 0, 4)
    wv = fmt.values(*q)
    assert bool((wv.nan_to_num().abs() < 2.0 ** -126).any())
    y = ace.grouped_matmul(rows_of(x), dev(q), offs.to(DEV))
    want, err = ref.both(xv, wv, offs)
    ref.within(y, want, err, BF16, "y")


@pytest.mark.parametrize("rows", ["bf16", "mx4"])
@pytest.mark.parametrize("sizes,M,K", SIZES, ids=str)
def test_largest_scales(sizes, M, K, rows):
    """Scales up to 2^127.  Rows in 4 bits: exact.  bf16 rows: weights past bf16's largest number, 2^128 and up, are
    infinite, as mx4_dequantize gives them, so their columns are infinite or NaN; the others are exact."""
    x, xv, ws, offs = make(sizes, 0, 0, M, K, rows)
    x, xv = scaled(x, xv, rows, -100)
    codes, scales = with_scales(ws[0], K, 250, 255)
    scales[:, 1::2, :K // 32] = scales[:, 1::2, :K // 32].clamp_max(252)  # every other column holds none
    for e, n in enumerate(sizes):
        if n == 0:
            scales[e] = 255
    wv = fmt.values(codes, scales)
    past = wv.abs() >= 2.0 ** 128
    if rows == "mx4":
        past = torch.zeros_like(past)
    assert rows == "mx4" or (bool(past[:, ::2].any()) and not past[:, 1::2].any())
    y = ace.grouped_matmul(rows_of(x), dev((codes, scales)), offs.to(DEV)).cpu()
    want, err = ref.both(xv, torch.where(past, torch.zeros((), dtype=torch.float64), wv), offs)
    inf = torch.zeros(y.shape, dtype=torch.bool)
    for e in range(len(sizes)):
        inf[int(offs[e]):int(offs[e + 1])] = past[e].any(dim=1)
    assert torch.equal(~y.isfinite(), inf)
    ref.within(y[~inf], want[~inf], err[~inf], BF16, "y")
