"""Gradients of the norms where an operand is infinite: it reaches the results that the definition has it in,
and no others."""
import pytest
import torch

import ops_oracle as ref
import paper_2609_05228_amd as ace
from test_gpu_block_norm import DT, TERMS, dev, make

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
INF, NAN = float("inf"), float("nan")


def same(got, want, mag, dtype, name):
    """What is no finite number in the definition is the same one here, the rest within its rounding."""
    got = got.cpu()
    num = want.isfinite()
    assert torch.equal(got.isnan(), want.isnan()), name
    assert torch.equal(got.double()[~num & ~want.isnan()], want[~num & ~want.isnan()]), name
    ref.close(got[num], want[num], mag[num], DT[dtype], TERMS, name)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [1, 3, 9001])
@pytest.mark.parametrize("d", [40, 264])
@pytest.mark.parametrize("where", ["gate", "w_post"])
def test_an_infinite_parameter_and_rows_that_are_not_there(where, d, T, dtype):
    """A workgroup takes several rows at a time; where it has fewer, the missing ones add nothing.  All terms
    are positive, so the sums over an infinite column are infinite.  (Sums over 9001 rows: TERMS holds, they
    are split over more threads than its comment counts on.)"""
    t, dh, _ = make(T, d, dtype, "channel", True, False)
    t = {k: None if v is None else v.abs() + 0.01 for k, v in t.items()}
    dh = dh.abs() + 0.01
    t[where][3] = INF
    got = ace.block_norm_grad(dh.to(DEV), None, **dev(t))
    torch.cuda.synchronize()
    want, mag = ref.block_norm_grad(dh, None, **t)
    other = {"gate": "w_post", "w_post": "gate"}[where]
    assert want[other][3] == INF and bool(want[where].isfinite().all())
    for k in ("h", "gate", "w_post"):
        same(got[k], want[k], mag[k], dtype, k)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("gate", ["channel", "token", "full"])
@pytest.mark.parametrize("d", [40, 8200])
def test_y_does_not_reach_its_own_gradient_without_a_norm(d, gate, dtype):
    """u = gate y: the gradient of y is the gate's times dh', whatever y holds."""
    t, dh, _ = make(5, d, dtype, gate, False, False)
    t["y"][1, 7], t["y"][2, 30], t["y"][4, 0] = INF, NAN, -INF
    got = ace.block_norm_grad(dh.to(DEV), None, **dev(t))
    torch.cuda.synchronize()
    want, mag = ref.block_norm_grad(dh, None, **t)
    assert bool(want["y"].isfinite().all()) and not bool(want["gate"].isfinite().all())
    for k in ("h", "y"):
        ref.close(got[k], want[k], mag[k], DT[dtype], TERMS, k)
    same(got["gate"], want["gate"], mag["gate"], dtype, "gate")
