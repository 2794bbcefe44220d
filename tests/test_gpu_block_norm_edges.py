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


PLACES = ("dh", "dn", "h", "y")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,d,gate", [(9001, 264, "channel"), (9001, 264, "token"), (9001, 264, "full"), (600, 8200, "channel"),
                                      (5, 40, "token")])
def test_gradients_on_their_inputs(T, d, gate, dtype):
    """The C entry allows the gradients of h and of y each on one of dh, dn, h and y: the same bits as apart from
    them, also where a workgroup copies its next rows before it writes the present ones' results."""
    from paper_2609_05228_amd import _lib

    t, dh, dn = make(T, d, dtype, gate)
    src = dict(dev(t), dh=dh.to(DEV), dn=dn.to(DEV))
    code = _lib.ACE_BF16 if dtype == "bf16" else _lib.ACE_F32
    desc = _lib.NormDesc(T, d, code, {"channel": 1, "token": 2, "full": 3}[gate], 0.75, 0.3, 1e-6)
    lib = ace.lib()
    ws = torch.empty(lib.ace_block_norm_grad_workspace_size(desc), dtype=torch.uint8, device=DEV)

    def run(on_h, on_y):
        g = {k: v.clone() for k, v in src.items()}
        out = {k: torch.full_like(g[k], 3) for k in ("w_post", "w_pre", "gate")}
        out["h"] = g[on_h] if on_h else torch.full_like(g["h"], 3)
        out["y"] = g[on_y] if on_y else torch.full_like(g["y"], 3)
        inp = _lib.NormInputs(*[g[k].data_ptr() for k in ("h", "y", "w_post", "w_pre", "gate")])
        grads = _lib.NormGrads(*[out[k].data_ptr() for k in ("h", "y", "w_post", "w_pre", "gate")])
        st = lib.ace_block_norm_grad(desc, inp, g["dh"].data_ptr(), g["dn"].data_ptr(), grads, ws.data_ptr(), ws.numel(),
                                     torch.cuda.current_stream().cuda_stream)
        assert st == _lib.ACE_OK, (on_h, on_y)
        torch.cuda.synchronize()
        for k in PLACES:  # what no result lies on stays
            assert k in (on_h, on_y) or torch.equal(g[k], src[k]), (on_h, on_y, k)
        return out

    want = run(None, None)
    w = ace.block_norm_grad(src["dh"], src["dn"], src["h"], src["y"], w_post=src["w_post"], w_pre=src["w_pre"],
                            gate=src["gate"], res_scale=0.75, branch_scale=0.3)
    for k in want:
        assert torch.equal(want[k], w[k]), k
    for on_h in (None, *PLACES):
        for on_y in (None, *PLACES):
            if on_h == on_y:
                continue
            got = run(on_h, on_y)
            for k in want:
                assert torch.equal(got[k], want[k]), (on_h, on_y, k)
