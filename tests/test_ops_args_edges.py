"""Calls that the operators' wrappers refuse although every tensor of them has the right shape, on the CPU."""
import pytest
import torch

import paper_2609_05228_amd as ace


def _z(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype)


def test_a_buffer_for_h_without_y_is_refused():
    """Without y, h' is h and nothing is written for it: a buffer given for it would stay as it was."""
    h, w = _z(6, 16), _z(16)
    with pytest.raises(ValueError, match=r"out\['h'\] needs y"):
        ace.block_norm(h, w_pre=w, out={"h": _z(6, 16)})
    with pytest.raises(ValueError, match="GPU"):  # h itself holds it
        ace.block_norm(h, w_pre=w, out={"h": h, "n": _z(6, 16)})
    with pytest.raises(ValueError, match="GPU"):  # and so does another view of it
        ace.block_norm(h, w_pre=w, out={"h": h.view(6, 16)})


def test_a_refused_gradient_names_no_function_that_is_not_there():
    x, dy = _z(6, 16), _z(6, 8)
    with pytest.raises(ValueError, match="no_grad.*adapter_add has none"):
        ace.adapter_add(dy, x.requires_grad_(), _z(2, 8, 16), _z(2, 8, 8), torch.tensor([0, 2, 6], dtype=torch.int32),
                        torch.tensor([0, -1], dtype=torch.int32))


@pytest.mark.parametrize("which", range(4))
def test_forward_mode_tangents_are_refused(which):
    """A dual tensor's tangent would be lost without a word; the same call outside needs only a GPU."""
    from torch.autograd import forward_ad

    x, w, dy, o = _z(6, 16), _z(2, 8, 16), _z(6, 8), torch.tensor([0, 2, 6], dtype=torch.int32)
    a, b, ids = _z(2, 8, 16), _z(2, 8, 8), torch.tensor([0, -1], dtype=torch.int32)
    call, args = [(lambda p, q: ace.grouped_matmul(p, q, o), (x, w)), (lambda p, q: ace.grouped_matmul_grad_w(p, q, o), (dy, x)),
                  (lambda p, q: ace.block_norm(x, p, gate=q), (x, _z(16))),
                  (lambda p, q: ace.adapter_add(dy, x, p, q, o, ids), (a, b))][which]
    with forward_ad.dual_level():
        for i in range(2):
            duals = [forward_ad.make_dual(t, torch.ones_like(t)) if i == j else t for j, t in enumerate(args)]
            with pytest.raises(ValueError, match="tangent"):
                call(*duals)
            with torch.no_grad(), pytest.raises(ValueError, match="tangent"):
                call(*duals)
        with pytest.raises(ValueError, match="GPU"):
            call(*args)
    with pytest.raises(ValueError, match="GPU"):
        call(*args)
