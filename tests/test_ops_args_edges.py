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
