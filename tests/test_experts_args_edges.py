"""Arguments of the operators that are no tensors, or not as many as asked for: refused by name before anything is done."""
import torch

import paper_2609_05228_amd as ace
from test_experts_args import _o, _z, refused


def test_pairs_are_pairs():
    x, w, a, o = _z(6, 16), _z(2, 8, 16), _z(6, 8), _o(0, 2, 6)
    refused([
        (lambda: ace.grouped_gated(x, w, w, o, keep=True, out=a), r"out: .*\(a, \(g, u\)\)"),
        (lambda: ace.grouped_gated(x, w, w, o, keep=True, out=(a, a)), r"out: .*\(a, \(g, u\)\)"),
        (lambda: ace.grouped_gated(x, w, w, o, keep=True, out=(a, (a,))), r"out: .*\(a, \(g, u\)\)"),
        (lambda: ace.grouped_gated(x, w, w, o, keep=True, out=(a, None)), r"out: .*\(a, \(g, u\)\)"),
        (lambda: ace.grouped_gated(x, w, w, o, keep=True, out=(a, (None, None))), "out's g must be a tensor"),
        (lambda: ace.grouped_gated(x, w, w, o, keep=True, out=(a, (a, None))), "out's u must be a tensor"),
        (lambda: ace.grouped_gated(x, w, w, o, keep=True, out=(None, (a, a))), "out must be a tensor"),
        (lambda: ace.grouped_gated(x, w, w, o, out=(a, (a, a))), "out must be a tensor"),
        (lambda: ace.grouped_gated_grad(a, x, w, w, o, kept=(a, None)), "kept's u must be a tensor"),
        (lambda: ace.grouped_gated_grad(a, x, w, w, o, kept=(None, a)), "kept's g must be a tensor"),
        (lambda: ace.grouped_gated_grad(a, x, w, w, o, kept=(None, None)), "kept's g must be a tensor"),
        (lambda: ace.grouped_gated_grad(a, None, w, w, o, kept=(None, None), weights=False), "kept's g must be a tensor"),
        (lambda: ace.grouped_gated_grad(a, x, w, w, o, kept=(a, a, a)), r"kept: .*\(g, u\)"),
        (lambda: ace.grouped_gated_grad(a, x, w, w, o, kept=a), r"kept: .*\(g, u\)"),
    ])


def test_what_is_no_tensor():
    x, w, a, o = _z(6, 64), _z(2, 8, 64), _z(6, 8), _o(0, 2, 6)
    q = ace.Mx4(_z(2, 8, 32, dtype=torch.uint8), _z(2, 8, 4, dtype=torch.uint8))
    refused([
        (lambda: ace.grouped_matmul(x, w, None), "offsets must be a tensor"),
        (lambda: ace.grouped_matmul(x, w, [0, 2, 6]), "offsets must be a tensor"),
        (lambda: ace.grouped_matmul(x, w, o, out=[a]), "out must be a tensor"),
        (lambda: ace.grouped_matmul_grad_x(a, w, None), "offsets must be a tensor"),
        (lambda: ace.grouped_matmul_grad_w(a, x, None), "offsets"),
        (lambda: ace.grouped_matmul(x, q, None), "offsets must be a tensor"),
        (lambda: ace.grouped_gated(x, q, q, None), "offsets must be a tensor"),
        (lambda: ace.grouped_gated(x, w, None, o), "w_up must be a tensor"),
        (lambda: ace.grouped_gated(x, w, w, None), "offsets must be a tensor"),
        (lambda: ace.grouped_gated_grad(a, x, w, None, o), "w_up must be a tensor"),
        (lambda: ace.grouped_gated_grad(a, q, w, w, o), "x must be a tensor"),
        (lambda: ace.grouped_gated_grad(a, x, w, w, None), "offsets must be a tensor"),
        (lambda: ace.grouped_gated(x, w, w, o, activation=["silu"]), "activation"),
        (lambda: ace.block_norm(x, a.tolist(), w_pre=_z(64)), "y must be a tensor"),
    ])
    with torch.autograd.forward_ad.dual_level():
        refused([(lambda: ace.grouped_gated(x, w, w, None), "offsets must be a tensor"),
                 (lambda: ace.grouped_gated_grad(a, x, w, w, o, kept=(a, None)), "kept's u must be a tensor")])
