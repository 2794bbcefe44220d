"""4-bit weights where a reduction in parts ends short of a whole panel of scales."""
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
