"""How the tiles of 4-bit operands are staged, replayed on the host: nothing is read outside the tensors, also where a
reduction is in parts."""
from test_gemm_pipe import _build_and_run


def test_mx4_staging(tmp_path):
    _build_and_run(tmp_path, "mx4_panel_check")
