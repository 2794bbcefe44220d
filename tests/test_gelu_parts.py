"""The parts of the gated block's GELU, on the host against 64 bits."""
from test_gemm_pipe import _build_and_run


def test_gelu_parts(tmp_path):
    _build_and_run(tmp_path, "gelu_check")
