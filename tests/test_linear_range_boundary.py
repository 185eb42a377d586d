"""Scales of linear attention at the boundary, CPU-only."""
import ctypes as C

import pytest

import paper_2206_08888_amd as pp
from test_linear_boundary import _config, lib  # noqa: F401


@pytest.mark.parametrize("dtype, scale, code", [
    (pp.POP_F16, 2.0 ** 80, 0), (pp.POP_F16, -(2.0 ** 80), 0), (pp.POP_F16, 2.0 ** 81, pp.POP_EUNSUPPORTED), (pp.POP_F16, -3e38, pp.POP_EUNSUPPORTED),
    (pp.POP_BF16, 3e38, 0), (pp.POP_F32, -3e38, 0), (pp.POP_F32, 0.0, 0)])
def test_scales(lib, dtype, scale, code):  # noqa: F811
    cfg = _config(dtype=dtype, scale=scale)
    for size in (lib.pop_linear_forward_workspace_bytes, lib.pop_linear_backward_workspace_bytes):
        assert min(size(C.byref(cfg)), 0) == code
    if code:
        assert "2^80" in pp.pop_last_error(None)
