"""Gates whose parts are large and cancel, against the oracle's bounds."""
import pytest
import torch

import paper_2206_08888_amd as pp
from gpu_common import ensure_built
from oracle import recurrence as R
from test_gpu_recurrence import F16, F32, ROUNDING, _case, _check, _np, _verify

pytestmark = pytest.mark.gpu


def _cancelling(kw, size):
    """bias of about +-size, g the same the other way round: their sum is what g was."""
    P, B, T, C = kw["x"].shape
    sign = torch.ones((P, C), device="cuda")
    sign[:, ::2] = -1
    kw["bias"] = sign * size * (1 + torch.rand((P, C), device="cuda"))
    kw["g"] = (kw["g"].float() - kw["bias"][:, None, None]).to(kw["g"].dtype)


# whole sequences, segments, chains; vectors and single elements
@pytest.mark.parametrize("size", [5.0, 100.0, 3e4])
@pytest.mark.parametrize("P, B, T, C, dtype", [(2, 3, 100, 40, F32), (1, 2, 700, 33, F32), (10, 7, 300, 65, F32), (2, 3, 300, 64, F16)])
def test_parts_that_cancel(P, B, T, C, dtype, size):
    ensure_built()
    kw, dy, dh = _case(P, B, T, C, dtype=dtype, seed=17)
    _cancelling(kw, size)
    _verify(kw, dy, dh)


@pytest.mark.parametrize("size", [100.0, 3e4])
@pytest.mark.parametrize("C", [33, 40])
def test_parts_that_cancel_in_single_steps(C, size):
    ensure_built()
    kw, _, _ = _case(3, 5, 1, C, seed=18, lengths=False)
    _cancelling(kw, size)
    x, g, reset, state = kw["x"][:, :, 0], kw["g"][:, :, 0], kw["reset"][:, :, 0].contiguous(), kw["h0"].clone()
    y = pp.Recurrence(3, 5, 1, C).step(x, g, state, bias=kw["bias"], reset=reset)
    wy, ws, Ey, Es = R.step(_np(x), _np(g), _np(kw["h0"]), _np(kw["bias"]), _np(reset), None, rounding=ROUNDING)
    _check("y", y, wy, Ey)
    _check("state", state, ws, Es)
