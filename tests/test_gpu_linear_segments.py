"""Linear attention in many segments: scans of several wavefronts and rounds, and element-by-element arrays in segments."""
import ctypes as ct

import pytest
import torch

from gpu_common import ensure_built
from linear_common import BF16, F16, F32, check_backward, check_forward, make, plan_of

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, scope="module")
def _built():
    ensure_built()


def _segments(shape, dtype):
    """(forward's, backward's) numbers, by what the workspaces hold: a state and a factor for each segment, backward for two roles."""
    P, B, T, H, K, V = shape
    plan, each = plan_of(shape, dtype), P * B * H * (K * V + 1) * 4
    cfg = plan._config(T)
    return plan.lib.pop_linear_forward_workspace_bytes(ct.byref(cfg)) // each, plan.lib.pop_linear_backward_workspace_bytes(ct.byref(cfg)) // (2 * each)


@pytest.mark.parametrize("T, dtype, least, reset", [(12000, F32, 65, 0.001), (12000, BF16, 65, 0.0), (45000, F32, 257, 0.0002), (45000, BF16, 257, 0.0), (12000, F16, 65, 0.001)])
def test_many_segments(T, dtype, least, reset):
    """More than 64 segments: sixteen wavefronts share them; more than 256: in rounds that hand the state on.  Memories last for most of the
    sequence, so that states of all segments in front count."""
    shape = (1, 1, T, 1, 12, 10)
    assert all(least <= n <= 2 * least + 64 for n in _segments(shape, dtype))
    c, do, dlast = make(shape, dtype, seed=T, decay=(0.2 / T, 0.2 / T), reset=reset, state0=True)
    check_forward(shape, dtype, c)
    check_backward(shape, dtype, c, do, dlast)


def test_a_first_state_through_all_rounds():
    """Nothing but the first state, which does not fade: every output has it, on both sides of each border between segments and rounds."""
    T = 70000
    shape = (1, 1, T, 1, 4, 4)
    assert _segments(shape, F32)[0] > 512
    plan = plan_of(shape, F32, scale=1.0)
    one, zero = torch.ones((1, 1, T, 1, 4), device="cuda"), torch.zeros((1, 1, T, 1, 4), device="cuda")
    S = torch.arange(16.0, device="cuda").view(1, 1, 1, 4, 4)
    o, last = plan.forward(one, zero, zero, state0=S)
    assert torch.equal(last, S) and bool((o == S.sum(3, keepdim=True).view(1, 1, 1, 1, 4)).all())
    dq, dk, dv, first = plan.backward(zero, one, one, zero, dstate_last=S)
    assert torch.equal(first, S) and not dq.any()
    assert bool((dk == S.sum(4).view(1, 1, 1, 1, 4)).all()) and bool((dv == S.sum(3).view(1, 1, 1, 1, 4)).all())


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_one_step_for_all_in_segments(dtype):
    """Keys and values that all steps share go element by element, here in segments."""
    shape = (1, 2, 700, 2, 16, 24)
    assert all(n > 1 for n in _segments(shape, dtype))
    c, do, dlast = make(shape, dtype, seed=4, decay=(0.001, 0.1), reset=0.004, ragged=True, state0=True)
    c["k"], c["v"] = (c[n][:, :, 5:6].expand(c[n].shape) for n in ("k", "v"))
    check_forward(shape, dtype, c)
    check_backward(shape, dtype, c, do, dlast)
    check_backward(shape, dtype, c, do[:, :, 9:10].expand(do.shape), dlast)
