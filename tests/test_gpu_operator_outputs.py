"""Outputs that reach into inputs without meeting them, and those that lie over inputs where that is allowed."""
import ctypes as C

import pytest
import torch

import paper_2206_08888_amd as pp
from gpu_common import ensure_built
from test_gpu_recurrence import BF16, F16, F32, _case

pytestmark = pytest.mark.gpu

def _halves(shape, dtype):
    wide = torch.full(shape[:3] + (2 * shape[3],), float("nan"), dtype=dtype, device="cuda")
    return wide, wide[..., :shape[3]], wide[..., shape[3]:]


@pytest.mark.parametrize("P, B, T, channels, dtype", [(3, 2, 150, 40, F32), (16, 5, 300, 64, F32), (2, 2, 40, 33, BF16)])
def test_outputs_in_halves_of_wider_rows(P, B, T, channels, dtype):
    """y beside x in one array, dx and dg the halves of another: what a projection's backward pass takes as it lies."""
    ensure_built()
    kw, dy, dh = _case(P, B, T, channels, dtype=dtype, seed=7)
    plan = pp.Recurrence(P, B, T, channels, dtype)
    want, last, states = plan.forward(save=True, **kw)
    back = {k: v for k, v in kw.items() if k != "h0"}
    want_back = plan.backward(states, dy=dy, dh_last=dh, **back)

    both, x, y = _halves((P, B, T, channels), dtype)
    x.copy_(kw["x"])
    cfg, io, shape = plan._io(x, kw["g"], kw["bias"], kw["h0"], kw["reset"], kw["lengths"])
    h_last, kept = torch.empty_like(last), torch.empty_like(states)
    io.y, io.h_last, io.states = plan._sequence(y, "y", shape), h_last.data_ptr(), kept.data_ptr()
    ws, n = plan._workspace(cfg)
    plan._call(plan.lib.pop_recurrence_forward, C.byref(cfg), C.byref(io), ws.data_ptr(), n)
    assert torch.equal(y, want) and torch.equal(h_last, last) and torch.equal(x, kw["x"]) and torch.equal(kept, states)

    wide, dx, dg = _halves((P, B, T, channels), dtype)
    dbias, dh0 = torch.empty_like(want_back[2]), torch.empty_like(want_back[3])
    grads = pp.pop_recurrence_grads(plan._sequence(dy, "dy", shape), plan._sequence(dx, "dx", shape), plan._sequence(dg, "dg", shape),
                                    dh.data_ptr(), dh0.data_ptr(), dbias.data_ptr())
    plan._call(plan.lib.pop_recurrence_backward, C.byref(cfg), C.byref(io), C.byref(grads), ws.data_ptr(), n)
    assert all(torch.equal(a, b) for a, b in zip((dx, dg, dbias, dh0), want_back))


@pytest.mark.parametrize("channels, dtype", [(40, F32), (33, F16)])
def test_steps_over_their_inputs(channels, dtype):
    """y over x, and over g."""
    ensure_built()
    kw, _, _ = _case(3, 5, 1, channels, dtype=dtype, seed=8, lengths=False)
    plan = pp.Recurrence(3, 5, 1, channels, dtype)
    slots = torch.randperm(5, device="cuda").to(torch.int32).expand(3, 5).contiguous()
    slots[1, 2] = -1
    for over in ("x", "g"):
        x, g, state = kw["x"][:, :, 0].clone(), kw["g"][:, :, 0].clone(), kw["h0"].clone()
        want, after = None, state.clone()
        want = plan.step(x, g, after, bias=kw["bias"], slots=slots)
        at = x if over == "x" else g
        io = pp.pop_recurrence_io(plan._sequence(x, "x", x.shape), plan._sequence(g, "g", g.shape), plan._sequence(at, "y", at.shape))
        io.bias = kw["bias"].data_ptr()
        plan._call(plan.lib.pop_recurrence_step, plan._one_ref, C.byref(io), state.data_ptr(), 5, slots.data_ptr())
        assert torch.equal(at, want) and torch.equal(state, after)
