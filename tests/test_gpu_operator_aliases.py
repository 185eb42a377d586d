"""Last states written over first ones (h_last over h0, dh0 over dh_last), as the boundary allows: in every way that sequences
are shared, also while other work holds parts of the chip, so that workgroups of one launch start far apart."""
import ctypes as C

import pytest
import torch

import paper_2206_08888_amd as pp
from gpu_common import ensure_built
from test_gpu_recurrence import BF16, F16, F32, _case

pytestmark = pytest.mark.gpu

# whole sequences, segments (128, 128 and 103 of them), chains
SHAPES = [(2, 3, 50, 40, F32), (1, 1, 30000, 64, F32), (1, 2, 20000, 200, BF16), (2, 5, 13100, 64, F16), (10, 7, 300, 65, F32), (40, 13, 300, 64, BF16)]


def _forward(plan, kw, y, h_last, states):
    cfg, io, shape = plan._io(kw["x"], kw["g"], kw["bias"], kw["h0"], kw["reset"], kw["lengths"])
    io.y, io.h_last, io.states = plan._sequence(y, "y", shape), h_last.data_ptr(), states.data_ptr()
    ws, n = plan._workspace(cfg)
    plan._call(plan.lib.pop_recurrence_forward, C.byref(cfg), C.byref(io), ws.data_ptr(), n)


def _backward(plan, kw, states, dy, dh_last, dh0):
    cfg, io, shape = plan._io(kw["x"], kw["g"], kw["bias"], None, kw["reset"], kw["lengths"])
    io.states = states.data_ptr()
    dx, dg, dbias = torch.empty_like(dy), torch.empty_like(dy), torch.empty_like(kw["bias"])
    grads = pp.pop_recurrence_grads(plan._sequence(dy, "dy", shape), plan._sequence(dx, "dx", shape), plan._sequence(dg, "dg", shape),
                                    dh_last.data_ptr(), dh0.data_ptr(), dbias.data_ptr())
    ws, n = plan._workspace(cfg)
    plan._call(plan.lib.pop_recurrence_backward, C.byref(cfg), C.byref(io), C.byref(grads), ws.data_ptr(), n)
    return dx, dg, dbias


@pytest.mark.parametrize("busy", [False, True])
@pytest.mark.parametrize("P, B, T, channels, dtype", SHAPES)
def test_last_over_first(P, B, T, channels, dtype, busy):
    ensure_built()
    kw, dy, dh = _case(P, B, T, channels, dtype=dtype, seed=T, reset=False, lengths=False)
    kw["bias"] = kw["bias"] + 8                          # first states last for thousands of steps
    plan = pp.Recurrence(P, B, T, channels, dtype)
    y, last, states = plan.forward(save=True, **kw)
    want = plan.backward(states, dy=dy, dh_last=dh, **{k: v for k, v in kw.items() if k != "h0"})
    again, kept = torch.empty_like(y), torch.empty_like(states)
    left, other = torch.randn((4096, 4096), device="cuda"), torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    if busy:
        with torch.cuda.stream(other):
            for _ in range(4):
                left @ left
    _forward(plan, kw, again, kw["h0"], kept)
    got = _backward(plan, kw, kept, dy, dh, dh)
    torch.cuda.current_stream().wait_stream(other)
    assert torch.equal(again, y) and torch.equal(kw["h0"], last) and torch.equal(kept, states)
    assert all(torch.equal(a, b) for a, b in zip(got, want[:3])) and torch.equal(dh, want[3])
