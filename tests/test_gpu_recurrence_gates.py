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


def _steps32(kw, dy, dh):
    """Forward and backward step by step in 32 bits on the CPU."""
    x, g, bias, h = (kw[k].cpu() for k in ("x", "g", "bias", "h0"))
    z = g + bias[:, None, None]
    a, b = torch.sigmoid(z), torch.sigmoid(-z)
    T, before, y = x.shape[2], [], []
    for t in range(T):
        before.append(h)
        h = a[:, :, t] * h + b[:, :, t] * x[:, :, t]
        y.append(h)
    d, dx, dg = dh.cpu(), [None] * T, [None] * T
    for t in reversed(range(T)):
        d = d + dy[:, :, t].cpu()
        dx[t] = d * b[:, :, t]
        dg[t] = dx[t] * (before[t] - x[:, :, t]) * a[:, :, t]
        d = d * a[:, :, t]
    dg = torch.stack(dg, 2)
    return dict(y=torch.stack(y, 2), h_last=h, dx=torch.stack(dx, 2), dg=dg, dbias=dg.sum((1, 2)), dh0=d)


@pytest.mark.parametrize("P, B, T, C", [(3, 2, 500, 64), (2, 3, 300, 33), (16, 5, 300, 64)])
def test_errors_are_those_of_steps_in_32_bits(P, B, T, C):
    """Memories of a few to a few hundred steps: states and gradients pass through hundreds of gates near one, the rounding of
    each of which counts.  As many roundings as the steps have: no further off than they are, but for a fifth."""
    ensure_built()
    kw, dy, dh = _case(P, B, T, C, seed=23, reset=False, lengths=False)
    kw["bias"] = kw["bias"] * 1.25 + 0.5
    kw["g"] = kw["g"] / 1.5
    plan = pp.Recurrence(P, B, T, C)
    y, h_last, states = plan.forward(save=True, **kw)
    got = dict(zip(("dx", "dg", "dbias", "dh0"), plan.backward(states, dy=dy, dh_last=dh, **{k: v for k, v in kw.items() if k != "h0"})), y=y, h_last=h_last)
    host = {k: _np(v) for k, v in kw.items()}
    wy, wh, _, _ = R.forward(**host)
    want, _ = R.backward(dy=_np(dy), dh_last=_np(dh), **host)
    want.update(y=wy, h_last=wh)
    for name, v in _steps32(kw, dy, dh).items():
        err, err32 = ((_np(t) - want[name]).ravel() for t in (got[name], v))
        assert (err @ err) ** 0.5 <= 1.2 * (err32 @ err32) ** 0.5, (name, (err @ err) ** 0.5, (err32 @ err32) ** 0.5)
