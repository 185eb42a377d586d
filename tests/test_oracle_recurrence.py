"""The oracle of the gated linear recurrence: its gradients against differences, its masks, single steps against
sequences, its rounding bounds against 32-bit arithmetic."""
import numpy as np
import pytest

from oracle import recurrence as R


def _inputs(seed, P=2, B=3, T=9, C=4):
    rng = np.random.default_rng(seed)
    return dict(x=rng.standard_normal((P, B, T, C)), g=rng.standard_normal((P, B, T, C)), bias=rng.uniform(0, 3, (P, C)),
                h0=rng.standard_normal((P, B, C)), reset=rng.random((P, B, T)) < 0.2,
                lengths=rng.integers(0, T + 1, (P, B))), rng.standard_normal((P, B, T, C)), rng.standard_normal((P, B, C))


@pytest.mark.parametrize("seed", range(4))
def test_gradients_match_differences(seed):
    kw, dy, dh = _inputs(seed)

    def loss(**change):
        y, h, _, _ = R.forward(**dict(kw, **change))
        return (y * dy).sum() + (h * dh).sum()

    grads, _ = R.backward(dy=dy, dh_last=dh, **kw)
    rng, eps = np.random.default_rng(seed + 100), 1e-6
    for name, got in (("x", grads["dx"]), ("g", grads["dg"]), ("bias", grads["dbias"]), ("h0", grads["dh0"])):
        v = rng.standard_normal(kw[name].shape)
        slope = (loss(**{name: kw[name] + eps * v}) - loss(**{name: kw[name] - eps * v})) / (2 * eps)
        # central differences: curvature eps^2 and the loss's own rounding 1e-16 * |loss| / eps, together below 1e-8
        assert abs(slope - (got * v).sum()) < 1e-8 * max(1.0, abs(slope)), name


def test_masks():
    kw, dy, dh = _inputs(7)
    kw["lengths"][:] = [[0, 1, 9], [9, 5, 0]]
    kw["reset"][0, 1, 0] = True
    y, h, _, _ = R.forward(**kw)
    assert np.array_equal(h[0, 0], kw["h0"][0, 0]) and np.array_equal(h[1, 2], kw["h0"][1, 2])
    assert not y[0, 0].any() and not y[0, 1, 1:].any()
    a, b = R.sigmoids(kw["g"] + kw["bias"][:, None, None])
    assert np.allclose(y[0, 1, 0], b[0, 1, 0] * kw["x"][0, 1, 0])               # the reset drops h0
    g, _ = R.backward(dy=dy, dh_last=dh, **kw)
    assert np.array_equal(g["dh0"][0, 0], dh[0, 0]) and not g["dh0"][0, 1].any()
    assert not g["dx"][1, 1, 5:].any()


def test_steps_are_a_sequence():
    kw, _, _ = _inputs(3)
    kw.pop("lengths")
    want, _, _, _ = R.forward(**kw)
    state = kw["h0"]
    for t in range(9):
        y, state, _, _ = R.step(kw["x"][:, :, t], kw["g"][:, :, t], state, kw["bias"], kw["reset"][:, :, t])
        assert np.allclose(y, want[:, :, t], rtol=1e-14)


def test_bounds_hold_for_32_bit_arithmetic():
    kw, _, _ = _inputs(11, T=400)
    kw = {k: v.astype(np.float32) if v.dtype == np.float64 else v for k, v in kw.items()}
    kw["bias"] += np.float32(3)
    y, h, E, _ = R.forward(rounding=2.0 ** -24, **kw)
    got, state = np.zeros_like(kw["x"]), kw["h0"].copy()
    for t in range(400):
        z = kw["g"][:, :, t] + kw["bias"][:, None]
        a = 1 / (1 + np.exp(-z))
        v = np.where(kw["reset"][:, :, t, None], 0, a * state) + (1 / (1 + np.exp(z))) * kw["x"][:, :, t]
        live = (t < kw["lengths"])[..., None]
        got[:, :, t], state = np.where(live, v, 0), np.where(live, v, state)
    assert got.dtype == np.float32 and (np.abs(got - y) <= E["y"]).all()
    assert np.median(np.abs(got - y)[E["y"] > 0] / E["y"][E["y"] > 0]) > 1e-3    # and they are not empty


def test_bounds_hold_for_chunks_in_32_bits():
    """Chunk maps found first and applied to the state afterwards, where terms cancel that step by step never grow."""
    f = np.float32
    rng = np.random.default_rng(5)
    x = rng.standard_normal((1, 1, 512, 3000)).astype(f)
    g, h0 = (rng.standard_normal(x.shape) + 4).astype(f), rng.standard_normal((1, 1, 3000)).astype(f) * f(20)
    y, h, E, _ = R.forward(x, g, h0=h0, rounding=2 * 2.0 ** -24)
    a, b = 1 / (1 + np.exp(-g)), 1 / (1 + np.exp(g))
    state = h0
    for lo in range(0, 512, 128):
        A, H = np.ones_like(h0), np.zeros_like(h0)
        for t in range(lo, lo + 128):
            A, H = A * a[:, :, t], a[:, :, t] * H + b[:, :, t] * x[:, :, t]
        state = A * state + H
    assert state.dtype == f and (np.abs(state - h) <= E["h_last"]).all()
