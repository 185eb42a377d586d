"""The oracle of linear attention: against the double sum over pairs of steps, and its gradients against differences."""
import numpy as np
import pytest

from oracle import linear as L


def _case(T=9, reset=True, ragged=True, seed=0):
    rng = np.random.default_rng(seed)
    P, B, H, K, V = 2, 3, 2, 4, 3
    draw = lambda *s: rng.standard_normal(s)
    c = dict(q=draw(P, B, T, H, K), k=draw(P, B, T, H, K), v=draw(P, B, T, H, V), log_decay=-rng.random((P, H)), state0=draw(P, B, H, K, V))
    c["reset"] = rng.random((P, B, T)) < 0.2 if reset else None
    c["lengths"] = rng.integers(0, T + 1, (P, B)) if ragged else None
    return c, draw(P, B, T, H, V), draw(P, B, H, K, V)


def _pairs(q, k, v, log_decay, state0, reset, lengths):
    P, B, T, H, K = q.shape
    o, last = np.zeros(v.shape), np.zeros(state0.shape)
    for p, b, h in np.ndindex(P, B, H):
        n = T if lengths is None else lengths[p, b]
        starts = np.zeros(T, int) if reset is None else np.cumsum(reset[p, b])
        lam = np.exp(log_decay[p, h])
        for t in range(n + 1):
            S = lam ** min(t + 1, n) * state0[p, b, h] * (starts[min(t, n - 1)] == 0 if n else 1)
            for s in range(min(t + 1, n)):
                if starts[s] == starts[min(t, n - 1)]:
                    S = S + lam ** (min(t, n - 1) - s) * np.outer(k[p, b, s, h], v[p, b, s, h])
            if t == n:
                last[p, b, h] = S
            else:
                o[p, b, t, h] = K ** -0.5 * S.T @ q[p, b, t, h]
    return o, last


@pytest.mark.parametrize("reset", [False, True])
@pytest.mark.parametrize("ragged", [False, True])
def test_forward_is_the_sum_over_pairs(reset, ragged):
    c, _, _ = _case(reset=reset, ragged=ragged)
    o, last, E = L.forward(**c)
    want = _pairs(**c)
    assert np.abs(o - want[0]).max() < 1e-12 and np.abs(last - want[1]).max() < 1e-12
    assert not E["o"].any() and not E["state_last"].any()


@pytest.mark.parametrize("reset", [False, True])
@pytest.mark.parametrize("ragged", [False, True])
def test_gradients_against_differences(reset, ragged):
    c, do, dlast = _case(reset=reset, ragged=ragged, seed=1)
    grads, _ = L.backward(do=do, dstate_last=dlast, **c)

    def loss(**kw):
        o, last, _ = L.forward(**dict(c, **kw))
        return (o * do).sum() + (last * dlast).sum()

    rng = np.random.default_rng(2)
    for name, of in (("dq", "q"), ("dk", "k"), ("dv", "v"), ("dstate0", "state0")):
        for _ in range(4):
            d = rng.standard_normal(c[of].shape)
            h = 1e-4                                     # the loss is quadratic along a direction: no error of differences
            got = (loss(**{of: c[of] + h * d}) - loss(**{of: c[of] - h * d})) / (2 * h)
            assert abs(got - (grads[name] * d).sum()) < 1e-7 * (1 + np.abs(grads[name] * d).sum()), name


def test_bounds_hold_for_32_bits():
    """Step by step in fp32, the most roundings of any order."""
    c, do, dlast = _case(T=60, seed=3)
    f = lambda x: x.astype(np.float32)
    c = {k: f(x) if x.dtype.kind == "f" else x for k, x in c.items()}
    o, last, E = L.forward(unit=2.0 ** -24, **c)
    lam = np.exp(c["log_decay"])[:, None, :, None, None].astype(np.float32)
    S = c["state0"].copy()
    for t in range(60):
        live = (t < c["lengths"])[:, :, None, None, None]
        new = np.where(c["reset"][:, :, t][:, :, None, None, None], np.float32(0), lam * S) + c["k"][:, :, t][..., :, None] * c["v"][:, :, t][..., None, :]
        S = np.where(live, new, S)
        y = (c["q"][:, :, t][..., :, None] * new).sum(-2) * np.float32(0.5)
        assert (np.abs(np.where(live[..., 0], y, 0) - o[:, :, t]) <= E["o"][:, :, t]).all()
    assert (np.abs(S - last) <= E["state_last"]).all()
    assert E["o"].max() < 1e-4 * np.abs(o).max()


def test_a_step_is_a_sequence_of_one():
    c, _, _ = _case(T=1, ragged=False)
    o, last, _ = L.forward(**c)
    y, state, _, _ = L.step(c["q"][:, :, 0], c["k"][:, :, 0], c["v"][:, :, 0], c["state0"], c["log_decay"], c["reset"][:, :, 0])
    assert np.array_equal(o[:, :, 0], y) and np.array_equal(last, state)
    slots = np.array([[2, -1, 0], [1, 3, 7]])
    y, state, _, _ = L.step(c["q"][:, :, 0], c["k"][:, :, 0], c["v"][:, :, 0], c["state0"], c["log_decay"], None, slots)
    assert not y[0, 1].any() and not y[1, 1].any() and not y[1, 2].any()
    assert np.array_equal(state[0, 1], c["state0"][0, 1]) and not np.array_equal(state[0, 2], c["state0"][0, 2])
