"""Gated linear recurrence in 64 bits, step by step, with its backward pass and bounds on what rounding may do.

  a_t = sigmoid(g_t + bias), h_t = a_t keep_t h_{t-1} + (1 - a_t) x_t, y_t = h_t for t < length;  keep_t = 0 at resets

Arrays are [P, batch, T, C] (numpy).  `rounding` is the unit roundoff of the arithmetic whose result is to be judged:
with it, the functions return for every output a bound on its distance from the exact value, propagated along the
recurrence beside the values themselves (first order).  A scan may add the terms in any grouping, so what is rounded is
as large as the sum of the terms' magnitudes, not as their sum: the magnitudes are propagated as well.
"""
import numpy as np


def sigmoids(z):
    """sigmoid(z), sigmoid(-z) without overflow."""
    with np.errstate(invalid="ignore"):
        e = np.exp(-np.abs(z))
        big, small = 1 / (1 + e), e / (1 + e)
        return np.where(z >= 0, big, np.where(z < 0, small, z)), np.where(z >= 0, small, np.where(z < 0, big, z))


def _setup(x, g, bias, reset, lengths):
    P, B, T, C = x.shape
    z = g.astype(np.float64) + (0 if bias is None else bias.astype(np.float64)[:, None, None, :])
    reset = np.zeros((P, B, T), bool) if reset is None else reset.astype(bool)
    lengths = np.full((P, B), T) if lengths is None else np.clip(lengths, 0, T)
    return z, reset[..., None], lengths[..., None]


def gate_rounding(z):
    """Relative error of a computed gate in units of the roundoff: the argument's own rounding passes through exp
    (z twice: sum, factor log2 e), then exp, 1 + e, the reciprocal and a product, at most two units each."""
    return 3 * np.minimum(np.abs(z), 100) + 8


def forward(x, g, bias=None, h0=None, reset=None, lengths=None, rounding=0.0):
    """y, h_last, {"y": bound, "h_last": bound} and the state in front of every step (0 behind a reset) with its bound."""
    P, B, T, C = x.shape
    z, reset, lengths = _setup(x, g, bias, reset, lengths)
    a, b = sigmoids(z)
    x = x.astype(np.float64)
    h = np.zeros((P, B, C)) if h0 is None else h0.astype(np.float64)
    E, M = np.zeros_like(h), np.abs(h)
    y, before, Ey, Eb = (np.zeros((P, B, T, C)) for _ in range(4))
    with np.errstate(invalid="ignore", over="ignore"):
        for t in range(T):
            k = gate_rounding(z[:, :, t]) * rounding
            hp, Ep, Mp = (np.where(reset[:, :, t], 0, v) for v in (h, E, M))
            before[:, :, t], Eb[:, :, t] = hp, Ep
            carried, new = np.where(reset[:, :, t], 0, a[:, :, t] * hp), b[:, :, t] * x[:, :, t]
            v = carried + new
            Mv = a[:, :, t] * Mp + np.abs(new)
            Ev = a[:, :, t] * Ep + (k + 2 * rounding) * Mv
            live = t < lengths
            y[:, :, t], Ey[:, :, t] = np.where(live, v, 0), np.where(live, Ev, 0)
            h, E, M = np.where(live, v, h), np.where(live, Ev, E), np.where(live, Mv, M)
    return y, h, {"y": Ey, "h_last": E}, (before, Eb)


def backward(x, g, dy, bias=None, h0=None, reset=None, lengths=None, dh_last=None, rounding=0.0):
    """{"dx", "dg", "dbias", "dh0"} and their bounds."""
    P, B, T, C = x.shape
    _, _, _, (before, Eb) = forward(x, g, bias, h0, reset, lengths, rounding)
    z, reset, lengths = _setup(x, g, bias, reset, lengths)
    a, b = sigmoids(z)
    x, dy = x.astype(np.float64), dy.astype(np.float64)
    d = np.zeros((P, B, C)) if dh_last is None else dh_last.astype(np.float64)
    E, M = np.zeros_like(d), np.abs(d)
    dx, dg, Ex, Eg = (np.zeros((P, B, T, C)) for _ in range(4))
    with np.errstate(invalid="ignore", over="ignore"):
        for t in reversed(range(T)):
            live, k = t < lengths, gate_rounding(z[:, :, t]) * rounding
            at, ab = d + dy[:, :, t], a[:, :, t] * b[:, :, t]
            Mat = M + np.abs(dy[:, :, t])
            Eat = E + rounding * Mat
            diff = before[:, :, t] - x[:, :, t]
            dx[:, :, t] = np.where(live, at * b[:, :, t], 0)
            dg[:, :, t] = np.where(live, at * diff * ab, 0)
            Ex[:, :, t] = np.where(live, Eat * b[:, :, t] + (k + rounding) * Mat * b[:, :, t], 0)
            Eg[:, :, t] = np.where(live, ab * (Eat * np.abs(diff) + np.abs(at) * (Eb[:, :, t] + rounding * np.abs(diff))
                                         + (2 * k + 4 * rounding) * Mat * np.abs(diff)), 0)
            back = np.where(reset[:, :, t], 0, at * a[:, :, t])
            Mback = np.where(reset[:, :, t], 0, Mat * a[:, :, t])
            Eback = np.where(reset[:, :, t], 0, Eat * a[:, :, t]) + (k + 2 * rounding) * Mback
            d, E, M = np.where(live, back, d), np.where(live, Eback, E), np.where(live, Mback, M)
    n = B * T
    return ({"dx": dx, "dg": dg, "dbias": dg.sum((1, 2)), "dh0": d},
            {"dx": Ex, "dg": Eg, "dbias": Eg.sum((1, 2)) + rounding * min(n, 4096) * np.abs(dg).sum((1, 2)), "dh0": E})


def step(x, g, state, bias=None, reset=None, slots=None, rounding=0.0):
    """y, new state and their bounds; x, g [P, batch, C], state [P, n_slots, C]."""
    P, B, C = x.shape
    y, Ey, state = np.zeros((P, B, C)), np.zeros((P, B, C)), state.astype(np.float64).copy()
    Es = np.zeros_like(state)
    for p in range(P):
        for r in range(B):
            s = r if slots is None else int(slots[p, r])
            if not 0 <= s < state.shape[1]:
                continue
            one = lambda v: v[p:p + 1, r:r + 1, None]
            v, _, E, _ = forward(one(x), one(g), None if bias is None else bias[p:p + 1], state[p, s][None, None],
                                 None if reset is None else reset[p, r].reshape(1, 1, 1), None, rounding)
            y[p, r], Ey[p, r] = v[0, 0, 0], E["y"][0, 0, 0]
            state[p, s], Es[p, s] = y[p, r], Ey[p, r]
    return y, state, Ey, Es
