"""Linear attention with a decay for each head in 64 bits, step by step, with its backward pass and bounds on what rounding may do.

  S_t = lambda keep_t S_{t-1} + k_t v_t^T, o_t = scale S_t^T q_t for t < length;  lambda = exp(log_decay), keep_t = 0 at resets
  D_t = scale q_t do_t^T + lambda keep_{t+1} D_{t+1}: dq_t = scale S_t do_t, dk_t = D_t v_t, dv_t = D_t^T k_t, dstate0 = lambda keep_0 D_0

Arrays are [P, batch, T, heads, width] (numpy).  Bounds: sums may be grouped in any way, so that what is rounded is as large as
the sum of the terms' magnitudes, which are carried along as states of their own (|k| |v|^T in the place of k v^T).  `unit` is the
roundoff of sums and factors, `operand` how far an operand of a product may be from its value, relative to its magnitude.
"""
import numpy as np


def decays(log_decay, P, H):
    z = np.zeros((P, H)) if log_decay is None else np.clip(log_decay.astype(np.float64), -200, 0)
    return z[:, None, :, None, None]


def _setup(q, v, log_decay, reset, lengths):
    P, B, T, H, _ = q.shape
    z = decays(log_decay, P, H)
    reset = np.zeros((P, B, T), bool) if reset is None else reset.astype(bool)
    lengths = np.full((P, B), T) if lengths is None else np.clip(lengths, 0, T)
    five = lambda m: m[:, :, None, None, None]
    return z, np.exp(z), [five(reset[:, :, t]) for t in range(T)], [five(t < lengths) for t in range(T)]


def _outer(a, b):
    return a[..., :, None] * b[..., None, :]


def _over_keys(x, S):
    return (x[..., :, None] * S).sum(-2)


def _over_values(S, x):
    return (S * x[..., None, :]).sum(-1)


def _start(state, P, B, H, K, V):
    return np.zeros((P, B, H, K, V)) if state is None else state.astype(np.float64)


class _Scan:
    """A state S with its magnitude M and the bound E on its error.  A factor lambda counts as far as exp's argument may be off (its
    rounding, the product with a count of steps, exp itself: 4 (1 - z) units), the rounding of the product and of the sum."""

    def __init__(self, S, z, lam, unit, operand):
        self.S, self.M, self.E = S, np.abs(S), np.zeros_like(S)
        self.z, self.lam, self.unit, self.operand = z, lam, unit, operand

    def decay(self, cut):
        self.S, self.M, self.E = (np.where(cut, 0, self.lam * x) for x in (self.S, self.M, self.E))
        self.E = self.E + (4 * (1 - self.z) + 2) * self.unit * self.M

    def add(self, a, b):
        self.S = self.S + _outer(a, b)
        new = _outer(np.abs(a), np.abs(b))
        self.M = self.M + new
        self.E = self.E + 2 * self.unit * self.M + (4 * self.operand + 4 * self.unit) * new

    def read(self, x, over):
        """The sum over one axis of the state and the bound on its error: products of operands, sums of up to the axis' length, of
        64 steps of a tile and of what joins them."""
        value = over(self.S, x)
        n = x.shape[-1] + 64 + 8
        return value, over(self.E + (n * self.unit + 4 * self.operand) * self.M, np.abs(x))


def forward(q, k, v, log_decay=None, state0=None, reset=None, lengths=None, scale=None, unit=0.0, operand=0.0):
    """o, state_last, {"o": bound, "state_last": bound}"""
    P, B, T, H, K = q.shape
    V, scale = v.shape[-1], K ** -0.5 if scale is None else scale
    q, k, v = (x.astype(np.float64) for x in (q, k, v))
    z, lam, cut, live = _setup(q, v, log_decay, reset, lengths)
    s = _Scan(_start(state0, P, B, H, K, V), z, lam, unit, operand)
    o, Eo = np.zeros((P, B, T, H, V)), np.zeros((P, B, T, H, V))
    with np.errstate(all="ignore"):
        for t in range(T):
            before = (s.S, s.M, s.E)
            s.decay(cut[t])
            s.add(k[:, :, t], v[:, :, t])
            value, E = s.read(q[:, :, t], lambda S, x: _over_keys(x, S))
            on = live[t][..., 0]
            o[:, :, t] = np.where(on, scale * value, 0)
            Eo[:, :, t] = np.where(on, abs(scale) * (E + 2 * unit * np.abs(value)), 0)
            s.S, s.M, s.E = (np.where(live[t], new, old) for new, old in zip((s.S, s.M, s.E), before))
    return o, s.S, {"o": Eo, "state_last": s.E}


def backward(q, k, v, do, log_decay=None, state0=None, reset=None, lengths=None, dstate_last=None, scale=None, unit=0.0, operand=0.0):
    """{"dq", "dk", "dv", "dstate0"} and their bounds."""
    P, B, T, H, K = q.shape
    V, scale = v.shape[-1], K ** -0.5 if scale is None else scale
    q, k, v, do = (x.astype(np.float64) for x in (q, k, v, do))
    z, lam, cut, live = _setup(q, v, log_decay, reset, lengths)
    out = {"dq": np.zeros(q.shape), "dk": np.zeros(k.shape), "dv": np.zeros(v.shape)}
    E = {name: np.zeros(x.shape) for name, x in out.items()}

    def put(name, t, value, bound, factor=1.0):
        on = live[t][..., 0]
        out[name][:, :, t] = np.where(on, factor * value, 0)
        E[name][:, :, t] = np.where(on, abs(factor) * (bound + 2 * unit * np.abs(value)), 0)

    with np.errstate(all="ignore"):
        s = _Scan(_start(state0, P, B, H, K, V), z, lam, unit, operand)
        for t in range(T):
            before = (s.S, s.M, s.E)
            s.decay(cut[t])
            s.add(k[:, :, t], v[:, :, t])
            put("dq", t, *s.read(do[:, :, t], _over_values), factor=scale)
            s.S, s.M, s.E = (np.where(live[t], new, old) for new, old in zip((s.S, s.M, s.E), before))
        s = _Scan(_start(dstate_last, P, B, H, K, V), z, lam, unit, operand)
        for t in reversed(range(T)):
            before = (s.S, s.M, s.E)
            s.add(scale * q[:, :, t], do[:, :, t])
            put("dk", t, *s.read(v[:, :, t], _over_values))
            put("dv", t, *s.read(k[:, :, t], lambda S, x: _over_keys(x, S)))
            s.decay(cut[t])
            s.S, s.M, s.E = (np.where(live[t], new, old) for new, old in zip((s.S, s.M, s.E), before))
    out["dstate0"], E["dstate0"] = s.S, s.E
    return out, E


def step(q, k, v, state, log_decay=None, reset=None, slots=None, scale=None, unit=0.0, operand=0.0):
    """o, new state and their bounds; q, k, v [P, batch, heads, width], state [P, n_slots, heads, K, V]."""
    P, B, H, _ = q.shape
    o, Eo, state = np.zeros(v.shape), np.zeros(v.shape), state.astype(np.float64).copy()
    Es = np.zeros_like(state)
    for p in range(P):
        for r in range(B):
            at = r if slots is None else int(slots[p, r])
            if not 0 <= at < state.shape[1]:
                continue
            one = lambda x: x[p:p + 1, r:r + 1, None]
            y, last, E = forward(one(q), one(k), one(v), None if log_decay is None else log_decay[p:p + 1], state[p, at][None, None],
                                 None if reset is None else reset[p, r].reshape(1, 1, 1), None, scale, unit, operand)
            o[p, r], Eo[p, r] = y[0, 0, 0], E["o"][0, 0, 0]
            state[p, at], Es[p, at] = last[0, 0], E["state_last"][0, 0]
    return o, state, Eo, Es
