"""Performance cases of the operators for populations of recurrent agents: the gated linear recurrence over sequences
(forward, training pass, one step) and the orthogonalised update (the bare orthogonalisation, the whole Muon step).

Every kind of pass exists twice: in its plain form, elementary torch operations in 32 bits (`own` false), and through
the package's entry points (`own` true).  `exact` computes the same outputs from the definitions in 64 bits.

  step     one step of the recurrence for the rows of a state table, as acting agents take it
  forward  the recurrence over sequences, without what a backward pass needs
  train    forward and backward over sequences
  orth     Newton-Schulz orthogonalisation of a stack of matrices
  muon     momentum, orthogonalisation and weight update of the weight matrices of every agent
"""
import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
NS_STEPS, NS_EPS = 5, 1e-7
NS_COEF = (3.4445, -4.7750, 2.0315)


def _seq(name, kind, dtype, agents, batch, T, C, **kw):
    c = {"name": name, "kind": kind, "dtype": dtype, "agents": agents, "batch": batch, "T": T, "C": C,
         "reset": False, "ragged": False, "h0": False, "time_major": False, "packed": False}
    c.update(kw)
    return c


def _mats(name, kind, dtype, agents, shapes, **kw):
    c = {"name": name, "kind": kind, "dtype": dtype, "agents": agents, "nesterov": True}
    for i, (r, k) in enumerate(shapes):
        c["rows%d" % i], c["cols%d" % i] = r, k
    c["shapes"] = len(shapes)
    c.update(kw)
    return c


def listed():
    return [
        # one environment step of the benchmark's smallest population, every agent in one environment: latency
        _seq("step_10_agents_1_row", "step", "f32", 10, 1, 1, 256, reset=True),
        # one step of a large population on 256 environments each, some of which wait for their simulator
        _seq("step_80_agents_256_rows", "step", "bf16", 80, 256, 1, 256, reset=True, ragged=True),
        # values of recorded rollouts of a small population, time-major as simulators fill them
        _seq("forward_10_agents_rollouts", "forward", "f32", 10, 4, 1000, 256, reset=True, h0=True, time_major=True),
        # one agent reads one long history: the work lies along time alone
        _seq("forward_1_agent_long", "forward", "bf16", 1, 1, 65536, 256),
        # a training batch of a large population, candidate and gate from one projection; the largest of the sequences
        _seq("train_80_agents", "train", "bf16", 80, 8, 512, 256, reset=True, packed=True),
        # odd everything, sequences of any length from none on, states carried in and out
        _seq("train_23_agents_ragged", "train", "f32", 23, 3, 777, 129, reset=True, ragged=True, h0=True, packed=True),
        # a few long sequences
        _seq("train_2_agents_long", "train", "f16", 2, 2, 16383, 512, h0=True),
        # the hidden layers of a small population
        _mats("orth_10_hidden", "orth", "f32", 10, [(256, 256)]),
        # large rectangular matrices of a few models
        _mats("orth_4_of_1024_by_4096", "orth", "bf16", 4, [(1024, 4096)]),
        # all weight matrices of the policies of a large population
        _mats("muon_80_policies", "muon", "f32", 80, [(17, 256), (256, 256), (256, 6)]),
        # critics at the widest observations of the benchmark
        _mats("muon_20_wide_critics", "muon", "bf16", 20, [(393, 256), (256, 256), (256, 1)]),
        # odd everything, plain momentum
        _mats("muon_3_ragged", "muon", "f16", 3, [(129, 200), (200, 333), (333, 7)], nesterov=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cost(c):
    w = work(c)
    return w["bytes"] / 4e12 + w["flops"] / 1e14


def draw(rng):
    kind = rng.choice(("step", "forward", "train", "orth", "muon"))
    dtype = rng.choice(("f32", "bf16", "f16"))
    most = max(_cost(c) for c in listed() if c["kind"] in (("orth", "muon") if kind in ("orth", "muon") else ("step", "forward", "train")))
    while True:
        agents = _log_int(rng, 1, 256)
        if kind == "step":
            c = _seq("", kind, dtype, agents, _log_int(rng, 1, 256), 1, _log_int(rng, 32, 1024),
                     reset=rng.random() < 0.5, ragged=rng.random() < 0.5)
        elif kind in ("forward", "train"):
            c = _seq("", kind, dtype, agents, _log_int(rng, 1, 32), _log_int(rng, 1, 65536), _log_int(rng, 32, 1024),
                     reset=rng.random() < 0.5, ragged=rng.random() < 0.5, h0=rng.random() < 0.5,
                     time_major=rng.random() < 0.3, packed=rng.random() < 0.5)
        elif kind == "orth":
            c = _mats("", kind, dtype, agents, [(_log_int(rng, 1, 2048), _log_int(rng, 1, 2048))])
        else:
            obs, act, hidden = _log_int(rng, 3, 376), _log_int(rng, 1, 34), rng.choice((64, 128, 200, 256, 256, 333))
            c = _mats("", kind, dtype, agents, [(obs, hidden), (hidden, hidden), (hidden, act)], nesterov=rng.random() < 0.7)
        if _cost(c) <= most:
            del c["name"]
            return c


def _shapes(c):
    return [(c["rows%d" % i], c["cols%d" % i]) for i in range(c["shapes"])]


def work(case):
    c = case
    e, P = SIZE[c["dtype"]], c["agents"]
    if c["kind"] in ("orth", "muon"):
        nbytes = flops = 0.0
        for r, k in _shapes(c):
            m, n = min(r, k), max(r, k)
            # X X^T and A A are symmetric: half of each
            flops += P * NS_STEPS * (m * m * n + m * m * m + 2.0 * m * m * n)
            nbytes += P * r * k * (2.0 * e if c["kind"] == "orth" else e + 16.0)
        return {"bytes": nbytes, "flops": flops}
    rows = P * c["batch"] * c["C"]
    n = rows * c["T"] * (0.5 if c["ragged"] and c["T"] > 1 else 1.0)
    if c["kind"] == "step":
        return {"bytes": rows * (3.0 * e + 8.0), "flops": 8.0 * rows}
    if c["kind"] == "forward":
        return {"bytes": 2.0 * n * e + rows * c["T"] * e + 4.0 * rows * (2 if c["h0"] else 1), "flops": 8.0 * n}
    return {"bytes": 3.0 * n * e + 3.0 * rows * c["T"] * e + 4.0 * rows * (4 if c["h0"] else 1), "flops": 28.0 * n}


# ---- inputs

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _sequence(c, gen, scale=1.0):
    """[agents, batch, T, C] of the case's type, stored time-major where the case says so."""
    P, B, T, C = c["agents"], c["batch"], c["T"], c["C"]
    shape = (T, P, B, C) if c["time_major"] else (P, B, T, C)
    v = (torch.randn(shape, generator=gen, device="cuda") * scale).to(DTYPES[c["dtype"]])
    return v.permute(1, 2, 0, 3) if c["time_major"] else v


def _sequence_inputs(c, seed):
    P, B, T, C = c["agents"], c["batch"], c["T"], c["C"]
    gen, rng, dt = _gen(seed), random.Random(seed), DTYPES[c["dtype"]]
    s = {"reset": None, "lengths": None, "h0": None, "dh_last": None, "slots": None}
    if c["packed"]:                                     # candidate and gate are the halves of one projection's output
        both = _sequence(dict(c, C=2 * C), gen)
        s["x"], s["g"] = both[..., :C], both[..., C:]
    else:
        s["x"], s["g"] = _sequence(c, gen), _sequence(c, gen)
    # memories of a few to a few hundred steps
    s["bias"] = torch.rand((P, C), generator=gen, device="cuda") * 5 + 0.5
    if c["reset"]:                                      # an episode ends every hundred steps
        r = torch.rand((T, P, B) if c["time_major"] else (P, B, T), generator=gen, device="cuda") < 0.01
        r = r.to(torch.uint8)
        s["reset"] = r.permute(1, 2, 0) if c["time_major"] else r
    if c["kind"] == "step":
        slots = torch.stack([torch.randperm(B, generator=gen, device="cuda") for _ in range(P)]).to(torch.int32)
        if c["ragged"]:
            slots[torch.rand((P, B), generator=gen, device="cuda") < 0.2] = -1
            s["slots"] = slots
        s["state"] = torch.randn((P, B, C), generator=gen, device="cuda") * 0.5
        s["x"], s["g"] = s["x"][:, :, 0], s["g"][:, :, 0]
        s["reset"] = s["reset"][:, :, 0] if c["reset"] else None
        return s
    if c["ragged"]:
        few = [0, 1, T]
        rng.shuffle(few)
        s["lengths"] = torch.tensor([few[i] if i < 3 else rng.randint(0, T) for i in range(P * B)],
                                    dtype=torch.int32, device="cuda").view(P, B)
    if c["h0"]:
        s["h0"] = torch.randn((P, B, C), generator=gen, device="cuda") * 0.5
    if c["kind"] == "train":
        s["dy"] = _sequence(c, gen, 0.1)
        if c["h0"]:
            s["dh_last"] = torch.randn((P, B, C), generator=gen, device="cuda") * 0.1
    return s


def _gradient(c, gen, rows, cols):
    """What a layer's weight gradient is: inputs (behind a ReLU) times output gradients, summed over a batch."""
    P, n = c["agents"], max(256, 2 * max(rows, cols))
    out = torch.empty((P, rows, cols), device="cuda")
    for p in range(P):
        left = torch.relu(torch.randn((n, rows), generator=gen, device="cuda"))
        right = torch.randn((n, cols), generator=gen, device="cuda") * 0.1
        torch.matmul(left.t(), right, out=out[p])
    return (out / n).to(DTYPES[c["dtype"]])


def _matrix_inputs(c, seed):
    gen, rng, P = _gen(seed), random.Random(seed), c["agents"]
    s = {"grads": [_gradient(c, gen, r, k) for r, k in _shapes(c)]}
    if c["kind"] == "muon":
        s["weights"] = [(torch.rand((P, r, k), generator=gen, device="cuda") * 2 - 1) * math.sqrt(6.0 / (r + k)) for r, k in _shapes(c)]
        s["momenta"] = [torch.randn((P, r, k), generator=gen, device="cuda") * 0.01 for r, k in _shapes(c)]
        s["scales"] = [math.sqrt(max(1.0, k / r)) for r, k in _shapes(c)]
        # learning rate, momentum, weight decay of every agent
        s["hparams"] = torch.tensor([[math.exp(rng.uniform(math.log(1e-3), math.log(5e-2))), rng.uniform(0.9, 0.98),
                                      rng.uniform(0.0, 0.1)] for _ in range(P)], dtype=torch.float32, device="cuda")
    return s


def _inputs(case, seed):
    return _matrix_inputs(case, seed) if case["kind"] in ("orth", "muon") else _sequence_inputs(case, seed)


def prepare(case, seed):
    c = case
    s = _inputs(c, seed)
    s["case"] = c
    if own:
        import paper_2206_08888_amd as pp
        if c["kind"] == "orth":
            s["plan"] = pp.Orthogonalizer(c["agents"], c["rows0"], c["cols0"], DTYPES[c["dtype"]], steps=NS_STEPS, eps=NS_EPS)
        elif c["kind"] == "muon":
            s["plan"] = pp.Muon(c["agents"], _shapes(c), DTYPES[c["dtype"]], scales=s["scales"], nesterov=c["nesterov"],
                                steps=NS_STEPS, eps=NS_EPS)
        else:
            s["plan"] = pp.Recurrence(c["agents"], c["batch"], c["T"], c["C"], DTYPES[c["dtype"]])
    torch.cuda.synchronize()
    return s


# ---- the plain forms

def _scan(a, u):
    """h_t = a_t h_{t-1} + u_t along axis 2 from zero, by doubling."""
    d, T = 1, a.shape[2]
    while d < T:
        u = torch.cat([u[:, :, :d], u[:, :, d:] + a[:, :, d:] * u[:, :, :-d]], 2)
        if 2 * d < T:
            a = torch.cat([a[:, :, :d], a[:, :, d:] * a[:, :, :-d]], 2)
        d *= 2
    return u


def _plain_gates(s):
    """Multiplier of the state and of x, the multiplier of the state with resets, which steps exist."""
    x, g = s["x"].float(), s["g"].float() + s["bias"][:, None, None, :]
    a, b = torch.sigmoid(g), torch.sigmoid(-g)
    valid = None
    if s["lengths"] is not None:
        valid = (torch.arange(x.shape[2], device=x.device) < s["lengths"][..., None])[..., None]
    keep = a if s["reset"] is None else torch.where(s["reset"][..., None] != 0, torch.zeros_like(a), a)
    if valid is not None:
        keep = torch.where(valid, keep, torch.ones_like(a))
    return x, a, b, keep, valid


def _plain_forward(s):
    x, a, b, keep, valid = _plain_gates(s)
    u = b * x
    if valid is not None:
        u = torch.where(valid, u, torch.zeros_like(u))
    if s["h0"] is not None:
        u = torch.cat([u[:, :, :1] + keep[:, :, :1] * s["h0"][:, :, None], u[:, :, 1:]], 2)
    h = _scan(keep, u)
    y = h if valid is None else torch.where(valid, h, torch.zeros_like(h))
    return y.to(s["x"].dtype), h


def _plain_train(s):
    y, h = _plain_forward(s)
    x, a, b, keep, valid = _plain_gates(s)
    h0 = s["h0"] if s["h0"] is not None else torch.zeros_like(h[:, :, 0])
    hp = torch.cat([h0[:, :, None], h[:, :, :-1]], 2)
    if s["reset"] is not None:
        hp = torch.where(s["reset"][..., None] != 0, torch.zeros_like(hp), hp)
    dy = s["dy"].float()
    if valid is not None:
        dy = torch.where(valid, dy, torch.zeros_like(dy))
    if s["dh_last"] is not None:
        dy = torch.cat([dy[:, :, :-1], dy[:, :, -1:] + s["dh_last"][:, :, None]], 2)
    after = torch.cat([keep[:, :, 1:], torch.ones_like(keep[:, :, :1])], 2)
    delta = _scan(after.flip(2), dy.flip(2)).flip(2)
    dx, dg = delta * b, delta * (hp - x) * (a * b)
    if valid is not None:
        dx, dg = (torch.where(valid, v, torch.zeros_like(v)) for v in (dx, dg))
    dt = s["x"].dtype
    return {"y": y, "h_last": h[:, :, -1].contiguous(), "dx": dx.to(dt), "dg": dg.to(dt), "dbias": dg.sum((1, 2)),
            "dh0": keep[:, :, 0] * delta[:, :, 0]}


def _plain_step(s):
    g = s["g"].float() + s["bias"][:, None]
    P, B, C = g.shape
    state = s["state"]
    slots = s["slots"] if s["slots"] is not None else torch.arange(B, device=g.device, dtype=torch.int32).expand(P, B)
    on = (slots >= 0)[..., None]
    at = slots.clamp(min=0).long()[..., None].expand(P, B, C)
    h = torch.gather(state, 1, at)
    if s["reset"] is not None:
        h = torch.where(s["reset"][..., None] != 0, torch.zeros_like(h), h)
    h = torch.sigmoid(g) * h + torch.sigmoid(-g) * s["x"].float()
    agent, row = torch.nonzero(on[..., 0], as_tuple=True)
    state[agent, slots[agent, row].long()] = h[agent, row]
    return torch.where(on, h, torch.zeros_like(h)).to(s["x"].dtype)


def _plain_orth(u):
    """Newton-Schulz products on a stack of matrices, in u's type."""
    turn = u.shape[1] > u.shape[2]
    x = u.transpose(1, 2).contiguous() if turn else u
    x = x / (torch.sqrt((x * x).sum((1, 2), keepdim=True)) + NS_EPS)
    a, b, c = NS_COEF
    for _ in range(NS_STEPS):
        A = torch.bmm(x, x.transpose(1, 2).contiguous())
        x = a * x + torch.bmm(b * A + c * torch.bmm(A, A), x)
    return x.transpose(1, 2).contiguous() if turn else x


def _plain_muon(s):
    lr, mu, wd = (s["hparams"][:, i, None, None] for i in range(3))
    for w, m, g, scale in zip(s["weights"], s["momenta"], s["grads"], s["scales"]):
        g = g.float()
        m.mul_(mu).add_(g)
        o = _plain_orth(g + mu * m if s["case"]["nesterov"] else m)
        w.mul_(1 - lr * wd).sub_(lr * scale * o)


def _run_plain(s):
    kind = s["case"]["kind"]
    if kind == "step":
        return {"y": _plain_step(s), "state": s["state"]}
    if kind == "forward":
        y, h = _plain_forward(s)
        return {"y": y, "h_last": h[:, :, -1].contiguous()}
    if kind == "train":
        return _plain_train(s)
    if kind == "orth":
        return _plain_orth(s["grads"][0].float()).to(s["grads"][0].dtype)
    _plain_muon(s)
    return {"weights": s["weights"], "momenta": s["momenta"]}


def _run_own(s):
    plan, kind = s["plan"], s["case"]["kind"]
    if kind == "step":
        return {"y": plan.step(s["x"], s["g"], s["state"], bias=s["bias"], reset=s["reset"], slots=s["slots"]), "state": s["state"]}
    if kind == "forward":
        y, h_last = plan.forward(s["x"], s["g"], bias=s["bias"], h0=s["h0"], reset=s["reset"], lengths=s["lengths"])
        return {"y": y, "h_last": h_last}
    if kind == "train":
        y, h_last, states = plan.forward(s["x"], s["g"], bias=s["bias"], h0=s["h0"], reset=s["reset"], lengths=s["lengths"],
                                         save=True)
        dx, dg, dbias, dh0 = plan.backward(states, s["x"], s["g"], s["dy"], bias=s["bias"], reset=s["reset"],
                                           lengths=s["lengths"], dh_last=s["dh_last"])
        return {"y": y, "h_last": h_last, "dx": dx, "dg": dg, "dbias": dbias, "dh0": dh0}
    if kind == "orth":
        return plan(s["grads"][0])
    plan.step(s["weights"], s["momenta"], s["grads"], s["hparams"])
    return {"weights": s["weights"], "momenta": s["momenta"]}


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---- the definitions in 64 bits

def _exact_sequence(c, s):
    x, g = s["x"].double(), s["g"].double() + s["bias"].double()[:, None, None]
    P, B, T, C = x.shape
    a = 1 / (1 + torch.exp(-g))
    del g
    length = s["lengths"].long() if s["lengths"] is not None else torch.full((P, B), T, device=x.device)
    live = [None if s["lengths"] is None else (t < length)[..., None] for t in range(T)]
    stays = [None if s["reset"] is None else (s["reset"][:, :, t] == 0).double()[..., None] for t in range(T)]
    h = s["h0"].double() if s["h0"] is not None else torch.zeros((P, B, C), dtype=torch.float64, device=x.device)
    y, before = torch.zeros_like(x), torch.zeros_like(x)
    for t in range(T):
        kept = h if stays[t] is None else h * stays[t]
        before[:, :, t] = kept
        new = torch.lerp(x[:, :, t], kept, a[:, :, t])
        if live[t] is not None:
            y[:, :, t] = new * live[t]
            h = torch.where(live[t], new, h)
        else:
            y[:, :, t] = new
            h = new
    if c["kind"] == "forward":
        return {"y": y, "h_last": h}
    d = s["dh_last"].double() if s["dh_last"] is not None else torch.zeros_like(h)
    dx, dg = torch.zeros_like(x), torch.zeros_like(x)
    for t in reversed(range(T)):
        at = d + s["dy"][:, :, t].double()
        through = at * a[:, :, t]
        dx_t, dg_t = at - through, at * (before[:, :, t] - x[:, :, t]) * a[:, :, t] * (1 - a[:, :, t])
        back = through if stays[t] is None else through * stays[t]
        if live[t] is not None:
            dx_t, dg_t, back = dx_t * live[t], dg_t * live[t], torch.where(live[t], back, d)
        dx[:, :, t], dg[:, :, t], d = dx_t, dg_t, back
    return {"y": y, "h_last": h, "dx": dx, "dg": dg, "dbias": dg.sum(2).sum(1), "dh0": d}


def _exact_step(s):
    g = s["g"].double() + s["bias"].double()[:, None]
    P, B, C = g.shape
    state, y = s["state"].double(), torch.zeros_like(g)
    slots = s["slots"].tolist() if s["slots"] is not None else [list(range(B))] * P
    a = 1 / (1 + torch.exp(-g))
    for p in range(P):
        rows = [b for b in range(B) if slots[p][b] >= 0]
        at = [slots[p][b] for b in rows]
        h = state[p, at]
        if s["reset"] is not None:
            h = h * (s["reset"][p, rows] == 0).double()[:, None]
        new = a[p, rows] * h + (1 - a[p, rows]) * s["x"][p, rows].double()
        y[p, rows] = new
        state[p, at] = new
    return {"y": y, "state": state}


def _exact_orth(u):
    out = torch.empty_like(u)
    a, b, c = NS_COEF
    for p in range(u.shape[0]):
        x = u[p] / (torch.linalg.norm(u[p]) + NS_EPS)
        for _ in range(NS_STEPS):                       # the same polynomial from whichever side is the smaller
            if x.shape[0] <= x.shape[1]:
                A = x @ x.t()
                x = a * x + b * (A @ x) + c * (A @ (A @ x))
            else:
                A = x.t() @ x
                x = a * x + b * (x @ A) + c * ((x @ A) @ A)
        out[p] = x
    return out


def exact(case, seed):
    c, s = case, _inputs(case, seed)
    if c["kind"] == "step":
        return _exact_step(s)
    if c["kind"] in ("forward", "train"):
        return _exact_sequence(c, s)
    if c["kind"] == "orth":
        return _exact_orth(s["grads"][0].double())
    lr, mu, wd = (s["hparams"][:, i, None, None].double() for i in range(3))
    weights, momenta = [], []
    for w, m, g, scale in zip(s["weights"], s["momenta"], s["grads"], s["scales"]):
        m, g = m.double(), g.double()
        m = mu * m + g
        o = _exact_orth(g + mu * m if c["nesterov"] else m)
        weights.append(w.double() * (1 - lr * wd) - lr * scale * o)
        momenta.append(m)
    return {"weights": weights, "momenta": momenta}
