"""Performance cases of the operators for agents with a matrix for a memory, and for their gradients: linear attention with a
decay for each head (one step, forward, training pass) and the norm of every agent's gradients with clipping.

Every kind of pass exists twice: in its plain form, elementary torch operations in 32 bits (`own` false), and through
the package's entry points (`own` true).  `exact` computes the same outputs from the definitions in 64 bits.

  step     one step for the rows of a state table, as acting agents take it
  forward  whole sequences, without a backward pass
  train    forward and backward over sequences
  clip     the norm of every agent's gradients over all of its tensors, and the gradients scaled down where it is above the agent's limit
"""
import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
CHUNK = 64                                               # steps that the plain form takes as one product
CLIP_EPS = 1e-6


def _seq(name, kind, dtype, agents, batch, T, heads, key, value, **kw):
    c = {"name": name, "kind": kind, "dtype": dtype, "agents": agents, "batch": batch, "T": T, "heads": heads, "key": key, "value": value,
         "reset": False, "ragged": False, "state0": False, "time_major": False, "packed": False}
    c.update(kw)
    return c


def _grads(name, kind, dtype, agents, obs, act, hidden, layers, **kw):
    """Gradients of a network obs -> hidden -> ... -> act with `layers` matrices and their biases."""
    c = {"name": name, "kind": kind, "dtype": dtype, "agents": agents, "obs": obs, "act": act, "hidden": hidden, "layers": layers}
    c.update(kw)
    return c


def listed():
    return [
        # one environment step of the benchmark's smallest population, every agent in one environment: latency
        _seq("step_10_agents_1_row", "step", "f32", 10, 1, 1, 4, 64, 64, reset=True),
        # one step of a large population on 64 environments each, some of which wait for their simulator
        _seq("step_80_agents_64_rows", "step", "bf16", 80, 64, 1, 4, 64, 64, reset=True, ragged=True),
        # values of recorded rollouts of a small population, time-major as simulators fill them
        _seq("forward_10_agents_rollouts", "forward", "f32", 10, 4, 1000, 4, 64, 64, reset=True, state0=True, time_major=True),
        # one agent reads one long history: the work lies along time alone
        _seq("forward_1_agent_long", "forward", "bf16", 1, 1, 65536, 4, 64, 64),
        # a training batch of a large population, queries, keys and values from one projection; the largest of the sequences
        _seq("train_80_agents", "train", "bf16", 80, 8, 512, 4, 64, 64, reset=True, packed=True),
        # odd everything, sequences of any length from none on, states carried in and out
        _seq("train_23_agents_ragged", "train", "f32", 23, 3, 777, 3, 24, 41, reset=True, ragged=True, state0=True, packed=True),
        # a few long sequences with the largest heads
        _seq("train_2_agents_long", "train", "f16", 2, 2, 16383, 4, 128, 128, state0=True),
        # the policies of a small population, six tensors each: latency
        _grads("clip_10_policies", "clip", "f32", 10, 17, 6, 256, 3),
        # critics of a large population at the widest observations of the benchmark
        _grads("clip_80_wide_critics", "clip", "bf16", 80, 393, 1, 256, 3),
        # a few large networks of many layers; the largest of the gradients
        _grads("clip_4_large", "clip", "f32", 4, 376, 17, 2048, 9),
        # odd everything
        _grads("clip_23_odd", "clip", "f16", 23, 129, 7, 333, 5),
        # the policies of a large population
        _grads("clip_80_policies", "clip", "f32", 80, 17, 6, 256, 3),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cost(c):
    w = work(c)
    return w["bytes"] / 4e12 + w["flops"] / 1e14


def draw(rng):
    kind = rng.choice(("step", "forward", "train", "train", "clip", "clip"))
    dtype = rng.choice(("f32", "bf16", "f16"))
    most = max(_cost(c) for c in listed() if (c["kind"] == "clip") == (kind == "clip"))
    while True:
        agents = _log_int(rng, 1, 256)
        if kind == "clip":
            c = _grads("", kind, dtype, agents, _log_int(rng, 3, 400), _log_int(rng, 1, 34), _log_int(rng, 16, 2048), rng.randint(1, 9))
        else:
            key = _log_int(rng, 8, 128)
            value = key if rng.random() < 0.5 else _log_int(rng, 8, 128)
            heads = rng.randint(1, 8)
            if kind == "step":
                c = _seq("", kind, dtype, agents, _log_int(rng, 1, 256), 1, heads, key, value, reset=rng.random() < 0.5, ragged=rng.random() < 0.5)
            else:
                c = _seq("", kind, dtype, agents, _log_int(rng, 1, 32), _log_int(rng, 1, 65536 if kind == "forward" else 16384), heads, key, value,
                         reset=rng.random() < 0.5, ragged=rng.random() < 0.5, state0=rng.random() < 0.5,
                         time_major=rng.random() < 0.3, packed=rng.random() < 0.5)
        if _cost(c) <= most:
            del c["name"]
            return c


def _shapes(c):
    widths = [c["obs"]] + [c["hidden"]] * (c["layers"] - 1) + [c["act"]]
    out = []
    for r, k in zip(widths, widths[1:]):
        out += [(r, k), (k,)]
    return out


def work(case):
    c = case
    e, P = SIZE[c["dtype"]], c["agents"]
    if c["kind"] == "clip":
        n = float(P * sum(math.prod(s) for s in _shapes(c)))
        return {"bytes": n * e * 2 + 8.0 * P, "flops": 3.0 * n}
    rows, Dk, Dv = float(P * c["batch"] * c["heads"]), c["key"], c["value"]
    n = rows * c["T"] * (0.5 if c["ragged"] and c["T"] > 1 else 1.0)        # steps that exist; outputs are written for all
    if c["kind"] == "step":
        n = rows * (0.8 if c["ragged"] else 1.0)
        return {"bytes": n * e * (2 * Dk + Dv) + rows * e * Dv + 8.0 * n * Dk * Dv, "flops": 5.0 * n * Dk * Dv}
    states = 4.0 * rows * Dk * Dv * (2 if c["state0"] else 1)
    nbytes = n * e * (2 * Dk + Dv) + rows * c["T"] * e * Dv + states
    if c["kind"] == "forward":
        return {"bytes": nbytes, "flops": 4.0 * n * Dk * Dv}
    nbytes += n * e * (2 * Dk + 2 * Dv) + rows * c["T"] * e * (2 * Dk + Dv) + states * (1.5 if c["state0"] else 1.0)
    return {"bytes": nbytes, "flops": 14.0 * n * Dk * Dv}


# ---- inputs

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _sequence(c, gen, width, scale=1.0):
    """[agents, batch, T, width] of the case's type, stored time-major where the case says so."""
    P, B, T = c["agents"], c["batch"], c["T"]
    shape = (T, P, B, width) if c["time_major"] else (P, B, T, width)
    v = (torch.randn(shape, generator=gen, device="cuda") * scale).to(DTYPES[c["dtype"]])
    return v.permute(1, 2, 0, 3) if c["time_major"] else v


def _sequence_inputs(c, seed):
    P, B, T, H, Dk, Dv = c["agents"], c["batch"], c["T"], c["heads"], c["key"], c["value"]
    gen, rng = _gen(seed), random.Random(seed)
    s = {"reset": None, "lengths": None, "state0": None, "dstate_last": None, "slots": None}
    if c["packed"]:                                     # queries, keys and values are parts of one projection's output
        parts = _sequence(c, gen, H * (2 * Dk + Dv)).split((H * Dk, H * Dk, H * Dv), -1)
    else:
        parts = [_sequence(c, gen, H * D) for D in (Dk, Dk, Dv)]
    s["q"], s["k"], s["v"] = (x.unflatten(-1, (H, D)) for x, D in zip(parts, (Dk, Dk, Dv)))
    # memories of four to five hundred steps
    s["log_decay"] = -torch.exp(torch.rand((P, H), generator=gen, device="cuda") * math.log(128.0) - math.log(512.0))
    if c["reset"]:                                      # an episode ends every hundred steps
        r = torch.rand((T, P, B) if c["time_major"] else (P, B, T), generator=gen, device="cuda") < 0.01
        r = r.to(torch.uint8)
        s["reset"] = r.permute(1, 2, 0) if c["time_major"] else r
    if c["kind"] == "step":
        slots = torch.stack([torch.randperm(B, generator=gen, device="cuda") for _ in range(P)]).to(torch.int32)
        if c["ragged"]:
            slots[torch.rand((P, B), generator=gen, device="cuda") < 0.2] = -1
            s["slots"] = slots
        s["state"] = torch.randn((P, B, H, Dk, Dv), generator=gen, device="cuda")
        s["q"], s["k"], s["v"] = s["q"][:, :, 0], s["k"][:, :, 0], s["v"][:, :, 0]
        s["reset"] = s["reset"][:, :, 0] if c["reset"] else None
        return s
    if c["ragged"]:
        few = [0, 1, T]
        rng.shuffle(few)
        s["lengths"] = torch.tensor([few[i] if i < 3 else rng.randint(0, T) for i in range(P * B)],
                                    dtype=torch.int32, device="cuda").view(P, B)
    if c["state0"]:
        s["state0"] = torch.randn((P, B, H, Dk, Dv), generator=gen, device="cuda")
    if c["kind"] == "train":
        s["do"] = _sequence(c, gen, H * Dv, 0.1).unflatten(-1, (H, Dv))
        if c["state0"]:
            s["dstate_last"] = torch.randn((P, B, H, Dk, Dv), generator=gen, device="cuda") * 0.1
    return s


def _gradient_inputs(c, seed):
    gen, P = _gen(seed), c["agents"]
    grads = [(torch.randn((P, *shape), generator=gen, device="cuda") * 0.02).to(DTYPES[c["dtype"]]) for shape in _shapes(c)]
    # limits around the norms: about half of the agents are above theirs
    usual = 0.02 * math.sqrt(sum(math.prod(shape) for shape in _shapes(c)))
    return {"grads": grads, "max_norm": usual * torch.exp(torch.rand(P, generator=gen, device="cuda") * 2 - 1)}


def _inputs(case, seed):
    return _gradient_inputs(case, seed) if case["kind"] == "clip" else _sequence_inputs(case, seed)


def prepare(case, seed):
    c = case
    s = _inputs(c, seed)
    s["case"] = c
    if own:
        import paper_2206_08888_amd as pp
        if c["kind"] == "clip":
            s["plan"] = pp.GradientClip(c["agents"], _shapes(c), DTYPES[c["dtype"]], eps=CLIP_EPS)
        else:
            s["plan"] = pp.LinearAttention(c["agents"], c["batch"], c["T"], c["heads"], c["key"], c["value"], DTYPES[c["dtype"]])
    torch.cuda.synchronize()
    return s


# ---- the plain forms

def _rows(x):
    """[P, B, T, H, D] -> [P * B * H, T, D] in 32 bits."""
    P, B, T, H, D = x.shape
    return x.float().permute(0, 1, 3, 2, 4).reshape(P * B * H, T, D)


def _unrows(x, like):
    P, B, T, H, D = like.shape
    return x.view(P, B, H, T, D).permute(0, 1, 3, 2, 4).to(like.dtype).contiguous()


def _links(s):
    """What the state is multiplied with on its way to step t, as a logarithm [N, T] (0 behind a sequence's end), whether it is cut
    off there, and which steps exist (or None)."""
    P, B, T, H, _ = s["q"].shape
    log = s["log_decay"].double()[:, None, :, None].expand(P, B, H, T)
    cut = valid = None
    if s["lengths"] is not None:
        valid = (torch.arange(T, device=log.device) < s["lengths"][..., None])[:, :, None].expand(P, B, H, T)
        log = torch.where(valid, log, torch.zeros_like(log))
    if s["reset"] is not None:
        cut = (s["reset"] != 0)[:, :, None].expand(P, B, H, T)
        cut = (cut if valid is None else cut & valid).reshape(-1, T)
    return log.reshape(-1, T), cut, None if valid is None else valid.reshape(-1, T)


def _chunked(x, n):
    pad = n * CHUNK - x.shape[1]
    if pad:
        x = torch.cat([x, x.new_zeros((x.shape[0], pad, *x.shape[2:]))], 1)
    return x.view(x.shape[0], n, CHUNK, *x.shape[2:])


def _linear(q, k, v, log, cut, first):
    """o_t = q_t S_t, S_t = exp(log_t) keep_t S_{t-1} + k_t v_t^T from `first`: products within chunks, a scan over them."""
    N, T, Dk = q.shape
    n = max(1, -(-T // CHUNK))
    q, k, v = (_chunked(x, n) for x in (q, k, v))
    G = _chunked(log, n).cumsum(2)
    pair = torch.ones((CHUNK, CHUNK), dtype=torch.bool, device=q.device).tril()
    into, out, whole = torch.exp(G).float(), torch.exp(G[..., -1:] - G).float(), torch.exp(G[..., -1]).float()
    if cut is not None:
        seg = _chunked(cut.to(torch.int32), n).cumsum(2)
        pair = pair & (seg[..., :, None] == seg[..., None, :])
        into, out = into * (seg == 0), out * (seg == seg[..., -1:])
        whole = whole * (seg[..., -1] == 0)
    weight = torch.where(pair, torch.exp((G[..., :, None] - G[..., None, :]).clamp(max=0)).float(), torch.zeros((), device=q.device))
    o = torch.matmul(torch.matmul(q, k.transpose(2, 3).contiguous()) * weight, v)
    S = torch.matmul((k * out[..., None]).transpose(2, 3).contiguous(), v)
    A = whole[..., None, None]
    S = torch.cat([S[:, :1] + A[:, :1] * first[:, None], S[:, 1:]], 1)
    d = 1
    while d < n:
        S = torch.cat([S[:, :d], S[:, d:] + A[:, d:] * S[:, :-d]], 1)
        A = torch.cat([A[:, :d], A[:, d:] * A[:, :-d]], 1)
        d *= 2
    before = torch.cat([first[:, None], S[:, :-1]], 1)
    o = o + into[..., None] * torch.matmul(q, before)
    return o.reshape(N, n * CHUNK, -1)[:, :T], S[:, -1]


def _first(state, N, Dk, Dv, device):
    return torch.zeros((N, Dk, Dv), device=device) if state is None else state.reshape(N, Dk, Dv)


def _existing(x, valid):
    return x if valid is None else torch.where(valid[..., None], x, torch.zeros_like(x))


def _plain_forward(s):
    P, B, T, H, Dk = s["q"].shape
    Dv = s["v"].shape[-1]
    log, cut, valid = _links(s)
    q, k, v = (_existing(_rows(s[name]), valid) for name in ("q", "k", "v"))
    o, last = _linear(q * Dk ** -0.5, k, v, log, cut, _first(s["state0"], P * B * H, Dk, Dv, q.device))
    return _unrows(o, s["v"]), last.view(P, B, H, Dk, Dv)


def _plain_train(s):
    P, B, T, H, Dk = s["q"].shape
    Dv, N = s["v"].shape[-1], P * B * H
    o, last = _plain_forward(s)
    log, cut, valid = _links(s)
    q, k, v, do = (_existing(_rows(s[name]), valid) for name in ("q", "k", "v", "do"))
    q, scale = q * Dk ** -0.5, Dk ** -0.5
    first = _first(s["state0"], N, Dk, Dv, q.device)
    dq = _linear(do, v, k, log, cut, first.transpose(1, 2).contiguous())[0] * scale
    # from the end: what leads from step t + 1 back to step t
    behind = torch.cat([log[:, 1:], torch.zeros_like(log[:, :1])], 1).flip(1)
    cut_behind = None if cut is None else torch.cat([cut[:, 1:], torch.zeros_like(cut[:, :1])], 1).flip(1)
    q, k, v, do = (x.flip(1) for x in (q, k, v, do))
    after = _first(s["dstate_last"], N, Dk, Dv, q.device)
    dv, d = _linear(k, q, do, behind, cut_behind, after)
    dk = _linear(v, do, q, behind, cut_behind, after.transpose(1, 2).contiguous())[0]
    d = d * torch.exp(log[:, 0]).float()[:, None, None]
    if cut is not None:
        d = torch.where(cut[:, 0, None, None], torch.zeros_like(d), d)
    dq, dk, dv = _existing(dq, valid), _existing(dk.flip(1), valid), _existing(dv.flip(1), valid)
    return {"o": o, "state_last": last, "dq": _unrows(dq, s["q"]), "dk": _unrows(dk, s["k"]), "dv": _unrows(dv, s["v"]),
            "dstate0": d.view(P, B, H, Dk, Dv)}


def _plain_step(s):
    q, k, v, state = s["q"].float(), s["k"].float(), s["v"].float(), s["state"]
    P, B, H, Dk = q.shape
    slots = s["slots"] if s["slots"] is not None else torch.arange(B, device=q.device, dtype=torch.int32).expand(P, B)
    on = slots >= 0
    agent = torch.arange(P, device=q.device)[:, None].expand(P, B)
    S = state[agent, slots.clamp(min=0).long()]
    if s["reset"] is not None:
        S = torch.where((s["reset"] != 0)[..., None, None, None], torch.zeros_like(S), S)
    S = torch.exp(s["log_decay"])[:, None, :, None, None] * S + k[..., :, None] * v[..., None, :]
    o = (q[..., :, None] * S).sum(-2) * Dk ** -0.5
    p, b = torch.nonzero(on, as_tuple=True)
    state[p, slots[p, b].long()] = S[p, b]
    return torch.where(on[..., None, None], o, torch.zeros_like(o)).to(s["v"].dtype)


def _plain_clip(s):
    norms = torch.sqrt(sum(torch.sum(g.float().square().flatten(1), 1, dtype=torch.float64) for g in s["grads"]))
    above = norms + CLIP_EPS
    factor = torch.where(above <= s["max_norm"], torch.ones_like(above), s["max_norm"] / above).float()
    return {"grads": [(g.float() * factor.view(-1, *[1] * (g.dim() - 1))).to(g.dtype) for g in s["grads"]], "norms": norms.float()}


def _run_plain(s):
    kind = s["case"]["kind"]
    if kind == "step":
        return {"o": _plain_step(s), "state": s["state"]}
    if kind == "forward":
        o, last = _plain_forward(s)
        return {"o": o, "state_last": last}
    if kind == "train":
        return _plain_train(s)
    return _plain_clip(s)


def _run_own(s):
    plan, kind = s["plan"], s["case"]["kind"]
    if kind == "clip":
        grads, norms = plan(s["grads"], s["max_norm"])
        return {"grads": grads, "norms": norms}
    if kind == "step":
        return {"o": plan.step(s["q"], s["k"], s["v"], s["state"], s["log_decay"], reset=s["reset"], slots=s["slots"]), "state": s["state"]}
    given = dict(log_decay=s["log_decay"], state0=s["state0"], reset=s["reset"], lengths=s["lengths"])
    o, last = plan.forward(s["q"], s["k"], s["v"], **given)
    if kind == "forward":
        return {"o": o, "state_last": last}
    dq, dk, dv, dstate0 = plan.backward(s["q"], s["k"], s["v"], s["do"], dstate_last=s["dstate_last"], **given)
    return {"o": o, "state_last": last, "dq": dq, "dk": dk, "dv": dv, "dstate0": dstate0}


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---- the definitions in 64 bits

def _exact_sequence(c, s):
    q, k, v = (s[name].double() for name in ("q", "k", "v"))
    P, B, T, H, Dk = q.shape
    Dv, scale = v.shape[-1], c["key"] ** -0.5
    decay = torch.exp(s["log_decay"].double())[:, None, :, None, None]
    length = s["lengths"].long() if s["lengths"] is not None else torch.full((P, B), T, device=q.device)
    lam = [decay if s["reset"] is None else decay * (s["reset"][:, :, t] == 0).double()[:, :, None, None, None] for t in range(T)]
    live = [None if s["lengths"] is None else (t < length)[:, :, None, None] for t in range(T)]
    S = s["state0"].double() if s["state0"] is not None else torch.zeros((P, B, H, Dk, Dv), dtype=torch.float64, device=q.device)
    train = c["kind"] == "train"
    o = torch.zeros_like(v)
    dq, do = (torch.zeros_like(q), s["do"].double()) if train else (None, None)
    for t in range(T):
        new = torch.addcmul(S * lam[t], k[:, :, t, :, :, None], v[:, :, t, :, None, :])
        S = new if live[t] is None else torch.where(live[t][..., None], new, S)
        o[:, :, t] = scale * (q[:, :, t, :, None, :] @ new).squeeze(-2)
        if train:
            dq[:, :, t] = scale * (new @ do[:, :, t, :, :, None]).squeeze(-1)
        if live[t] is not None:
            for x in (o, dq) if train else (o,):
                x[:, :, t] = torch.where(live[t], x[:, :, t], 0)
    if not train:
        return {"o": o, "state_last": S}
    D = s["dstate_last"].double() if s["dstate_last"] is not None else torch.zeros_like(S)
    dk, dv = torch.zeros_like(k), torch.zeros_like(v)
    for t in reversed(range(T)):
        at = torch.addcmul(D, scale * q[:, :, t, :, :, None], do[:, :, t, :, None, :])
        dk[:, :, t] = (at @ v[:, :, t, :, :, None]).squeeze(-1)
        dv[:, :, t] = (k[:, :, t, :, None, :] @ at).squeeze(-2)
        back = at * lam[t]
        D = back if live[t] is None else torch.where(live[t][..., None], back, D)
        if live[t] is not None:
            for x in (dk, dv):
                x[:, :, t] = torch.where(live[t], x[:, :, t], 0)
    return {"o": o, "state_last": S, "dq": dq, "dk": dk, "dv": dv, "dstate0": D}


def _exact_step(c, s):
    q, k, v, state = (s[name].double() for name in ("q", "k", "v", "state"))
    P, B, H, _ = q.shape
    o = torch.zeros_like(v)
    slots = s["slots"].tolist() if s["slots"] is not None else [list(range(B))] * P
    decay = torch.exp(s["log_decay"].double())[:, :, None, None]
    for p in range(P):
        rows = [b for b in range(B) if slots[p][b] >= 0]
        at = [slots[p][b] for b in rows]
        S = decay[p] * state[p, at]
        if s["reset"] is not None:
            S = S * (s["reset"][p, rows] == 0).double()[:, None, None, None]
        S = S + k[p, rows][..., None] * v[p, rows][..., None, :]
        state[p, at] = S
        o[p, rows] = c["key"] ** -0.5 * (q[p, rows][..., None, :] @ S).squeeze(-2)
    return {"o": o, "state": state}


def exact(case, seed):
    c, s = case, _inputs(case, seed)
    if c["kind"] == "clip":
        norms = torch.stack([torch.linalg.norm(torch.cat([g[p].double().flatten() for g in s["grads"]])) for p in range(c["agents"])])
        limit = s["max_norm"].double()
        factor = [1.0 if n + CLIP_EPS <= m else m / (n + CLIP_EPS) for n, m in zip(norms.tolist(), limit.tolist())]
        return {"grads": [torch.stack([g[p].double() * factor[p] for p in range(c["agents"])]) for g in s["grads"]], "norms": norms}
    if c["kind"] == "step":
        return _exact_step(c, s)
    if c["agents"] * c["batch"] * c["heads"] * c["key"] * c["value"] * c["T"] > 5e10 or c["T"] > 70000:
        return None
    return _exact_sequence(c, s)
