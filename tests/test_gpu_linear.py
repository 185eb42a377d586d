"""Linear attention with a decay for each head on the GPU against the oracle in 64 bits, element by element."""
import numpy as np
import pytest
import torch

import paper_2206_08888_amd as pp
from gpu_common import ensure_built
from linear_common import BF16, F16, F32, OPERAND, UNIT, check, check_backward, check_forward, make, numpy_of, plan_of
from oracle import linear as L

pytestmark = pytest.mark.gpu
TYPES = [F32, BF16, F16]
SHAPES = [  # P, batch, T, heads, key_dim, value_dim
    (1, 1, 1, 1, 1, 1), (2, 3, 64, 2, 16, 16), (1, 2, 65, 3, 33, 7), (2, 1, 130, 1, 64, 64), (1, 1, 200, 2, 128, 128), (1, 2, 77, 1, 5, 128),
    (1, 1, 63, 1, 128, 1), (3, 2, 129, 4, 24, 41), (1, 1, 300, 1, 96, 72), (5, 1, 31, 1, 40, 80)]


@pytest.fixture(autouse=True, scope="module")
def _built():
    ensure_built()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_forward_and_backward(shape, dtype):
    c, do, dlast = make(shape, dtype, seed=sum(shape))
    check_forward(shape, dtype, c)
    check_backward(shape, dtype, c, do, dlast)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES[1:8:2])
def test_resets_lengths_and_states(shape, dtype):
    c, do, dlast = make(shape, dtype, seed=sum(shape), reset=0.03, ragged=True, state0=True)
    check_forward(shape, dtype, c)
    check_backward(shape, dtype, c, do, dlast)
    c["reset"] = c["reset"].to(torch.uint8) * 7          # any value but zero
    check_forward(shape, dtype, c)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("layout", ["time_major", "head_major", "packed", "padded", "broadcast"])
@pytest.mark.parametrize("shape", [(2, 3, 70, 2, 32, 64), (1, 2, 67, 3, 9, 21)])
def test_layouts(shape, layout, dtype):
    c, do, dlast = make(shape, dtype, layout=layout, ragged=True, state0=True)
    check_forward(shape, dtype, c)
    check_backward(shape, dtype, c, do, dlast)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rate", [1.0, 0.3])
def test_every_step_and_many_start_episodes(rate, dtype):
    shape = (1, 2, 140, 2, 20, 48)
    c, do, dlast = make(shape, dtype, reset=rate, state0=True)
    check_forward(shape, dtype, c)
    check_backward(shape, dtype, c, do, dlast)


@pytest.mark.parametrize("shape", [(1, 1, 4100, 1, 64, 64), (1, 2, 3000, 1, 32, 16), (2, 1, 2500, 2, 17, 40)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_few_long_sequences(shape, dtype):
    c, do, dlast = make(shape, dtype, seed=3, decay=(0.0005, 0.05), reset=0.0005, ragged=shape[1] > 1, state0=True)
    check_forward(shape, dtype, c)
    check_backward(shape, dtype, c, do, dlast)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("log", [0.0, -1e-6, -30.0, -200.0, -1e30, float("-inf"), 3.0, None])
def test_decays(log, dtype):
    """No decay, one within fp32's last bits, ones that leave nothing of a state, ones beyond the range (taken as its ends)."""
    shape = (1, 1, 150, 2, 16, 24)
    c, do, dlast = make(shape, dtype, state0=True)
    c["log_decay"] = None if log is None else torch.full((1, 2), log, device="cuda")
    check_forward(shape, dtype, c)
    check_backward(shape, dtype, c, do, dlast)


@pytest.mark.parametrize("scale", [0.0, -2.5, 1.0])
def test_scales(scale):
    shape = (1, 1, 80, 1, 16, 24)
    c, do, dlast = make(shape, F32, state0=True)
    check_forward(shape, F32, c, scale=scale)
    check_backward(shape, F32, c, do, dlast, scale=scale)


def test_no_steps():
    plan = pp.LinearAttention(2, 3, 8, 2, 5, 6)
    q, v = torch.empty((2, 3, 0, 2, 5), device="cuda"), torch.empty((2, 3, 0, 2, 6), device="cuda")
    s = torch.randn((2, 3, 2, 5, 6), device="cuda")
    o, last = plan.forward(q, q, v, state0=s)
    assert o.shape == v.shape and torch.equal(last, s)
    assert not plan.forward(q, q, v)[1].any()
    dq, dk, dv, d0 = plan.backward(q, q, v, v, state0=s, dstate_last=s)
    assert dq.shape == q.shape and torch.equal(d0, s) and not plan.backward(q, q, v, v)[3].any()


@pytest.mark.parametrize("dtype", TYPES)
def test_lengths_outside_the_range(dtype):
    shape = (1, 4, 70, 1, 16, 8)
    c, do, dlast = make(shape, dtype, state0=True)
    c["lengths"] = torch.tensor([[-5, 1000, 1, 70]], dtype=torch.int32, device="cuda")
    check_forward(shape, dtype, c)
    check_backward(shape, dtype, c, do, dlast)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("at", [0, 5, 63, 64, 100])
def test_what_is_not_finite_stays_where_it_belongs(at, bad, dtype):
    """One value of k or v: not the steps before it (behind it, backward), not other columns, not other heads and sequences, nothing
    behind a reset, nothing where a length ends before it."""
    shape = (1, 3, 160, 2, 20, 36)
    c, do, dlast = make(shape, dtype, state0=True)
    c["reset"] = torch.zeros((1, 3, 160), dtype=torch.bool, device="cuda")
    c["reset"][:, :, 120] = True
    c["reset"][0, 2, 70] = True
    c["lengths"] = torch.tensor([[160, 4, 160]], dtype=torch.int32, device="cuda")
    for name, index in (("k", (0, 0, at, 0, 3)), ("v", (0, 2, at, 1, 30)), ("k", (0, 1, at, 1, 0)), ("q", (0, 2, at, 0, 19))):
        c[name][index] = bad
    check_forward(shape, dtype, c)
    check_backward(shape, dtype, c, do, dlast)
    do[0, 0, at, 1, 2] = bad
    check_backward(shape, dtype, c, do, dlast)


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_states_that_are_not_finite(bad):
    shape = (1, 2, 150, 1, 12, 20)
    c, do, dlast = make(shape, F32, state0=True)
    c["reset"] = torch.zeros((1, 2, 150), dtype=torch.bool, device="cuda")
    c["reset"][0, 0, 0] = c["reset"][0, 1, 90] = True    # dropped at once, and later
    c["state0"][:, :, 0, 2, 7] = bad
    dlast[:, :, 0, 1, 3] = bad
    check_forward(shape, F32, c)
    check_backward(shape, F32, c, do, dlast)


def test_nothing_is_written_outside():
    """Outputs in the middle of larger arrays, through the boundary's own structures."""
    import ctypes as ct
    from paper_2206_08888_amd import operators as ops
    shape = (2, 2, 70, 2, 12, 20)
    P, B, T, H, K, V = shape
    c, do, dlast = make(shape, BF16, ragged=True, state0=True)
    plan = plan_of(shape, BF16)
    wide = {n: torch.full((P, B, T + 2, H, D + 5), 3.0, dtype=BF16, device="cuda") for n, D in (("o", V), ("dq", K), ("dk", K), ("dv", V))}
    inner = {n: x[:, :, 1:-1, :, 2:-3] for n, x in wide.items()}
    cfg, io, keys, values = plan._io(c["q"], c["k"], c["v"], c["log_decay"], c["state0"], None, c["lengths"])
    io.o = plan._heads(inner["o"], "o", values)
    ws, n = plan._workspace("pop_linear_forward_workspace_bytes", cfg)
    plan._call(plan.lib.pop_linear_forward, ct.byref(cfg), ct.byref(io), ws.data_ptr(), n)
    grads = ops.pop_linear_grads(plan._heads(do, "do", values), *(plan._heads(inner[n], n, s) for n, s in (("dq", keys), ("dk", keys), ("dv", values))))
    ws, n = plan._workspace("pop_linear_backward_workspace_bytes", cfg)
    plan._call(plan.lib.pop_linear_backward, ct.byref(cfg), ct.byref(io), ct.byref(grads), ws.data_ptr(), n)
    assert torch.equal(inner["o"], plan.forward(**c)[0])
    for x, want in zip((inner["dq"], inner["dk"], inner["dv"]), plan.backward(do=do, **c)):
        assert torch.equal(x, want)
    for n, x in wide.items():
        inner[n].fill_(3.0)
        assert (x == 3.0).all(), n


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("P, B, H, K, V", [(1, 1, 1, 1, 1), (3, 5, 2, 16, 8), (2, 3, 3, 33, 65), (1, 2, 1, 128, 128), (2, 2, 4, 64, 64), (1, 1, 2, 7, 100)])
def test_step(P, B, H, K, V, dtype):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(K)
    draw = lambda *s: torch.randn(s, generator=gen, device="cuda")
    q, k, v = draw(P, B, H, K).to(dtype), draw(P, B, 2 * H, K).to(dtype)[:, :, H:], draw(P, B, H, V + 3).to(dtype)[..., 3:]
    log = -torch.rand((P, H), generator=gen, device="cuda")
    for slots in (None, torch.stack([torch.randperm(B + 2, generator=gen, device="cuda")[:B] for _ in range(P)]).to(torch.int32)):
        state = draw(P, B + 2, H, K, V)
        reset = torch.rand((P, B), generator=gen, device="cuda") < 0.4
        if slots is not None:
            slots[0, 0] = -1
            slots[-1, -1] = B + 2
        want, ws, E, Es = L.step(*(numpy_of(x) for x in (q, k, v, state, log, reset)), None if slots is None else slots.cpu().numpy(), unit=UNIT,
                                 operand=OPERAND[dtype])
        o = pp.LinearAttention(P, B, 1, H, K, V, dtype).step(q, k, v, state, log, reset, slots)
        check("o", o, want, E, dtype)
        check("state", state, ws, Es)


def test_idle_rows_read_nothing():
    q = torch.full((1, 2, 1, 4), float("nan"), device="cuda")
    state = torch.randn((1, 3, 1, 4, 4), device="cuda")
    kept = state.clone()
    o = pp.LinearAttention(1, 2, 1, 1, 4, 4).step(q, q, q, state, slots=torch.tensor([[-1, 3]], dtype=torch.int32, device="cuda"))
    assert not o.any() and torch.equal(state, kept)


def test_a_reset_drops_what_is_not_finite():
    q = torch.randn((1, 2, 1, 4), device="cuda")
    state = torch.full((1, 2, 1, 4, 4), float("nan"), device="cuda")
    o = pp.LinearAttention(1, 2, 1, 1, 4, 4).step(q, q, q, state, reset=torch.tensor([[True, False]], device="cuda"))
    assert torch.isfinite(o[0, 0]).all() and torch.isfinite(state[0, 0]).all() and torch.isnan(state[0, 1]).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_steps_follow_the_sequence(dtype):
    """Steps one by one end where the whole sequence does, each within its bound of the exact value."""
    shape = (2, 2, 40, 2, 24, 16)
    c, _, _ = make(shape, dtype, reset=0.1, state0=True)
    plan, state = plan_of(shape, dtype), c["state0"].clone()
    o = torch.stack([plan.step(c["q"][:, :, t], c["k"][:, :, t], c["v"][:, :, t], state, c["log_decay"], c["reset"][:, :, t]) for t in range(40)], 2)
    check_forward(shape, dtype, c, got=(o, state))


def test_shorter_sequences_than_planned():
    plan = pp.LinearAttention(2, 2, 500, 2, 16, 16)
    c, do, dlast = make((2, 2, 70, 2, 16, 16), F32, state0=True)
    check_forward((2, 2, 70, 2, 16, 16), F32, c, got=plan.forward(**c))
    check_backward((2, 2, 70, 2, 16, 16), F32, c, do, dlast, got=plan.backward(do=do, dstate_last=dlast, **c))


def test_results_repeat_bit_by_bit():
    for shape in ((4, 2, 300, 2, 64, 64), (1, 1, 5000, 1, 32, 32)):
        c, do, dlast = make(shape, BF16, reset=0.01, state0=True)
        plan = plan_of(shape, BF16)
        first = plan.forward(**c) + plan.backward(do=do, dstate_last=dlast, **c)
        for _ in range(3):
            assert all(torch.equal(a, b) for a, b in zip(first, plan.forward(**c) + plan.backward(do=do, dstate_last=dlast, **c)))


def test_states_carried_on_through_pieces():
    """A sequence in pieces, state_last handed on as state0: as in one."""
    shape = (1, 2, 400, 2, 32, 48)
    c, _, _ = make(shape, F32, reset=0.01, state0=True)
    plan, state, outs = plan_of(shape, F32), c["state0"], []
    for lo, hi in ((0, 1), (1, 100), (100, 164), (164, 400)):
        o, state = plan.forward(c["q"][:, :, lo:hi], c["k"][:, :, lo:hi], c["v"][:, :, lo:hi], c["log_decay"], state, c["reset"][:, :, lo:hi])
        outs.append(o)
    check_forward(shape, F32, c, got=(torch.cat(outs, 2), state))


def test_last_states_over_first_ones():
    """Through the boundary: state_last may be state0."""
    import ctypes as ct
    for shape in ((2, 2, 200, 2, 16, 16), (1, 1, 6000, 1, 32, 32)):
        c, _, _ = make(shape, F32, state0=True)
        plan = plan_of(shape, F32)
        want = plan.forward(**c)
        cfg, io, _, values = plan._io(*(c[n] for n in ("q", "k", "v", "log_decay", "state0", "reset", "lengths")))
        o, state = torch.empty(values, device="cuda"), c["state0"].clone()
        io.o, io.state0, io.state_last = plan._heads(o, "o", values), state.data_ptr(), state.data_ptr()
        ws, n = plan._workspace("pop_linear_forward_workspace_bytes", cfg)
        plan._call(plan.lib.pop_linear_forward, ct.byref(cfg), ct.byref(io), ws.data_ptr(), n)
        assert torch.equal(o, want[0]) and torch.equal(state, want[1])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("K, V", [(7, 9), (8, 16), (9, 100), (66, 30), (127, 65), (128, 24)])
@pytest.mark.parametrize("layout", ["packed", "time_major"])
def test_widths_and_segments(K, V, layout, dtype):
    """Every width of kernel, rows that are not whole vectors, a few sequences in segments."""
    shape = (1, 2, 700, 2, K, V)
    c, do, dlast = make(shape, dtype, seed=K, layout=layout, reset=0.004, ragged=True, state0=True, decay=(0.001, 0.1))
    check_forward(shape, dtype, c)
    check_backward(shape, dtype, c, do, dlast)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("far", ["step", "over"])
def test_steps_far_apart_and_over_each_other(far, dtype):
    """Steps further apart than offsets of 32 bits reach (half of the memory untouched), and one step that all steps share."""
    shape = (1, 1, 40, 1, 16, 24)
    c, do, dlast = make(shape, dtype, state0=True)
    if far == "over":
        c["k"] = c["k"][:, :, :1].expand(c["k"].shape)
        c["v"] = c["v"][:, :, 3:4].expand(c["v"].shape)
    else:
        size = (1 << 31) // c["q"].element_size() // 40
        wide = torch.empty((1, 1, 40, size), dtype=dtype, device="cuda")
        wide[..., :16] = c["q"][:, :, :, 0]
        c["q"] = wide[..., :16].unflatten(-1, (1, 16))
    check_forward(shape, dtype, c)
    check_backward(shape, dtype, c, do, dlast)


@pytest.mark.parametrize("dtype", TYPES)
def test_not_finite_in_segments(dtype):
    """Long sequences in segments: what is not finite in one of them reaches those that follow until an episode starts."""
    shape = (1, 2, 3000, 1, 16, 20)
    c, do, dlast = make(shape, dtype, seed=9, decay=(0.0005, 0.01), state0=True)
    c["reset"] = torch.zeros((1, 2, 3000), dtype=torch.bool, device="cuda")
    c["reset"][0, 0, 2000] = c["reset"][0, 1, 700] = True
    c["k"][0, 0, 500, 0, 3] = float("inf")
    c["v"][0, 1, 1500, 0, 7] = float("nan")
    do[0, 0, 2500, 0, 2] = float("nan")
    check_forward(shape, dtype, c)
    check_backward(shape, dtype, c, do, dlast)


@pytest.mark.parametrize("shape", [(2, 2, 150, 2, 32, 32), (1, 1, 5000, 1, 32, 32)])
def test_captured_and_replayed(shape):
    """A graph of forward, backward and a step, replayed with eager work between; each replay against the eager result."""
    c, do, dlast = make(shape, BF16, reset=0.02, state0=True)
    plan, state = plan_of(shape, BF16), torch.zeros_like(c["state0"])
    one = lambda: plan.step(c["q"][:, :, 0], c["k"][:, :, 0], c["v"][:, :, 0], state, c["log_decay"])
    whole = lambda: plan.forward(**c) + plan.backward(do=do, dstate_last=dlast, **c)
    want = whole() + (one(),)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = whole() + (one(),)
    for k in range(3):
        state.zero_()
        for x in got:
            x.fill_(7.0)
        torch.randn((1 << 20,), device="cuda").sum()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), k
        c["q"].mul_(1.0)
        assert all(torch.equal(a, b) for a, b in zip(whole(), want))


def test_calls_on_two_streams_at_once():
    shape = (4, 2, 500, 2, 32, 32)
    calls = [(make(shape, BF16, seed=s, reset=0.02, state0=True), plan_of(shape, BF16)) for s in range(2)]
    run = lambda c, plan: plan.forward(**c[0]) + plan.backward(do=c[1], dstate_last=c[2], **c[0])
    want = [run(*x) for x in calls]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], []
    for s, x in zip(streams, calls):
        with torch.cuda.stream(s):
            got.append([run(*x) for _ in range(4)][-1])
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        assert all(torch.equal(a, b) for a, b in zip(g, w))


def test_gradients_against_differences():
    """The sum that backward differentiates, by differences of forward along random directions (quadratic: no error of differences
    but what rounding leaves)."""
    shape = (1, 2, 90, 2, 12, 16)
    c, do, dlast = make(shape, F32, reset=0.03, ragged=True, state0=True)
    plan = plan_of(shape, F32)
    grads = plan.backward(do=do, dstate_last=dlast, **c)

    def loss(**kw):
        o, last = plan.forward(**dict(c, **kw))
        return (o.double() * do.double()).sum() + (last.double() * dlast.double()).sum()

    gen = torch.Generator(device="cuda")
    gen.manual_seed(5)
    sizes = [float((o.double().abs() * d.double().abs()).sum()) for o, d in zip(plan.forward(**c), (do, dlast))]
    for name, g in zip(("q", "k", "v", "state0"), grads):
        d = torch.randn(c[name].shape, generator=gen, device="cuda")
        h = 2.0 ** -3
        got = (loss(**{name: c[name] + h * d}) - loss(**{name: c[name] - h * d})) / (2 * h)
        want = (g.double() * d.double()).sum()
        # each loss is off by its outputs' rounding: at most some 200 units of the sum of magnitudes, which moved by h d grow a few times
        assert abs(float(got - want)) <= 200 * 2.0 ** -24 * 4 * sum(sizes) / h, (name, float(got), float(want))


def test_another_device_or_host_tensors_are_refused():
    plan = pp.LinearAttention(1, 1, 4, 1, 4, 4)
    x = torch.zeros((1, 1, 4, 1, 4), device="cuda")
    with pytest.raises(ValueError, match="k must be a tensor on"):
        plan.forward(x, x.cpu(), x)
    with pytest.raises(ValueError, match="type"):
        plan.forward(x, x.half(), x)
    with pytest.raises(ValueError, match="shape"):
        plan.forward(x, x, x[..., :3])
    with pytest.raises(ValueError, match="adjacent"):
        plan.forward(x.transpose(2, 4), x, x)
    with pytest.raises(ValueError, match="up to 4"):
        plan.forward(torch.zeros((1, 1, 5, 1, 4), device="cuda"), x, x)
    with pytest.raises(ValueError, match="q requires gradients"):
        plan.forward(x.clone().requires_grad_(), x, x)
    with pytest.raises(ValueError, match="state must be"):
        plan.step(x[:, :, 0], x[:, :, 0], x[:, :, 0], torch.zeros((1, 1, 4, 4), device="cuda"))
    with pytest.raises(ValueError, match="no slots are given"):
        pp.LinearAttention(1, 2, 1, 1, 4, 4).step(*[torch.zeros((1, 2, 1, 4), device="cuda")] * 3, torch.zeros((1, 1, 1, 4, 4), device="cuda"))


def test_a_state_table_that_is_overwritten_is_seen():
    x, state = torch.randn((1, 1, 1, 4), device="cuda"), torch.randn((1, 1, 1, 4, 4), device="cuda")
    other = torch.ones_like(state, requires_grad=True)
    out = (other * state).sum()
    pp.LinearAttention(1, 1, 1, 1, 4, 4).step(x, x, x, state)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        out.backward()


@pytest.mark.parametrize("T", [1, 3])
def test_more_columns_than_a_row_of_the_grid(T):
    """Five million memories of one number each: o_t = scale q_t sum_s lambda^(t - s) k_s v_s."""
    B, H = 1 << 20, 5
    gen = torch.Generator(device="cuda")
    gen.manual_seed(2)
    q, k, v, do = (torch.randn((1, B, T, H, 1), generator=gen, device="cuda") for _ in range(4))
    log = torch.full((1, H), -0.25, device="cuda")
    plan = pp.LinearAttention(1, B, T, H, 1, 1, scale=0.5)
    o, last = plan.forward(q, k, v, log)
    dq, dk, dv, d0 = plan.backward(q, k, v, do, log)
    lam = torch.exp(torch.tensor(-0.25, dtype=torch.float64))
    Q, K, V, D = (x.double() for x in (q, k, v, do))
    S, M = torch.zeros_like(Q[:, :, 0]), torch.zeros_like(Q[:, :, 0])
    for t in range(T):
        S, M = lam * S + K[:, :, t] * V[:, :, t], lam * M + (K[:, :, t] * V[:, :, t]).abs()
        # operands to 2^-23, a dozen roundings of sums and factors
        for got, want, size in ((o, 0.5 * S * Q[:, :, t], M * Q[:, :, t].abs()), (dq, 0.5 * S * D[:, :, t], M * D[:, :, t].abs())):
            assert bool(((got[:, :, t] - want).abs() <= 32 * 2.0 ** -24 * size + 1e-37).all())
    assert bool(((last[..., 0] - S).abs() <= 32 * 2.0 ** -24 * M + 1e-37).all())
    G, N = torch.zeros_like(S), torch.zeros_like(S)
    for t in reversed(range(T)):
        G, N = lam * G + 0.5 * Q[:, :, t] * D[:, :, t], lam * N + (0.5 * Q[:, :, t] * D[:, :, t]).abs()
        for got, want, size in ((dk, G * V[:, :, t], N * V[:, :, t].abs()), (dv, G * K[:, :, t], N * K[:, :, t].abs())):
            assert bool(((got[:, :, t] - want).abs() <= 32 * 2.0 ** -24 * size + 1e-37).all())
    assert bool(((d0[..., 0] - lam * G).abs() <= 32 * 2.0 ** -24 * N + 1e-37).all())
