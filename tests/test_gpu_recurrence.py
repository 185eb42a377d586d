"""The gated linear recurrence on the GPU against the oracle in 64 bits, element by element within the bound that the
oracle propagates for 32-bit arithmetic (plus one rounding to the output's type)."""
import numpy as np
import pytest
import torch

import paper_2206_08888_amd as pp
from gpu_common import ensure_built
from oracle import recurrence as R

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
# a chunk's map is a product of its gates, so a state in front of a chunk passes through as many roundings as one that
# goes step by step, in another order: twice the bound of the steps covers both
ROUNDING = 2 * 2.0 ** -24
OUT = {F32: (0.0, 0.0), BF16: (2.0 ** -8, 2.0 ** -133), F16: (2.0 ** -11, 2.0 ** -24)}   # half a unit, smallest value


def _np(t):
    return None if t is None else t.detach().double().cpu().numpy()


def _check(name, got, want, bound, dtype=F32):
    got, (rel, least) = _np(got), OUT[dtype]
    tol = bound * (1 + rel) + rel * np.abs(want) + least + 1e-37
    same = np.isnan(got) & np.isnan(want) | (got == want)
    bad = ~(same | (np.abs(got - want) <= tol))
    assert not bad.any(), (name, int(bad.sum()), bad.size, np.argwhere(bad)[:3].tolist(), got[bad][:3], want[bad][:3], tol[bad][:3])


def _tensor(shape, dtype, gen, layout="plain", scale=1.0):
    """[P, B, T, C] in one of several memory layouts; what lies between the elements is NaN."""
    P, B, T, C = shape
    v = (torch.randn(shape, generator=gen, device="cuda") * scale).to(dtype)
    if layout == "plain":
        return v
    if layout == "time_major":
        return v.permute(2, 0, 1, 3).contiguous().permute(1, 2, 0, 3)
    if layout == "packed":                               # the second part of a wider row, at an odd offset
        wide = torch.full((P, B, T, 2 * C + 3), float("nan"), dtype=dtype, device="cuda")
        wide[..., C + 3:] = v
        return wide[..., C + 3:]
    if layout == "gaps":                                 # rows of whole 16 bytes with gaps between them
        wide = torch.full((P, B, T + 2, (C + 15) // 8 * 8), float("nan"), dtype=dtype, device="cuda")
        wide[:, :, 1:T + 1, :C] = v
        return wide[:, :, 1:T + 1, :C]
    assert layout == "broadcast"
    return v[:, :1].expand(shape)


def _case(P, B, T, C, dtype=F32, seed=0, layout="plain", bias=True, h0=True, reset=True, lengths=True, spread=4.0):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    kw = dict(x=_tensor((P, B, T, C), dtype, gen, layout), g=_tensor((P, B, T, C), dtype, gen, layout, 1.5),
              bias=torch.rand((P, C), generator=gen, device="cuda") * spread if bias else None,
              h0=torch.randn((P, B, C), generator=gen, device="cuda") if h0 else None, reset=None, lengths=None)
    if reset:
        r = (torch.rand((P, B, T), generator=gen, device="cuda") < 0.05).to(torch.uint8) * 3
        kw["reset"] = r.permute(2, 0, 1).contiguous().permute(1, 2, 0) if layout == "time_major" else r
    if lengths:
        n = torch.randint(0, T + 1, (P, B), generator=gen, device="cuda", dtype=torch.int32)
        flat = n.view(-1)
        for i, v in enumerate((T, 0, 1, -3, T + 9)[:flat.numel()]):
            flat[-1 - i] = v
        kw["lengths"] = n
    return kw, _tensor((P, B, T, C), dtype, gen, layout, 0.5), torch.randn((P, B, C), generator=gen, device="cuda")


def _verify(kw, dy, dh, plan=None):
    P, B, T, C = kw["x"].shape
    dtype = kw["x"].dtype
    plan = plan or pp.Recurrence(P, B, T, C, dtype)
    host = {k: _np(v) for k, v in kw.items()}
    if host["lengths"] is not None:
        host["lengths"] = host["lengths"].astype(np.int64)
    y, h_last, states = plan.forward(save=True, **kw)
    y2, h2 = plan.forward(**kw)
    wy, wh, E, _ = R.forward(rounding=ROUNDING, **host)
    _check("y", y, wy, E["y"], dtype)
    _check("h_last", h_last, wh, E["h_last"])
    assert torch.equal(y.nan_to_num(7), y2.nan_to_num(7)) and torch.equal(h_last.nan_to_num(7), h2.nan_to_num(7))
    back = {k: v for k, v in kw.items() if k != "h0"}
    got = dict(zip(("dx", "dg", "dbias", "dh0"), plan.backward(states, dy=dy, dh_last=dh, **back)))
    want, E = R.backward(dy=_np(dy), dh_last=_np(dh), rounding=ROUNDING, **host)
    for name in got:
        _check(name, got[name], want[name], E[name], dtype if name in ("dx", "dg") else F32)
    again = plan.backward(states, dy=dy, dh_last=dh, **back)
    for name, v in zip(got, again):
        assert torch.equal(got[name].nan_to_num(7), v.nan_to_num(7)), name        # every sum in a fixed order
    return got


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("shape", [(1, 1, 1, 1), (2, 3, 1, 5), (1, 2, 2, 64), (2, 2, 127, 7), (1, 3, 128, 130), (3, 1, 129, 65),
                                   (1, 1, 1000, 33), (2, 2, 300, 256), (5, 7, 40, 129), (1, 1, 4099, 8), (80, 9, 20, 72)])
def test_against_the_oracle(shape, dtype):
    ensure_built()
    _verify(*_case(*shape, dtype=dtype, seed=sum(shape)))


@pytest.mark.parametrize("layout", ["time_major", "packed", "gaps", "broadcast"])
@pytest.mark.parametrize("shape", [(2, 3, 140, 64), (1, 2, 33, 30)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_layouts(layout, shape, dtype):
    ensure_built()
    _verify(*_case(*shape, dtype=dtype, seed=3, layout=layout))


@pytest.mark.parametrize("which", range(16))
def test_optional_arguments(which):
    ensure_built()
    kw, dy, dh = _case(2, 2, 150, 40, seed=which, bias=bool(which & 1), h0=bool(which & 2), reset=bool(which & 4), lengths=bool(which & 8))
    _verify(kw, dy, dh if which & 2 else None)


@pytest.mark.parametrize("T", [1, 200, 2000])
def test_long_memories(T):
    """Gates within 1e-4 of one: states and gradients carry over every chunk."""
    ensure_built()
    kw, dy, dh = _case(2, 1, T, 64, seed=T, reset=False, lengths=False)
    kw["bias"] = kw["bias"] + 8
    _verify(kw, dy, dh)


def test_no_steps():
    ensure_built()
    kw, dy, dh = _case(2, 3, 0, 5, reset=False, lengths=False)
    plan = pp.Recurrence(2, 3, 10, 5)
    y, h, states = plan.forward(save=True, **kw)
    assert y.shape == (2, 3, 0, 5) and torch.equal(h, kw["h0"])
    back = {k: v for k, v in kw.items() if k != "h0"}
    dx, dg, dbias, dh0 = plan.backward(states, dy=dy, dh_last=dh, **back)
    assert dx.numel() == dg.numel() == 0 and torch.equal(dh0, dh) and not dbias.any()
    assert not plan.forward(**dict(kw, h0=None))[1].any()


@pytest.mark.parametrize("dtype", [F32, F16])
@pytest.mark.parametrize("T", [100, 700])
def test_what_masks_hide_does_not_show(T, dtype):
    """Steps behind a sequence's end and states in front of a reset hold NaN and infinities."""
    ensure_built()
    kw, dy, dh = _case(2, 3, T, 40, dtype=dtype, seed=9)
    for p in range(2):
        for b in range(3):
            n = min(max(int(kw["lengths"][p, b]), 0), T)
            for v, junk in ((kw["x"], float("nan")), (kw["g"], float("inf")), (dy, float("nan"))):
                v[p, b, n:] = junk
            kw["reset"][p, b, n:] = 1
    kw["h0"][1, 2] = float("nan")
    kw["lengths"][1, 2], kw["reset"][1, 2, 0] = T, 1
    kw["x"][1, 2] = kw["x"][0, 0, :1]
    kw["g"][1, 2] = 0
    dy[1, 2] = 0.5
    got = _verify(kw, dy, dh)
    assert all(bool(torch.isfinite(v).all()) for v in got.values())


def test_special_values_where_nothing_hides_them():
    """Saturated gates and non-finite inputs give what the formula gives, in every later step and chunk."""
    ensure_built()
    kw, dy, dh = _case(1, 1, 400, 8, seed=5, reset=False, lengths=False, bias=False)
    kw["g"][..., 0] = float("inf")                       # keeps h0
    kw["g"][..., 1] = float("-inf")                      # y = x
    kw["x"][0, 0, 10, 2] = float("nan")
    kw["x"][0, 0, 10, 3] = float("inf")
    kw["g"][0, 0, 130, 4] = float("nan")
    kw["g"][..., 5] = -30000.0
    kw["g"][..., 6] = 30000.0
    y, h = pp.Recurrence(1, 1, 400, 8).forward(**kw)
    y = y[0, 0].cpu()
    assert torch.equal(y[:, 0], kw["h0"].cpu()[0, 0, 0].expand(400)) and torch.equal(y[:, 6], kw["h0"].cpu()[0, 0, 6].expand(400))
    assert torch.equal(y[:, 1], kw["x"].cpu()[0, 0, :, 1]) and torch.equal(y[:, 5], kw["x"].cpu()[0, 0, :, 5])
    assert not y[:10, 2].isnan().any() and y[10:, 2].isnan().all()
    assert y[10:, 3].isinf().sum() > 1 and not y[10:, 3].isfinite().any()
    assert not y[:130, 4].isnan().any() and y[130:, 4].isnan().all()
    assert bool(y[:, 7].isfinite().all()) and bool(h[0, 0, 2].isnan())


def test_a_sequence_in_pieces():
    """States carried from call to call, h_last written over h0, give the sequence in one."""
    ensure_built()
    kw, _, _ = _case(2, 2, 500, 72, seed=21, lengths=False)
    plan = pp.Recurrence(2, 2, 500, 72)
    want, last = plan.forward(**kw)
    h, parts = kw["h0"], []
    for lo, hi in ((0, 1), (1, 130), (130, 130), (130, 500)):
        y, h = plan.forward(kw["x"][:, :, lo:hi], kw["g"][:, :, lo:hi], bias=kw["bias"], h0=h, reset=kw["reset"][:, :, lo:hi].contiguous())
        parts.append(y)
    torch.testing.assert_close(torch.cat(parts, 2), want, rtol=1e-4, atol=1e-5)
    torch.testing.assert_close(h, last, rtol=1e-4, atol=1e-5)


@pytest.mark.parametrize("T", [50, 900])
def test_last_state_over_the_first(T):
    ensure_built()
    import ctypes as C
    from paper_2206_08888_amd import operators as ops
    kw, _, _ = _case(2, 3, T, 40, seed=4)
    plan = pp.Recurrence(2, 3, T, 40)
    y, want = plan.forward(**kw)
    cfg, io, shape = plan._io(kw["x"], kw["g"], kw["bias"], kw["h0"], kw["reset"], kw["lengths"])
    again = torch.empty_like(y)
    io.y, io.h_last = plan._sequence(again, "y", shape), kw["h0"].data_ptr()
    ws, n = plan._workspace(cfg)
    plan._call(plan.lib.pop_recurrence_forward, C.byref(cfg), C.byref(io), ws.data_ptr(), n)
    assert torch.equal(kw["h0"], want) and torch.equal(again, y)


def test_offsets_beyond_32_bits():
    """Two rows of a buffer, more than 2^31 elements apart, and steps far apart within them."""
    ensure_built()
    C, T, far = 64, 3, (1 << 31) + 64
    flat = torch.empty(far + (1 << 30) * (T - 1) + 4 * C, dtype=BF16, device="cuda")
    view = lambda off: flat.as_strided((1, 2, T, C), (0, far, 1 << 30, 1), off)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    x, g = view(0), view(C)
    x.copy_(torch.randn((1, 2, T, C), generator=gen, device="cuda"))
    g.copy_(torch.randn((1, 2, T, C), generator=gen, device="cuda"))
    dy = torch.randn((1, 2, T, C), generator=gen, device="cuda").to(BF16)
    _verify(dict(x=x, g=g, bias=None, h0=None, reset=None, lengths=None), dy, None)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("P, B, C, slots, layout", [(1, 1, 1, None, 0), (3, 5, 40, None, 0), (2, 7, 129, 11, 0), (10, 1, 256, None, 1), (4, 6, 64, 6, 1),
                                                    (2, 300, 8, 400, 0)])
def test_single_steps(P, B, C, slots, layout, dtype):
    ensure_built()
    gen = torch.Generator(device="cuda")
    gen.manual_seed(P + B + C)
    rows = slots or B + 2
    x, g = (_tensor((P, B, 1, C), dtype, gen, "packed" if layout else "plain")[:, :, 0] for _ in range(2))
    bias, state = torch.rand((P, C), generator=gen, device="cuda") * 3, torch.randn((P, rows, C), generator=gen, device="cuda")
    reset = torch.rand((P, B), generator=gen, device="cuda") < 0.3
    which = None
    if slots:
        which = torch.stack([torch.randperm(rows, generator=gen, device="cuda")[:B] for _ in range(P)]).to(torch.int32)
        which[0, 0], which[-1, -1], which[0, 1] = -1, rows, 2147483647
        idle = (which < 0) | (which >= rows)
        x, g = x.clone(), g.clone()
        x[idle], g[idle] = float("nan"), float("nan")    # idle rows are not read
    before = state.clone()
    y = pp.Recurrence(P, B, 4, C, dtype).step(x, g, state, bias=bias, reset=reset, slots=which)
    wy, ws, Ey, Es = R.step(_np(x), _np(g), _np(before), _np(bias), _np(reset), _np(which), rounding=ROUNDING)
    _check("y", y, wy, Ey, dtype)
    _check("state", state, ws, Es)


def test_steps_follow_the_sequence():
    """Token by token as acting does, against one call over the sequence."""
    ensure_built()
    kw, _, _ = _case(3, 4, 60, 96, seed=8, lengths=False)
    plan = pp.Recurrence(3, 4, 60, 96)
    want, last = plan.forward(**kw)
    state = kw["h0"].clone()
    for t in range(60):
        y = plan.step(kw["x"][:, :, t], kw["g"][:, :, t], state, bias=kw["bias"], reset=kw["reset"][:, :, t])
        torch.testing.assert_close(y, want[:, :, t], rtol=1e-4, atol=1e-5)
    torch.testing.assert_close(state, last, rtol=1e-4, atol=1e-5)


def test_gradients_match_differences():
    """The kernels' gradients against differences of the kernels' own forward pass, along random directions."""
    ensure_built()
    kw, dy, dh = _case(2, 2, 300, 32, seed=6)
    plan = pp.Recurrence(2, 2, 300, 32)
    y, h, states = plan.forward(save=True, **kw)
    back = {k: v for k, v in kw.items() if k != "h0"}
    dx, dg, dbias, dh0 = plan.backward(states, dy=dy, dh_last=dh, **back)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(2)
    for name, grad in (("x", dx), ("g", dg), ("bias", dbias), ("h0", dh0)):
        v = torch.randn(grad.shape, generator=gen, device="cuda")
        eps = 1e-2

        def loss(sign):
            yy, hh = plan.forward(**dict(kw, **{name: kw[name] + sign * eps * v}))
            return float((yy.double() * dy).sum() + (hh.double() * dh).sum())

        slope, want = (loss(1) - loss(-1)) / (2 * eps), float((grad.double() * v).sum())
        # curvature: third derivatives times eps^2 / 6 of some 40,000 random terms; rounding: 1e-6 of them / eps
        assert abs(slope - want) < 1e-3 * float((grad.double() * v).norm()) + 2e-2 * abs(want), (name, slope, want)


def test_streams_and_graphs():
    """On a side stream, and captured: replays on new inputs equal eager calls."""
    ensure_built()
    kw, dy, dh = _case(2, 2, 700, 64, seed=13)
    plan = pp.Recurrence(2, 2, 700, 64)
    back = {k: v for k, v in kw.items() if k != "h0"}

    def both():
        y, h, states = plan.forward(save=True, **kw)
        return (y, h) + tuple(plan.backward(states, dy=dy, dh_last=dh, **back))

    want = both()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = both()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = both()
    for seed in range(3):
        new, ndy, ndh = _case(2, 2, 700, 64, seed=30 + seed)
        for k in kw:
            kw[k].copy_(new[k])
        dy.copy_(ndy)
        dh.copy_(ndh)
        graph.replay()
        torch.cuda.synchronize()
        for v, w in zip(out, both()):
            assert torch.equal(v, w), seed


def test_refusals():
    ensure_built()
    plan = pp.Recurrence(2, 3, 10, 4)
    x = torch.zeros((2, 3, 10, 4), device="cuda")
    for bad in (dict(x=x.double()), dict(x=x[:1]), dict(x=torch.zeros((2, 3, 11, 4), device="cuda")), dict(g=x.cpu()),
                dict(g=x[:, :, :9]), dict(x=x.transpose(2, 3).contiguous().transpose(2, 3)), dict(bias=torch.zeros(4, device="cuda")),
                dict(bias=torch.zeros((2, 4), dtype=BF16, device="cuda")), dict(h0=torch.zeros((2, 3, 4))), dict(h0=x[:, :, 0].expand(2, 3, 4)),
                dict(reset=torch.zeros((2, 3, 10), device="cuda")), dict(reset=torch.zeros((2, 3), dtype=torch.uint8, device="cuda")),
                dict(lengths=torch.zeros((2, 3), dtype=torch.int64, device="cuda"))):
        with pytest.raises(ValueError):
            plan.forward(**dict(dict(x=x, g=x.clone()), **bad))
    with pytest.raises(ValueError):
        plan.step(x[:, :, 0], x[:, :, 1], torch.zeros((2, 2, 4), device="cuda"))       # fewer states than rows
    with pytest.raises(ValueError):
        plan.backward(torch.zeros(5, device="cuda"), x, x, x)
    for bad in (dict(dtype=torch.float64), dict(device="cpu")):
        with pytest.raises(ValueError):
            pp.Recurrence(2, 3, 10, 4, **bad)
    with pytest.raises(pp.PopError) as e:
        pp.Recurrence(0, 3, 10, 4)
    assert e.value.code == pp.POP_EINVAL
