"""Newton-Schulz orthogonalisation and the Muon step on the GPU against the oracle in 64 bits, within the Frobenius
bound that the oracle derives for products of fp32's grade (plus one rounding to the output's type)."""
import numpy as np
import pytest
import torch

import paper_2206_08888_amd as pp
from gpu_common import ensure_built
from oracle import orthogonalize as O

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
QUINTIC = [pp.NS_COEF] * 5
OUT = {F32: (0.0, 0.0), BF16: (2.0 ** -9, 0.0), F16: (2.0 ** -12, 2.0 ** -25)}     # half a unit, relative and least


def _np(t):
    return t.detach().double().cpu().numpy()


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _gradient(shape, dtype, seed, batch=None):
    """Inputs times output gradients over a batch; fewer samples than rows: rank-deficient."""
    n, rows, cols = shape
    gen, batch = _gen(seed), batch or 2 * max(rows, cols)
    left = torch.relu(torch.randn((n, rows, batch), generator=gen, device="cuda"))
    right = torch.randn((n, batch, cols), generator=gen, device="cuda") * 0.01
    return torch.stack([a @ b for a, b in zip(left, right)]).to(dtype)


def _check(got, u, coef, eps, dtype):
    """got against the orthogonalised u (a device tensor)."""
    u, got, (rel, least) = _np(u), _np(got), OUT[dtype]
    want, bound = O.orthogonalize(u, coef, eps), O.rounding_bound(u, coef, eps)
    for p in range(len(u)):
        tol = bound[p] + rel * (np.linalg.norm(want[p]) + bound[p]) + least * np.sqrt(want[p].size)
        err = np.linalg.norm(got[p] - want[p])
        assert err <= tol, (p, err, tol, np.linalg.norm(want[p]))


SHAPES = [(1, 1, 1), (2, 1, 7), (3, 5, 1), (2, 6, 256), (2, 256, 6), (1, 17, 256), (2, 256, 256), (1, 33, 65), (1, 65, 33), (2, 393, 256),
          (1, 129, 200), (1, 300, 500), (1, 40, 2000), (1, 700, 64), (40, 31, 32)]


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("shape", SHAPES)
def test_against_the_oracle(shape, dtype):
    ensure_built()
    g = _gradient(shape, dtype, sum(shape))
    before = g.clone()
    plan = pp.Orthogonalizer(*shape, dtype)
    o = plan(g)
    assert torch.equal(g, before) and o.dtype == dtype
    _check(o, g, QUINTIC, 1e-7, dtype)
    assert torch.equal(plan(g), o)                       # sums in a fixed order
    assert plan(g, out=g) is g and torch.equal(g, o)     # in place


@pytest.mark.parametrize("shape", [(2, 256, 256), (1, 256, 1000), (1, 393, 256), (4, 17, 256)])
def test_errors_are_those_of_32_bit_products(shape):
    """The bound above is a worst case; over ordinary gradients the error is that of fp32 products, within a factor 4."""
    ensure_built()
    g = _gradient(shape, F32, 12)
    want, x = O.orthogonalize(_np(g), QUINTIC, 1e-7), g.cpu()
    if shape[1] > shape[2]:
        x = x.transpose(1, 2)
    x = x / (x.square().sum((1, 2), keepdim=True).sqrt() + 1e-7)
    for k0, k1, k2 in QUINTIC:
        a = x @ x.transpose(1, 2)
        x = k0 * x + (k1 * a + k2 * (a @ a)) @ x
    if shape[1] > shape[2]:
        x = x.transpose(1, 2)
    err32, err = np.linalg.norm(_np(x) - want), np.linalg.norm(_np(pp.Orthogonalizer(*shape)(g)) - want)
    assert err <= 4 * err32, (err, err32)


@pytest.mark.parametrize("shape", [(1, 600, 900), (1, 1024, 1024), (2, 1100, 520)])
def test_large(shape):
    ensure_built()
    g = _gradient(shape, F32, 1)
    _check(pp.Orthogonalizer(*shape)(g), g, QUINTIC, 1e-7, F32)


@pytest.mark.parametrize("shape", [(2, 20, 50), (2, 130, 60)])
def test_strides(shape):
    """Rows with gaps and at odd offsets, agents at odd distances; what lies between them stays."""
    ensure_built()
    n, r, c = shape
    wide = torch.full((n, r + 1, c + 3), float("nan"), device="cuda")
    flat = torch.full((n * (r * c + 7),), float("nan"), device="cuda")
    g, out = wide[:, 1:, 3:], flat.as_strided((n, r, c), (r * c + 7, c, 1), 5)
    g.copy_(_gradient(shape, F32, 2))
    o = pp.Orthogonalizer(*shape)(g, out=out)
    _check(o, g, QUINTIC, 1e-7, F32)
    assert int(flat.isnan().sum()) == 7 * n
    same = g[:1].expand(shape)                           # broadcast input
    want = pp.Orthogonalizer(1, r, c)(g[:1].contiguous())
    assert torch.equal(pp.Orthogonalizer(*shape)(same), want.expand(shape))


@pytest.mark.parametrize("coef, steps", [(QUINTIC, 0), (pp.NS_COEF, 1), ((1.5, -0.5, 0.0), 16), ((1.875, -1.25, 0.375), 8),
                                         ([(4.0, -6.0, 2.5), (3.0, -3.2, 1.2), (1.875, -1.25, 0.375)], 3), ((0.0, 1.0, 0.0), 2), ((-1.5, 0.5, 0.0), 3),
                                         ((0.01, 0.0, 0.0), 2)])
def test_coefficients(coef, steps):
    ensure_built()
    each = ([] if steps == 0 else [coef] * steps if not hasattr(coef[0], "__len__") else coef)
    for shape in ((2, 60, 90), (1, 100, 30)):
        g = _gradient(shape, F32, 4)
        _check(pp.Orthogonalizer(*shape, steps=steps, coef=each if steps else pp.NS_COEF)(g), g, each, 1e-7, F32)


@pytest.mark.parametrize("scale", [1e-30, 1e-8, 1e-3, 1e6, 1e30])
def test_magnitudes(scale):
    ensure_built()
    g = _gradient((2, 50, 70), F32, 5) * scale
    _check(pp.Orthogonalizer(2, 50, 70)(g), g, QUINTIC, 1e-7, F32)
    _check(pp.Orthogonalizer(2, 50, 70, eps=1e-30)(g), g, QUINTIC, float(np.float32(1e-30)), F32)


def test_uneven_and_deficient_matrices():
    """Rank 8 of 96, singular values over six decades, one row that dwarfs the others, zeros."""
    ensure_built()
    low = _gradient((1, 96, 128), F32, 6, batch=8)[0]
    gen = _gen(7)
    q = torch.linalg.qr(torch.randn((128, 96), generator=gen, device="cuda"))[0].t()
    decades = torch.diag(torch.logspace(0, -6, 96, device="cuda")) @ q
    tall = _gradient((1, 96, 128), F32, 8)[0]
    tall[5] *= 1e5
    g = torch.stack([low, decades, tall, torch.zeros_like(low)])
    o = pp.Orthogonalizer(4, 96, 128)(g)
    _check(o, g, QUINTIC, 1e-7, F32)
    assert not o[3].any()


def test_one_spoiled_matrix_does_not_spoil_the_others():
    ensure_built()
    g = _gradient((3, 40, 50), F32, 9)
    want = pp.Orthogonalizer(3, 40, 50)(g)
    for bad in (float("nan"), float("inf")):
        h = g.clone()
        h[1, 3, 4] = bad
        o = pp.Orthogonalizer(3, 40, 50)(h)
        assert torch.equal(o[0], want[0]) and torch.equal(o[2], want[2]) and bool(o[1].isnan().all())


def _muon_case(P, shapes, dtype, seed):
    gen = _gen(seed)
    grads = [_gradient((P, r, c), dtype, seed + i) for i, (r, c) in enumerate(shapes)]
    weights = [torch.randn((P, r, c), generator=gen, device="cuda") * 0.1 for r, c in shapes]
    momenta = [torch.randn((P, r, c), generator=gen, device="cuda") * 0.01 for r, c in shapes]
    hp = torch.stack([torch.rand(P, generator=gen, device="cuda") * 0.05, 0.8 + 0.19 * torch.rand(P, generator=gen, device="cuda"),
                      torch.rand(P, generator=gen, device="cuda") * 0.1], 1).contiguous()
    return weights, momenta, grads, hp


def _check_muon(plan, weights, momenta, grads, hp, nesterov, scales):
    old = [(_np(w), _np(m), _np(g)) for w, m, g in zip(weights, momenta, grads)]
    plan.step(weights, momenta, grads, hp)
    lr, mu, wd = _np(hp).T
    for (w, m, g), nw, nm, scale in zip(old, weights, momenta, scales):
        ww, wm = O.muon(w, m, g, lr, mu, wd, scale, QUINTIC, 1e-7, nesterov)
        u = g + mu[:, None, None] * wm if nesterov else wm
        bound = O.rounding_bound(u, QUINTIC, 1e-7)
        # mu m + g: one rounding of a fused product; U: 2^-23 of its terms, in place of the 2^-21 of its sum that the
        # bound has, where the terms cancel
        assert (np.abs(_np(nm) - wm) <= 2.0 ** -23 * (np.abs(mu[:, None, None] * m) + np.abs(g)) + 1e-37).all()
        for p in range(len(w)):
            terms = np.linalg.norm(np.abs(mu[p] * m[p]) + 2 * np.abs(g[p])) / np.linalg.norm(u[p])
            tol = lr[p] * scale * bound[p] * max(1.0, terms) + 2.0 ** -22 * np.linalg.norm(w[p])
            err = np.linalg.norm(_np(nw)[p] - ww[p])
            assert err <= tol, (p, w.shape, err, tol)


@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("P, shapes", [(3, [(17, 256), (256, 256), (256, 6)]), (2, [(23, 64)]), (1, [(1, 1), (7, 300), (300, 7), (33, 31)]),
                                       (2, [(9, 9)] * 8)])
def test_muon(P, shapes, dtype, nesterov):
    ensure_built()
    case = _muon_case(P, shapes, dtype, 3)
    plan = pp.Muon(P, shapes, dtype, nesterov=nesterov)
    _check_muon(plan, *case, nesterov, [float(np.float32(max(1.0, c / r) ** 0.5)) for r, c in shapes])
    _check_muon(plan, *case, nesterov, [float(np.float32(max(1.0, c / r) ** 0.5)) for r, c in shapes])     # and the step after it


def test_muon_on_flat_networks():
    """Weights and momenta inside flat networks [P, size], agents at an odd distance; biases between them stay."""
    ensure_built()
    P, shapes = 3, [(11, 40), (40, 3)]
    size = 11 * 40 + 40 + 40 * 3 + 3
    w, m, g, hp = _muon_case(P, shapes, F32, 8)
    nets = [torch.full((P, size), 7.0, device="cuda") for _ in range(2)]
    views = [[net[:, lo:lo + r * c].unflatten(1, (r, c)) for lo, (r, c) in zip((0, 480), shapes)] for net in nets]
    for to, src in zip(views, (w, m)):
        for a, b in zip(to, src):
            a.copy_(b)
    plan = pp.Muon(P, shapes, scales=[0.5, 2.0])
    plan.step(views[0], views[1], g, hp)
    plan.step(w, m, g, hp)
    for to, src in zip(views, (w, m)):
        for a, b in zip(to, src):
            assert torch.equal(a, b)
    assert all(bool((net[:, 440:480] == 7).all()) and bool((net[:, 600:] == 7).all()) for net in nets)


def test_no_steps_is_normalised_momentum():
    ensure_built()
    w, m, g, hp = _muon_case(2, [(20, 30)], F32, 1)
    ow, om = _np(w[0]), _np(m[0])
    pp.Muon(2, [(20, 30)], steps=0, scales=[1.0]).step(w, m, g, hp)
    ww, wm = O.muon(ow, om, _np(g[0]), *_np(hp).T, 1.0, [], 1e-7, True)
    assert np.abs(_np(w[0]) - ww).max() < 1e-6 and np.abs(_np(m[0]) - wm).max() < 1e-6


def test_streams_and_graphs():
    ensure_built()
    P, shapes = 4, [(17, 64), (64, 64)]
    w, m, g, hp = _muon_case(P, shapes, F32, 2)
    plan = pp.Muon(P, shapes)
    first = [[t.clone() for t in v] for v in (w, m)]
    plan.step(w, m, g, hp)
    want = [[t.clone() for t in v] for v in (w, m)]
    side = torch.cuda.Stream()
    a, b = [[t.clone() for t in v] for v in first]
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        plan.step(a, b, g, hp)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(x, y) for x, y in zip(a + b, want[0] + want[1]))
    a, b = [[t.clone() for t in v] for v in first]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        plan.step(a, b, g, hp)
    for seed in range(3):
        _, _, ng, nhp = _muon_case(P, shapes, F32, 20 + seed)
        for x, y in zip(g + [hp], ng + [nhp]):
            x.copy_(y)
        c, d = [t.clone() for t in a], [t.clone() for t in b]
        graph.replay()
        plan.step(c, d, g, hp)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(a + b, c + d)), seed


def test_refusals():
    ensure_built()
    g = torch.zeros((2, 5, 6), device="cuda")
    plan = pp.Orthogonalizer(2, 5, 6)
    for bad in (g.double(), g[:1], g.cpu(), torch.zeros((2, 6, 5), device="cuda").transpose(1, 2)):
        with pytest.raises(ValueError):
            plan(bad)
    with pytest.raises(pp.PopError):
        plan(g, out=g[:1].expand(2, 5, 6))               # an output that overlaps itself
    for kw in (dict(coef=(1.0, 2.0)), dict(coef=[(1.5, -0.5, 0.0)] * 3), dict(dtype=torch.float64), dict(device="cpu")):
        with pytest.raises(ValueError):
            pp.Orthogonalizer(2, 5, 6, **kw)
    with pytest.raises(ValueError):
        pp.Muon(2, [(5, 6)], scales=[1.0, 2.0])
    muon = pp.Muon(2, [(5, 6)])
    with pytest.raises(ValueError):
        muon.step([g], [g.clone()], [g.clone(), g.clone()], torch.zeros((2, 3), device="cuda"))
    with pytest.raises(ValueError):
        muon.step([g], [g.clone()], [g.clone()], torch.zeros((3, 3), device="cuda"))
    with pytest.raises(pp.PopError) as e:
        muon.step([g], [g], [g.clone()], torch.zeros((2, 3), device="cuda"))
    assert e.value.code == pp.POP_EINVAL
