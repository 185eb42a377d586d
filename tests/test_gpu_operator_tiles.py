"""Recurrence and orthogonalised updates on the GPU where a call's sizes take other tiles: many sequences of several
chunks, many matrices at once, large matrices, and matrices of up to 64 rows in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2206_08888_amd as pp
from gpu_common import ensure_built
from oracle import orthogonalize as O
from test_gpu_orthogonalize import BF16, F16, F32, QUINTIC, _check, _check_muon, _gen, _gradient, _muon_case, _np
from test_gpu_recurrence import _case, _verify

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shape", [(40, 13, 300, 64), (60, 9, 257, 7), (4, 40, 129, 256), (30, 20, 513, 6)])
def test_recurrence_over_many_sequences(shape, dtype):
    ensure_built()
    _verify(*_case(*shape, dtype=dtype, seed=sum(shape)))


# sequences whose tiles are handed from workgroup to workgroup: 64 groups of 64 columns or more in fp32, 128 in 16 bits,
# up to 256, and in fp32 beyond them from eight tiles on
CHAINS = [(10, 7, 300, 65, F32), (16, 5, 700, 64, F32), (8, 33, 1100, 64, F32), (9, 15, 400, 64, BF16), (133, 2, 260, 33, F16),
          (4, 4, 3500, 256, F32), (250, 1, 129, 33, F32)]


@pytest.mark.parametrize("P, B, T, C, dtype", CHAINS)
def test_recurrence_chains(P, B, T, C, dtype):
    ensure_built()
    _verify(*_case(P, B, T, C, dtype=dtype, seed=P))


@pytest.mark.parametrize("P, B, T, C, dtype", [CHAINS[0], CHAINS[1], CHAINS[3]])
def test_what_masks_hide_does_not_show_in_chains(P, B, T, C, dtype):
    ensure_built()
    kw, dy, dh = _case(P, B, T, C, dtype=dtype, seed=9)
    kw["lengths"][1, 2], kw["reset"][1, 2, 0] = T, 1
    kw["h0"][1, 2] = float("nan")                        # in front of a reset
    behind = torch.arange(T, device="cuda")[None, None] >= kw["lengths"].clamp(0, T)[..., None]
    kw["x"][behind], kw["g"][behind], dy[behind] = float("nan"), float("inf"), float("nan")
    kw["reset"][behind] = 1
    got = _verify(kw, dy, dh)
    assert all(bool(torch.isfinite(v).all()) for v in got.values())


@pytest.mark.parametrize("P, B, T, C, dtype", [CHAINS[0], CHAINS[3]])
def test_chains_on_streams_and_in_graphs(P, B, T, C, dtype):
    ensure_built()
    kw, dy, dh = _case(P, B, T, C, dtype=dtype, seed=10)
    plan, back = pp.Recurrence(P, B, T, C, dtype), {k: v for k, v in kw.items() if k != "h0"}

    def both():
        y, h, states = plan.forward(save=True, **kw)
        return (y, h) + plan.backward(states, dy=dy, dh_last=dh, **back)

    want, side = both(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = both()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = both()
    for seed in range(3):
        new, ndy, _ = _case(P, B, T, C, dtype=dtype, seed=20 + seed)
        for name in ("x", "g", "bias", "h0", "reset", "lengths"):
            kw[name].copy_(new[name])
        dy.copy_(ndy)
        graph.replay()
        want = both()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)), seed


@pytest.mark.parametrize("count, rows, cols, dtype", [(40, 256, 256, F32), (70, 256, 200, F32), (33, 130, 256, F32), (9, 512, 600, F32),
                                                      (70, 140, 256, BF16), (20, 200, 500, F16), (4, 300, 1000, BF16), (1, 700, 1100, BF16),
                                                      (40, 65, 100, F32), (3, 640, 640, F32)])
def test_many_or_large_matrices(count, rows, cols, dtype):
    ensure_built()
    g = _gradient((count, rows, cols), dtype, rows)
    plan = pp.Orthogonalizer(count, rows, cols, dtype)
    o = plan(g)
    _check(o, g, QUINTIC, 1e-7, dtype)
    assert torch.equal(plan(g), o)
    one = pp.Orthogonalizer(1, rows, cols, dtype)(g[-1:])       # another tiling of the same products
    _check(one, g[-1:], QUINTIC, 1e-7, dtype)


@pytest.mark.parametrize("count, rows, cols", [(3, 3, 3), (8, 20, 20), (16, 5, 6), (4, 33, 33), (5, 64, 64), (2, 64, 2048), (3, 1000, 48)])
def test_small_matrices_are_not_further_off_than_products_in_32_bits(count, rows, cols):
    """Square matrices have singular values near zero, which the steps raise: the error is that of fp32 products or less."""
    ensure_built()
    g = _gradient((count, rows, cols), F32, 21)
    want, x = O.orthogonalize(_np(g), QUINTIC, 1e-7), g.cpu()
    if rows > cols:
        x = x.transpose(1, 2)
    x = x / (x.square().sum((1, 2), keepdim=True).sqrt() + 1e-7)
    for k0, k1, k2 in QUINTIC:
        a = x @ x.transpose(1, 2)
        x = k0 * x + (k1 * a + k2 * (a @ a)) @ x
    if rows > cols:
        x = x.transpose(1, 2)
    o = pp.Orthogonalizer(count, rows, cols)(g)
    _check(o, g, QUINTIC, 1e-7, F32)
    # all in 64 bits but for the one rounding of the result, at most half a unit in each element
    assert np.linalg.norm(_np(o) - want) <= max(np.linalg.norm(_np(x) - want), 2.0 ** -24 * np.linalg.norm(want))


@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("P, shapes, dtype", [(30, [(256, 256), (256, 70)], F32), (3, [(64, 500), (40, 40), (2000, 33)], BF16),
                                              (70, [(200, 256)], BF16), (2, [(600, 700), (8, 600)], F32)])
def test_muon_steps_of_many_agents(P, shapes, dtype, nesterov):
    ensure_built()
    scales = [float(np.float32(max(1.0, r / c) ** 0.5)) for r, c in shapes]
    plan = pp.Muon(P, shapes, dtype=dtype, scales=scales, nesterov=nesterov)
    _check_muon(plan, *_muon_case(P, shapes, dtype, 31), nesterov, scales)


@pytest.mark.parametrize("count, rows, cols, dtype", [(100, 256, 256, F32), (30, 512, 400, F32), (34, 400, 640, BF16), (150, 200, 256, F16)])
def test_halves_and_whole_tiles_of_triangles(count, rows, cols, dtype):
    """From 128 to 400 tiles, and beyond: a matrix's result goes by its tiling alone within rounding."""
    ensure_built()
    g = _gradient((count, rows, cols), dtype, 5)
    o = pp.Orthogonalizer(count, rows, cols, dtype)(g)
    for p in (0, count // 2, count - 1):
        _check(o[p:p + 1], g[p:p + 1], QUINTIC, 1e-7, dtype)
    few = pp.Orthogonalizer(2, rows, cols, dtype)(g[:2])
    _check(few, g[:2], QUINTIC, 1e-7, dtype)
    assert bool(torch.isfinite(o).all())
