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
