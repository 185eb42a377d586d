"""The precision of every kernel that multiplies, against products in 32 bits on the same inputs: error over error, at most 4.
(test_split_products.py shows on the CPU that a product without one of its small halves fails this.)"""
import numpy as np
import pytest
import torch

import paper_2206_08888_amd as pp
from gpu_common import ensure_built
from oracle import orthogonalize as O
from test_gpu_orthogonalize import F32, QUINTIC, _gradient, _muon_case, _np
from test_split_products import products32

pytestmark = pytest.mark.gpu


def _some(count):
    return sorted({0, count // 2, count - 1})


# by launch: blocks; 64 x 64 tiles for X = Q X; 128 x 64 tiles there and for triangles; 128 x 128 tiles there; then for triangles
# as well; large matrices; more rows than columns; edges inside a tile
@pytest.mark.parametrize("count, rows, cols", [(2, 256, 256), (10, 256, 256), (20, 256, 256), (40, 256, 256), (70, 256, 256), (140, 256, 256), (2, 1024, 1024),
                                               (4, 1024, 1024), (12, 1024, 1024), (1, 700, 1100), (3, 300, 1000), (20, 393, 256), (70, 256, 190),
                                               (140, 250, 131), (9, 600, 520), (40, 130, 390)])
def test_errors_are_those_of_32_bit_products(count, rows, cols):
    ensure_built()
    g = _gradient((count, rows, cols), F32, rows + cols)
    few = _some(count)
    o, u = _np(pp.Orthogonalizer(count, rows, cols)(g)[few]), _np(g[few])
    want = O.orthogonalize(u, QUINTIC, 1e-7)
    err, err32 = np.linalg.norm(o - want), np.linalg.norm(products32(u, QUINTIC) - want)
    assert err <= 4 * err32, (err, err32, np.linalg.norm(want))


@pytest.mark.parametrize("P, shapes", [(10, [(256, 256), (70, 256)]), (40, [(256, 256), (256, 70)]), (80, [(17, 256), (256, 256), (256, 6)]), (2, [(1024, 1024)])])
def test_updates_are_those_of_32_bit_products(P, shapes):
    """Updates alone: no weights, a learning rate of one."""
    ensure_built()
    _, momenta, grads, hp = _muon_case(P, shapes, F32, 41)
    weights = [torch.zeros_like(m) for m in momenta]
    hp[:, 0], hp[:, 2] = 1.0, 0.0
    few = _some(P)
    mu = _np(hp)[few, 1][:, None, None]
    moved = [mu * _np(m[few]) + _np(g[few]) for m, g in zip(momenta, grads)]
    pp.Muon(P, shapes, scales=[1.0] * len(shapes)).step(weights, momenta, grads, hp)
    for w, m, g in zip(weights, moved, grads):
        u = _np(g[few]) + mu * m
        want = -O.orthogonalize(u, QUINTIC, 1e-7)
        err, err32 = np.linalg.norm(_np(w[few]) - want), np.linalg.norm(-products32(u, QUINTIC) - want)
        assert err <= 4 * err32, (w.shape, err, err32)
