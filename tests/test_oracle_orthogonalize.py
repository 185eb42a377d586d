"""The oracle of the orthogonalised update: singular values against products, what the steps do to singular values, the
rounding bound against 32-bit products, the Muon step against its formula."""
import numpy as np
import pytest

from oracle import orthogonalize as O

QUINTIC = [(3.4445, -4.7750, 2.0315)] * 5


@pytest.mark.parametrize("shape", [(2, 1, 1), (1, 6, 20), (3, 20, 6), (1, 40, 40)])
def test_singular_values_are_what_the_products_change(shape):
    u = np.random.default_rng(1).standard_normal(shape)
    assert np.allclose(O.orthogonalize(u, QUINTIC, 1e-7), O.products(u, QUINTIC, 1e-7), rtol=0, atol=1e-10)


def test_singular_values_go_to_one():
    u = np.random.default_rng(2).standard_normal((1, 64, 64))
    s = np.linalg.svd(O.orthogonalize(u, QUINTIC, 1e-7), compute_uv=False)[0]
    assert s.max() < 1.21 and np.median(s) > 0.6
    cubic = O.orthogonalize(u, [(1.5, -0.5, 0.0)] * 60, 1e-7)
    assert np.allclose(cubic[0] @ cubic[0].T, np.eye(64), atol=1e-6)


def test_zero_stays_zero():
    assert not O.orthogonalize(np.zeros((1, 4, 5)), QUINTIC, 1e-7).any()


@pytest.mark.parametrize("shape", [(1, 30, 50), (1, 64, 64), (1, 3, 300)])
def test_the_bound_holds_for_32_bit_products(shape):
    rng = np.random.default_rng(3)
    u = (rng.standard_normal(shape) @ np.diag(np.geomspace(1, 1e-4, shape[2]))).astype(np.float32)
    x = u / (np.sqrt((u ** 2).sum()) + np.float32(1e-7))
    for k0, k1, k2 in np.array(QUINTIC, np.float32):
        a = x @ x.transpose(0, 2, 1)
        x = k0 * x + (k1 * a + k2 * (a @ a)) @ x
    assert x.dtype == np.float32
    err, bound = np.linalg.norm(x - O.orthogonalize(u, QUINTIC, 1e-7)), O.rounding_bound(u, QUINTIC, 1e-7)[0]
    assert err < bound < 1e-2 * np.linalg.norm(x)        # a worst case: every error at the steepest slope


def test_muon():
    rng = np.random.default_rng(4)
    w, m, g = (rng.standard_normal((2, 3, 5)) for _ in range(3))
    lr, mu, wd = [0.1, 0.2], [0.9, 0.5], [0.0, 0.1]
    for nesterov in (False, True):
        nw, nm = O.muon(w, m, g, lr, mu, wd, 2.0, QUINTIC, 1e-7, nesterov)
        for p in range(2):
            mom = mu[p] * m[p] + g[p]
            o = O.products((g[p] + mu[p] * mom if nesterov else mom)[None], QUINTIC, 1e-7)[0]
            assert np.allclose(nm[p], mom) and np.allclose(nw[p], w[p] * (1 - lr[p] * wd[p]) - lr[p] * 2.0 * o)
