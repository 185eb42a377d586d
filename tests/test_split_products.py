"""What the precision tests of the orthogonalised updates can see, CPU-only: products from operands in two halves of 11 bits pass,
and fail without either of the two small products."""
import numpy as np
import pytest

from oracle import orthogonalize as O

QUINTIC = [(3.4445, -4.7750, 2.0315)] * 5


def products32(u, coef):
    """Newton-Schulz products in 32 bits from the smaller side; u [count, rows, cols]."""
    x = np.asarray(u, np.float32)
    turned = x.shape[1] > x.shape[2]
    x = np.ascontiguousarray(x.transpose(0, 2, 1)) if turned else x
    x = x / (np.sqrt((x.astype(np.float64) ** 2).sum((1, 2), keepdims=True)) + 1e-7).astype(np.float32)
    for k0, k1, k2 in np.float32(coef):
        a = x @ x.transpose(0, 2, 1)
        x = k0 * x + (k1 * a + k2 * (a @ a)) @ x
    assert x.dtype == np.float32
    return (x.transpose(0, 2, 1) if turned else x).astype(np.float64)


def _halves(x):
    """Two halves of 11 bits in units in which the largest entries of magnitude 1.5 lie below 2^15."""
    scaled = x * 2.0 ** 14
    hi = scaled.astype(np.float16)
    return hi.astype(np.float64) / 2 ** 14, (scaled - hi).astype(np.float16).astype(np.float64) / 2 ** 14


def _split(a, b, without):
    (ah, al), (bh, bl) = _halves(a), _halves(b)
    sum_ = ah @ bh
    if without != "hi lo":
        sum_ = sum_ + ah @ bl
    if without != "lo hi":
        sum_ = sum_ + al @ bh
    return sum_.astype(np.float32).astype(np.float64)


def _steps(u, without):
    x = u / (np.linalg.norm(u) + 1e-7)
    for k0, k1, k2 in QUINTIC:
        a = _split(x, x.T, without)
        x = _split(k0 * np.eye(len(a)) + k1 * a + k2 * _split(a, a, without), x, without)
    return x


@pytest.mark.parametrize("rows, cols", [(256, 256), (131, 250), (70, 256)])
def test_what_the_comparison_sees(rows, cols):
    rng = np.random.default_rng(rows)
    u = (np.maximum(rng.standard_normal((rows, 2 * cols)), 0) @ rng.standard_normal((2 * cols, cols))).astype(np.float32).astype(np.float64)
    want = O.orthogonalize(u[None], QUINTIC, 1e-7)[0]
    err32 = np.linalg.norm(products32(u[None], QUINTIC)[0] - want)
    assert np.linalg.norm(_steps(u, None) - want) <= 4 * err32
    for without in ("hi lo", "lo hi"):
        assert np.linalg.norm(_steps(u, without) - want) > 40 * err32
