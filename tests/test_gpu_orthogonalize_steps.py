"""Orthogonalisation by many or steep steps: errors stay those of products in 32 bits, whatever the path and the type."""
import numpy as np
import pytest
import torch

import paper_2206_08888_amd as pp
from gpu_common import ensure_built
from oracle import orthogonalize as O

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
ROUNDING = {F32: 2.0 ** -24, BF16: 2.0 ** -8, F16: 2.0 ** -11}       # of a result
# five times as steep at 0 and, where it meets its largest values, as steep as a quintic that keeps within 1.01 can be
STEEP = tuple(0.9999 * k for k in (5.0, -20 / 1.01 ** 2, 16 / 1.01 ** 4))


def _low_rank(rows, cols, rank, dtype, count=2):
    rng = np.random.default_rng(rows + cols + rank)
    u = rng.standard_normal((count, rows, rank)) @ rng.standard_normal((count, rank, cols))
    return torch.from_numpy(u).to(dtype)


def _errors(u, coef, steps):
    """What the kernels and products in 32 bits are off (Frobenius), the exact result's norm, the kernels' result."""
    each = [coef] * steps
    want = O.orthogonalize(u.double().numpy(), np.float32(each).astype(np.float64), 1e-7)
    x = u.float()
    if u.shape[1] > u.shape[2]:
        x = x.transpose(1, 2)
    x = x / (x.square().sum((1, 2), keepdim=True).sqrt() + 1e-7)
    for k0, k1, k2 in each:
        a = x @ x.transpose(1, 2)
        x = k0 * x + (k1 * a + k2 * (a @ a)) @ x
    if u.shape[1] > u.shape[2]:
        x = x.transpose(1, 2)
    got = pp.Orthogonalizer(*u.shape, u.dtype, steps=steps, coef=coef)(u.cuda()).cpu().double().numpy()
    return np.linalg.norm(got - want), np.linalg.norm(x.double().numpy() - want), np.linalg.norm(want), got


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("steps", [4, 7, 8])
@pytest.mark.parametrize("rows, cols, rank", [(96, 200, 96), (300, 100, 10), (72, 300, 30)])
def test_steep_steps_for_16_bit_results(rows, cols, rank, steps, dtype):
    """Errors of one step are enlarged by those behind it, by up to 25 each: as for products in 32 bits, within the factor
    4 that tests of other sizes grant."""
    ensure_built()
    err, err32, norm, _ = _errors(_low_rank(rows, cols, rank, dtype), STEEP, steps)
    assert err <= 4 * err32 + ROUNDING[dtype] * norm, (err, err32, norm)


@pytest.mark.parametrize("coef, steps", [(pp.NS_COEF, 6), (pp.NS_COEF, 11), (pp.NS_COEF, 12), (pp.NS_COEF, 14), (pp.NS_COEF, 16), (STEEP, 8), (STEEP, 9),
                                         (STEEP, 12), (STEEP, 14), (STEEP, 16)])
@pytest.mark.parametrize("rows, cols, rank, dtype", [(6, 256, 3, F32), (17, 256, 8, F32), (50, 64, 10, F32), (64, 300, 40, F32), (300, 40, 20, F32), (64, 64, 64, F32),
                                                     (300, 40, 20, BF16), (50, 64, 10, F16)])
def test_many_steps_of_small_deficient_matrices(rows, cols, rank, dtype, coef, steps):
    """Up to 64 rows or columns, singular values of zero: what rounding makes of those grows with every step."""
    ensure_built()
    err, err32, norm, got = _errors(_low_rank(rows, cols, rank, dtype), coef, steps)
    assert np.isfinite(got).all()
    assert err <= 4 * err32 + ROUNDING[dtype] * norm, (err, err32, norm)
