"""The largest matrix and very many small ones."""
import numpy as np
import pytest
import torch

import paper_2206_08888_amd as pp
from gpu_common import ensure_built
from oracle import orthogonalize as O

pytestmark = pytest.mark.gpu


def test_the_largest_square_matrix():
    """One entry in every row and column: its singular values are their magnitudes, its result has theirs in the same places."""
    ensure_built()
    n = 16384
    rng = np.random.default_rng(1)
    value = rng.uniform(0.5, 1.5, n).astype(np.float32) * rng.choice([-1.0, 1.0], n).astype(np.float32)
    at = torch.from_numpy(rng.permutation(n)).cuda()
    g = torch.zeros((1, n, n), device="cuda")
    g[0, torch.arange(n, device="cuda"), at] = torch.from_numpy(value).cuda()
    o = pp.Orthogonalizer(1, n, n)(g)[0]
    got = o[torch.arange(n, device="cuda"), at].double().cpu().numpy()
    want = O.polynomial(value / np.sqrt((value.astype(np.float64) ** 2).sum()), [pp.NS_COEF] * 5)
    # eight roundings of 2^-21 a step, enlarged threefold at most, relatively, by each of the steps behind
    assert (np.abs(got - want) <= 8 * 2.0 ** -21 * sum(3.0 ** k for k in range(6)) * np.abs(want)).all()
    o[torch.arange(n, device="cuda"), at] = 0
    assert not o.any()


def test_very_many_small_matrices():
    ensure_built()
    n = 1000000
    gen = torch.Generator(device="cuda")
    gen.manual_seed(2)
    g = torch.randn((n, 3, 5), generator=gen, device="cuda")
    o = pp.Orthogonalizer(n, 3, 5)(g)
    few = torch.cat([torch.arange(40), torch.arange(n // 2, n // 2 + 40), torch.arange(n - 40, n)]).cuda()
    assert torch.equal(o[few], pp.Orthogonalizer(len(few), 3, 5)(g[few]))
