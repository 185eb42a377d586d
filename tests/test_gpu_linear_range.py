"""Linear attention of large values: products of keys and queries beyond fp32's range where states and outputs are not."""
import pytest
import torch

from gpu_common import ensure_built
from linear_common import BF16, F32, check_backward, check_forward, make

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, scope="module")
def _built():
    ensure_built()


def _case(shape, dtype, scale, steps=slice(None), **sizes):
    """Inputs with values times `sizes` at `steps`, states and outputs within fp32's range: products that a group takes do not fall below it."""
    c, do, dlast = make(shape, dtype, seed=7, reset=0.01, state0=True)
    for name, size in sizes.items():
        x = do if name == "do" else c[name]
        x[:, :, steps] = (x[:, :, steps].double() * size).to(dtype)
    c["state0"] *= sizes.get("k", 1.0) * sizes.get("v", 1.0)
    dlast *= scale * sizes.get("q", 1.0) * sizes.get("do", 1.0)
    check_forward(shape, dtype, c, scale=scale)
    check_backward(shape, dtype, c, do, dlast, scale=scale)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T", [1, 40, 3000])
def test_large_keys_and_queries(T, dtype):
    _case((1, 1, T, 1, 12, 20), dtype, 1e-6, q=1e20, k=1e20, v=1e-14, do=1e-14)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T", [1, 40, 3000])
def test_large_values_and_gradients(T, dtype):
    _case((1, 1, T, 1, 12, 20), dtype, 1.0, q=1e-14, k=1e-14, v=1e20, do=1e20)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_one_large_step(dtype):
    _case((2, 1, 100, 2, 64, 64), dtype, 0.125, steps=slice(45, 46), q=1e20, k=1e20, v=1e-15, do=1e-15)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("size", [2.0 ** 50, 2.0 ** 58])
def test_values_next_to_the_border(size, dtype):
    """Values within 2^60 go through the groups' products, whose sums stay within the range."""
    _case((1, 2, 70, 1, 128, 128), dtype, 1.0, q=size, k=size, v=2.0 ** -40, do=2.0 ** -40)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("scale, v, do", [(2.0 ** 100, 2.0 ** -60, 1.0), (-(2.0 ** 100), 2.0 ** -60, 1.0), (3e38, 2.0 ** -60, 2.0 ** -30)])
def test_large_scales(scale, v, do, dtype):
    """scale * (k . q) within the range, and beyond it at ordinary keys and queries."""
    _case((1, 1, 70, 1, 12, 20), dtype, scale, v=v, do=do)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_a_large_scale_step_by_step(dtype):
    """scale * do beyond the range where scale * q * do is not, in a sequence that one large query sends step by step."""
    shape, scale, at = (1, 1, 100, 1, 12, 20), 2.0 ** 80, slice(80, 81)
    c, do, dlast = make(shape, dtype, seed=9, reset=0.01)
    c["q"], c["k"], do = ((x.double() * size).to(dtype) for x, size in ((c["q"], 2.0 ** -60), (c["k"], 2.0 ** -20), (do, 2.0 ** 60)))
    c["q"][:, :, at] = (c["q"][:, :, at].double() * 2.0 ** 85).to(dtype)
    do[:, :, at] = (do[:, :, at].double() * 2.0 ** -85).to(dtype)
    check_forward(shape, dtype, c, scale=scale)
    check_backward(shape, dtype, c, do, dlast, scale=scale)
