"""Memory layouts in every way that sequences are shared."""
import pytest

from gpu_common import ensure_built
from test_gpu_recurrence import BF16, F16, F32, _case, _verify

pytestmark = pytest.mark.gpu

# chains in vectors and single elements; whole sequences of several tiles; segments of several tiles
SHAPES = [(16, 5, 400, 64, F32), (10, 7, 300, 65, F32), (9, 15, 300, 64, BF16), (133, 2, 260, 33, F16), (40, 13, 300, 64, F16),
          (60, 9, 257, 7, BF16), (4, 40, 129, 256, F32), (30, 20, 390, 12, F16), (2, 3, 1500, 40, F16), (1, 2, 2100, 33, F32)]


@pytest.mark.parametrize("layout", ["time_major", "packed", "gaps", "broadcast"])
@pytest.mark.parametrize("P, B, T, channels, dtype", SHAPES)
def test_layouts_of_many_and_long_sequences(P, B, T, channels, dtype, layout):
    ensure_built()
    _verify(*_case(P, B, T, channels, dtype=dtype, seed=T, layout=layout))
