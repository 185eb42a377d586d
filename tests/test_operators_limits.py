"""Largest sizes, CPU-only: what a launch can hold is taken, what it cannot is refused, as include/pop.h says."""
import pytest

import paper_2206_08888_amd as pp
from test_operators_boundary import lib  # noqa: F401


@pytest.mark.parametrize("count, rows, cols", [(1, 16384, 16384), (1, 12288, 12288), (256, 2048, 2048), (7, 16384, 16384), (200000, 30, 40), (1000000, 3, 5),
                                               (4000, 64, 16384), ((1 << 20) - 8, 1, 1)])
def test_what_fits_is_taken(lib, count, rows, cols):  # noqa: F811
    assert lib.pop_orthogonalize_workspace_bytes(count, rows, cols) > 0, pp.pop_last_error(None)


@pytest.mark.parametrize("count, rows, cols", [(1, 16385, 1), (1 << 20, 1, 1), ((1 << 20) - 7, 1, 1), (33, 16384, 16384), (2048, 2048, 2048), (1 << 30, 64, 64), ((1 << 31) - 1, 16384, 16384),
                                               (8192, 64, 16384)])
def test_what_does_not_is_refused(lib, count, rows, cols):  # noqa: F811
    assert lib.pop_orthogonalize_workspace_bytes(count, rows, cols) == pp.POP_EUNSUPPORTED
    assert pp.pop_last_error(None) != ""
