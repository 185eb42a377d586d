"""Sizes that the boundary's 32-bit numbers cannot hold, CPU-only: refused, not cut off."""
import pytest
import torch

import paper_2206_08888_amd as pp
from test_operators_boundary import lib  # noqa: F401

FAR = 1 << 32


@pytest.mark.parametrize("sizes", [(FAR + 2, 3, 10, 4), (2, FAR + 3, 10, 4), (2, 3, FAR + 10, 4), (2, 3, 10, FAR + 4), (2, 3, (1 << 31), 4)])
def test_recurrence(lib, sizes):  # noqa: F811
    pp.Recurrence(2, 3, 10, 4, device="cuda:0")
    with pytest.raises(ValueError, match="32 bits"):
        pp.Recurrence(*sizes, device="cuda:0")


@pytest.mark.parametrize("sizes", [(FAR + 2, 5, 6), (2, FAR + 5, 6), (2, 5, FAR + 6), (-FAR + 2, 5, 6)])
def test_matrices(lib, sizes):  # noqa: F811
    with pytest.raises(ValueError, match="32 bits"):
        pp.Orthogonalizer(*sizes, device="cuda:0")
    with pytest.raises(ValueError, match="32 bits"):
        pp.Muon(sizes[0], [(2, 2), sizes[1:]], device="cuda:0")


def test_states(lib):  # noqa: F811
    plan = pp.Recurrence(2, 3, 10, 4, device="cuda:0")
    state = torch.empty((2, FAR + 3, 4), device="meta")
    with pytest.raises(ValueError, match="32 bits"):
        plan.step(torch.empty((2, 3, 4), device="meta"), torch.empty((2, 3, 4), device="meta"), state)


@pytest.mark.parametrize("updates", [0, -1])
def test_an_example_without_updates(lib, updates):  # noqa: F811
    from paper_2206_08888_amd import recall
    with pytest.raises(ValueError, match="updates"):
        recall.train(updates=updates)
