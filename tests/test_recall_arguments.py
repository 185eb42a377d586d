"""What the example refuses, CPU-only."""
import pytest

from paper_2206_08888_amd import recall


def test_refusals():
    with pytest.raises(ValueError, match="memory must be one of recurrence, attention"):
        recall.train(memory="none")
    with pytest.raises(ValueError, match="width must be a positive multiple of 2"):
        recall.AttentionAgents(2, 7, 4, 4, [0.1, 0.1], device="cpu")
    with pytest.raises(ValueError, match="updates"):
        recall.train(updates=0, memory="attention")
