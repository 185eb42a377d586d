"""Clipping of gradients of many pieces: a launch of its own for the norms, results past the caches, tensors in several launches."""
import pytest
import torch

import paper_2206_08888_amd as pp
from gpu_common import ensure_built
from test_gpu_clip import BF16, F16, F32, _check, _grads, _limits

pytestmark = pytest.mark.gpu
PIECE = 1 << 13                                          # elements that a workgroup takes at a time


@pytest.fixture(autouse=True, scope="module")
def _built():
    ensure_built()


def _pieces(shapes):
    return sum(-(-torch.Size(s).numel() // PIECE) for s in shapes)


def _both_ways(P, shapes, dtypes, grads=None):
    """New tensors, then in place; agents at, under and over their limits, one without, one whose norm is NaN."""
    grads = _grads(P, shapes, dtypes, seed=P) if grads is None else grads
    limits = _limits(P, shapes, P)
    if P > 1:
        limits[-1] = float("inf")
    if P > 2:
        grads[-1][0].view(-1)[7] = float("nan")
    plan = pp.GradientClip(P, shapes, dtypes)
    kept = [g.clone() for g in grads]
    got, norms = plan(grads, limits)
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip([g.contiguous() for g in grads], kept))
    _check(kept, limits, got, norms)
    assert torch.equal(plan.norms(grads).view(torch.int32), norms.view(torch.int32))
    plan(grads, limits, out=grads)
    for a, b in zip(grads, got):
        assert torch.equal(a.contiguous().view(torch.uint8), b.view(torch.uint8))


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("P, shapes", [
    (2, [(257 * PIECE + 5,)]), (3, [(1031, 2041), (1000,), (7, 13)]),              # norms by a launch of their own
    (80, [(512, 512), (300,)]),                                                    # past the caches, norms found by each workgroup
    (4, [(2100, 2048), (2048,)]),                                                  # past the caches, norms by a launch of their own
    (4, [(701, 601)] * 10), (2, [(224, 256)] * 40), (8, [(224, 256)] * 40)])       # up to 32 tensors a launch
def test_many_pieces(P, shapes, dtype):
    pieces = _pieces(shapes)
    assert pieces > 256 or pieces * P >= 2048
    _both_ways(P, shapes, [dtype] * len(shapes))


def test_types_together():
    shapes = [(300 + k, 257 + 8 * (k % 2)) for k in range(36)]
    _both_ways(3, shapes, [(F32, BF16, F16)[k % 3] for k in range(36)])


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("first, width, P", [(1, 2048, 4), (3, 2041, 4), (1, 1024, 2)])
def test_strided_and_in_place(first, width, P, dtype):
    """Parts of wider rows at odd offsets, whole vectors and not: nothing beside them is written."""
    rows = 2110 if P == 4 else 2056
    gen = torch.Generator(device="cuda")
    gen.manual_seed(width)
    wide = torch.randn((P, rows, width + 7), generator=gen, device="cuda").to(dtype)
    part = wide[..., first:first + width]
    beside = wide.clone()
    shapes = [(rows, width)]
    limits = _limits(P, shapes, 3)
    want = part.clone()
    out = torch.full((P, rows, width + 9), 9.0, dtype=dtype, device="cuda")
    plan = pp.GradientClip(P, shapes, dtype)
    got, norms = plan([part], limits, out=[out[..., 5:5 + width]])
    _check([want], limits, got, norms)
    _, again = plan([part], limits, out=[part])
    assert torch.equal(again, norms) and torch.equal(part, got[0])
    got[0].fill_(9.0)
    assert bool((out == 9.0).all())
    part.copy_(want)
    assert torch.equal(wide, beside)


def test_captured_and_replayed():
    """The launch between the two others in a graph."""
    shapes, P = [(1031, 2041), (1000,)], 3
    grads, limits = _grads(P, shapes, [F32, BF16]), _limits(P, shapes)
    plan = pp.GradientClip(P, shapes, [F32, BF16])
    want, norms = plan(grads, limits)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got, got_norms = plan(grads, limits)
    for _ in range(3):
        for x in (*got, got_norms):
            x.fill_(7.0)
        torch.randn((1 << 20,), device="cuda").sum()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got_norms, norms) and all(torch.equal(a, b) for a, b in zip(got, want))
        assert all(torch.equal(a, b) for a, b in zip(plan(grads, limits)[0], want))
