"""Operators beside autograd: what they cannot record is refused, what they overwrite is seen."""
import pytest
import torch

import paper_2206_08888_amd as pp
from gpu_common import ensure_built

pytestmark = pytest.mark.gpu


def _inputs():
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    return [torch.randn((2, 3, 10, 8), generator=gen, device="cuda") for _ in range(3)]


@pytest.mark.parametrize("which", ["x", "g", "bias", "h0"])
def test_sequences_that_require_gradients(which):
    ensure_built()
    x, g, dy = _inputs()
    kw = dict(x=x, g=g, bias=torch.ones((2, 8), device="cuda"), h0=torch.ones((2, 3, 8), device="cuda"))
    plan = pp.Recurrence(2, 3, 10, 8)
    want = plan.forward(**kw)[0]
    kw[which] = kw[which].clone().requires_grad_()
    with pytest.raises(ValueError, match="%s requires gradients" % which):
        plan.forward(**kw)
    with torch.no_grad():
        assert torch.equal(plan.forward(**kw)[0], want)
    kw[which] = kw[which].detach()
    y, _, states = plan.forward(save=True, **kw)
    assert torch.equal(y, want) and not y.requires_grad
    if which != "h0":                                    # gradients of gradients are none of the operators'
        back = dict(states=states, x=x, g=g, dy=dy, bias=kw["bias"])
        back[which] = back[which].clone().requires_grad_()
        with pytest.raises(ValueError, match="%s requires gradients" % which):
            plan.backward(**back)


def test_steps_that_require_gradients():
    ensure_built()
    x, g, _ = (v[:, :, 0].clone() for v in _inputs())
    plan, state = pp.Recurrence(2, 3, 10, 8), torch.zeros((2, 3, 8), device="cuda")
    for args in ((x.clone().requires_grad_(), g, state), (x, g, state.clone().requires_grad_())):
        with pytest.raises(ValueError, match="requires gradients"):
            plan.step(*args)
        with torch.no_grad():
            assert not plan.step(*args).requires_grad


def test_orthogonalised_matrices_that_require_gradients():
    ensure_built()
    g = torch.randn((2, 20, 30), device="cuda")
    plan = pp.Orthogonalizer(2, 20, 30)
    want = plan(g)
    with pytest.raises(ValueError, match="g requires gradients"):
        plan(g.clone().requires_grad_())
    with torch.no_grad():
        assert torch.equal(plan(g.clone().requires_grad_()), want)


def test_an_optimiser_steps_parameters():
    """Weights that require gradients, in any mode: an update is no part of their graph."""
    ensure_built()
    w, grad = torch.randn((2, 20, 30), device="cuda"), torch.randn((2, 20, 30), device="cuda")
    hp = torch.tensor([[0.1, 0.9, 0.0]] * 2, device="cuda")
    muon, leaf = pp.Muon(2, [(20, 30)]), w.clone().requires_grad_()
    muon.step([w], [torch.zeros_like(w)], [grad], hp)
    muon.step([leaf], [torch.zeros_like(w)], [grad], hp)
    assert torch.equal(leaf.detach(), w) and leaf.is_leaf and leaf.requires_grad and leaf.grad is None


def _spoils(t, call):
    """Whether autograd notices that `call` overwrote t, which a graph had kept."""
    other = torch.ones_like(t, requires_grad=True)
    out = (other * t).sum()
    call()
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        out.backward()


def test_what_is_overwritten_is_seen():
    ensure_built()
    x, g, _ = (v[:, :, 0].clone() for v in _inputs())
    state = torch.zeros((2, 3, 8), device="cuda")
    _spoils(state, lambda: pp.Recurrence(2, 3, 10, 8).step(x, g, state))
    w, m, grad = (torch.randn((2, 20, 30), device="cuda") for _ in range(3))
    hp = torch.tensor([[0.1, 0.9, 0.0]] * 2, device="cuda")
    for t in (w, m):
        _spoils(t, lambda: pp.Muon(2, [(20, 30)]).step([w], [m], [grad], hp))
    _spoils(grad, lambda: pp.Orthogonalizer(2, 20, 30)(grad, out=grad))
    kept = grad._version
    pp.Orthogonalizer(2, 20, 30)(grad)
    assert grad._version == kept
