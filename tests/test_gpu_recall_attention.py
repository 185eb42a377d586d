"""The example's agents with linear attention for a memory: forward, backward, clipping, Muon and steps together."""
import pytest
import torch

from gpu_common import ensure_built
from paper_2206_08888_amd import recall

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, scope="module")
def _built():
    ensure_built()


def test_agents_train_and_act():
    P, B = 4, 16
    first, last, recalled, agents = recall.train(P=P, width=32, T=30, batch=B, updates=20, memory="attention")
    assert first.shape == last.shape == recalled.shape == (P,)
    assert bool(torch.isfinite(last).all()) and bool(((recalled >= 0) & (recalled <= 1)).all())
    assert all(bool(torch.isfinite(w).all()) for w in (agents.w_in, agents.w_out))


@pytest.mark.parametrize("max_norm", [1e6, 0.05])
def test_the_updates_gradients_match_autograd(max_norm):
    """Muon's momenta behind the first step are the clipped gradients: against PyTorch's of the same network in 64 bits."""
    P, T, B, W = 2, 12, 5, 16
    agents = recall.AttentionAgents(P, W, T, B, [0.01, 0.02], max_norm=max_norm)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    obs, cue = recall.episodes(P, B, T, gen, "cuda")
    w_in, w_out = leaves = [t.detach().double().clone().requires_grad_() for t in (agents.w_in, agents.w_out)]
    H, D = agents.HEADS, W // agents.HEADS
    x = torch.cat([obs.double(), torch.ones((P, B, T, 1), dtype=torch.float64, device="cuda")], 3)
    q, k, v = (x.reshape(P, B * T, -1) @ w_in).view(P, B, T, 3, H, D).unbind(3)
    S = torch.zeros((P, B, H, D, D), dtype=torch.float64, device="cuda")
    for t in range(T):
        S = torch.exp(agents.log_decay.double())[:, None, :, None, None] * S + k[:, :, t, :, :, None] * v[:, :, t, :, None, :]
    o = (q[:, :, -1, :, :, None] * S).sum(3) * D ** -0.5
    loss = (o.reshape(P, B, W) @ w_out - torch.nn.functional.one_hot(cue, recall.CUES)).square().mean((1, 2))
    loss.sum().backward()
    norms = sum(w.grad.square().sum((1, 2)) for w in leaves).sqrt()
    assert bool((norms > 0.05).all())                    # the smaller limit clips
    got = agents.update(obs, cue)
    # sums of some hundreds of fp32 products: far below 1e-5
    assert torch.allclose(got.double(), loss.detach(), rtol=1e-5)
    factor = torch.where(norms <= max_norm, torch.ones_like(norms), max_norm / norms)[:, None, None]
    for momentum, w in zip(agents.momenta, leaves):
        assert (momentum.double() - factor * w.grad).norm() < 1e-5 * (factor * w.grad).norm()
