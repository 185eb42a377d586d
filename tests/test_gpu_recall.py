"""The example that runs the operators together: agents with memory learn to recall a cue, then act step by step."""
import pytest
import torch

from gpu_common import ensure_built
from paper_2206_08888_amd import recall

pytestmark = pytest.mark.gpu


def test_agents_learn_to_recall():
    ensure_built()
    first, last, recalled, _ = recall.train(P=4, width=32, T=30, batch=32, updates=120)
    # guessing recalls a quarter (standard error 8 % over 32 episodes); the error of a constant answer is 0.19
    assert float(last.min()) < 0.05 and float(recalled.max()) > 0.9, (first, last, recalled)
    assert bool((last < first).all())


def test_gradients_of_the_whole_network_match_autograd():
    """The update's gradients, seen through a momentum-free first step's momenta, against PyTorch's of the same network."""
    ensure_built()
    P, T, B, C = 2, 12, 5, 16
    agents = recall.Agents(P, C, T, B, [0.01, 0.02])
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    obs, cue = recall.episodes(P, B, T, gen, "cuda")
    leaves = [t.detach().double().clone().requires_grad_() for t in (agents.w_in, agents.w_out, agents.bias)]
    w_in, w_out, bias = leaves
    both = torch.einsum("pbti,pio->pbto", obs.double(), w_in)
    h = torch.zeros((P, B, C), dtype=torch.float64, device="cuda")
    for t in range(T):
        a = torch.sigmoid(both[:, :, t, C:] + bias[:, None])
        h = a * h + (1 - a) * both[:, :, t, :C]
    loss = (torch.einsum("pbc,pco->pbo", h, w_out) - torch.nn.functional.one_hot(cue, recall.CUES)).square().mean((1, 2))
    loss.sum().backward()
    before = agents.bias.clone()
    got = agents.update(obs, cue)
    assert torch.allclose(got.double(), loss.detach(), rtol=1e-5)
    for momentum, w in zip(agents.momenta, (w_in, w_out)):        # 0.95 * 0 + gradient
        assert (momentum.double() - w.grad).norm() < 1e-5 * w.grad.norm()
    d_bias = (before - agents.bias) / (10 * agents.lr[:, None])
    assert (d_bias.double() - bias.grad).norm() < 1e-3 * bias.grad.norm()      # a difference of values near 2
