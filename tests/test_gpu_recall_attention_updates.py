"""The example's agents with linear attention: what an update changes, and that answers come from the cue and are the same step by step."""
import pytest
import torch

from gpu_common import ensure_built
from paper_2206_08888_amd import recall

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, scope="module")
def _built():
    ensure_built()


def _agents(P, lr, T=12, B=8, W=16):
    agents = recall.AttentionAgents(P, W, T, B, lr)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(11)
    return agents, recall.episodes(P, B, T, gen, "cuda")


def test_updates_move_every_agent_by_its_learning_rate():
    """Orthogonalised updates are of one size: twice the rate, twice as far (decay of weights goes with it); a rate of zero, not at all."""
    agents, (obs, cue) = _agents(4, [0.0, 0.01, 0.02, 0.04])
    for w in (agents.w_in, agents.w_out):
        w[1:] = w[:1]
    obs[:], cue[:] = obs[:1].clone(), cue[:1].clone()
    before = [w.clone() for w in (agents.w_in, agents.w_out)]
    agents.update(obs, cue)
    for w, b in zip((agents.w_in, agents.w_out), before):
        assert torch.equal(w[0], b[0])
        far = (w - b).flatten(1).double().norm(dim=1)
        assert bool((far[1:] > 0).all())
        assert torch.allclose(far[2:] / far[1:-1], torch.full((2,), 2.0, dtype=torch.float64, device="cuda"), rtol=1e-3)


def test_answers_come_from_the_cue():
    """The same noise behind another cue gives another read-out for every agent and sequence: memories reach over the episode."""
    agents, (obs, cue) = _agents(3, [0.01] * 3, T=40)

    def readout(x):
        _, (q, k, v) = agents._project(x)
        o, _ = agents.attention.forward(q, k, v, agents.log_decay)
        return torch.bmm(o[:, :, -1].reshape(3, 8, -1), agents.w_out)

    other = obs.clone()
    other[:, :, 0, :recall.CUES] = obs[:, :, 0, :recall.CUES].roll(1, 2)
    first, second = readout(obs), readout(other)
    # far above roundings: what a single step has in a memory of 40, faded by e^-2 at most
    assert bool(((first - second).abs().amax(2) > 1e-4 * first.abs().amax(2)).all())


def test_acting_answers_as_training_does():
    agents, (obs, cue) = _agents(3, [0.01, 0.02, 0.03])
    for _ in range(3):
        agents.update(obs, cue)
    _, (q, k, v) = agents._project(obs)
    o, _ = agents.attention.forward(q, k, v, agents.log_decay)
    scores = torch.bmm(o[:, :, -1].reshape(3, 8, -1), agents.w_out)
    best = scores.topk(2, dim=2).values
    clear = best[..., 0] - best[..., 1] > 1e-4 * scores.abs().amax(2)      # sums in another order do not turn these round
    assert bool(clear.any()) and torch.equal(agents.act(obs)[clear], scores.argmax(2)[clear])
