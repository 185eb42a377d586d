"""A population of agents with memory: python -m paper_2206_08888_amd.recall [--agents N] [--updates N]

Every agent sees a cue at the first step of an episode, noise from then on, and has to name the cue at the last step.
Its network is one recurrent layer (candidate and gate from one projection, Recurrence, a linear read-out of the last
state); the weight matrices are trained by Muon with a learning rate per agent, the gate's bias by plain gradient steps.
All agents advance together: stacked weights [P, in, out], one call per layer and update.  Afterwards the trained agents
act step by step from a state table, as a simulator would have them, over episodes that start at resets.
"""
import argparse

import torch

from .operators import Muon, Recurrence

CUES, NOISE = 4, 4


def episodes(P, batch, T, gen, device):
    """Observations [P, batch, T, CUES + NOISE] and the cues [P, batch] to be recalled."""
    cue = torch.randint(0, CUES, (P, batch), generator=gen, device=device)
    obs = torch.zeros((P, batch, T, CUES + NOISE), device=device)
    obs[:, :, 0, :CUES] = torch.nn.functional.one_hot(cue, CUES).float()
    obs[..., CUES:] = torch.randn((P, batch, T, NOISE), generator=gen, device=device)
    return obs, cue


class Agents:
    """P agents of `width` channels."""

    def __init__(self, P, width, T, batch, lr, device="cuda", seed=0):
        gen = torch.Generator(device=device)
        gen.manual_seed(seed)
        I = CUES + NOISE
        self.P, self.C, self.batch = P, width, batch
        self.w_in = torch.randn((P, I, 2 * width), generator=gen, device=device) * I ** -0.5
        self.w_out = torch.randn((P, width, CUES), generator=gen, device=device) * width ** -0.5
        self.bias = torch.full((P, width), 2.0, device=device)
        self.momenta = [torch.zeros_like(self.w_in), torch.zeros_like(self.w_out)]
        self.lr = torch.as_tensor(lr, dtype=torch.float32, device=device)
        self.hparams = torch.stack([self.lr, torch.full_like(self.lr, 0.95), torch.full_like(self.lr, 0.01)], 1).contiguous()
        self.recurrence = Recurrence(P, batch, T, width, device=device)
        self.muon = Muon(P, [(I, 2 * width), (width, CUES)], device=device)

    def _project(self, obs):
        P, B, T, I = obs.shape
        both = torch.bmm(obs.reshape(P, B * T, I), self.w_in).view(P, B, T, 2 * self.C)
        return both[..., :self.C], both[..., self.C:]            # strided halves, as they lie

    def update(self, obs, cue):
        """One step on the mean squared error of the read-out at the last step; the agents' losses."""
        P, B, T, I = obs.shape
        x, g = self._project(obs)
        y, last, states = self.recurrence.forward(x, g, bias=self.bias, save=True)
        error = torch.bmm(last, self.w_out) - torch.nn.functional.one_hot(cue, CUES).float()
        d_out = error * (2.0 / (B * CUES))
        d_last = torch.bmm(d_out, self.w_out.transpose(1, 2).contiguous())
        d_w_out = torch.bmm(last.transpose(1, 2).contiguous(), d_out)
        dx, dg, d_bias, _ = self.recurrence.backward(states, x, g, torch.zeros_like(y), bias=self.bias, dh_last=d_last)
        d_both = torch.cat([dx, dg], 3).view(P, B * T, 2 * self.C)
        d_w_in = torch.bmm(obs.reshape(P, B * T, I).transpose(1, 2).contiguous(), d_both)
        self.muon.step([self.w_in, self.w_out], self.momenta, [d_w_in, d_w_out], self.hparams)
        self.bias -= self.lr[:, None] * 10 * d_bias
        return error.square().mean((1, 2))

    def read_out(self, state):
        return torch.bmm(state, self.w_out).argmax(2)

    def act(self, obs):
        """Step by step over obs [P, batch, T, ..], two episodes in a row, the second after a reset: its answers."""
        P, B, T, _ = obs.shape
        state = torch.zeros((P, B, self.C), device=obs.device)
        reset = torch.zeros((P, B), dtype=torch.bool, device=obs.device)
        answers = []
        for episode in range(2):
            for t in range(T):
                x, g = self._project(obs[:, :, t:t + 1])
                self.recurrence.step(x[:, :, 0], g[:, :, 0], state, bias=self.bias, reset=reset if t else ~reset)
            answers.append(self.read_out(state))
        assert torch.equal(answers[0], answers[1])                # the reset cut the first episode off
        return answers[1]


def train(P=8, width=64, T=40, batch=32, updates=150, lr=None, device="cuda", seed=0):
    """(losses of the first and of the last update, share of cues recalled per agent, agents)."""
    if updates < 1:
        raise ValueError("updates must be positive, not %d" % updates)
    lr = torch.logspace(-1.5, -0.9, P) if lr is None else lr
    agents, gen = Agents(P, width, T, batch, lr, device, seed), torch.Generator(device=device)
    gen.manual_seed(seed + 1)
    for u in range(updates):
        loss = agents.update(*episodes(P, batch, T, gen, device))
        first = loss if u == 0 else first
    obs, cue = episodes(P, batch, T, gen, device)
    return first, loss, (agents.act(obs) == cue).float().mean(1), agents


if __name__ == "__main__":
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    p.add_argument("--agents", type=int, default=8)
    p.add_argument("--updates", type=int, default=150)
    a = p.parse_args()
    first, last, recalled, agents = train(P=a.agents, updates=a.updates)
    for i in range(a.agents):
        print("agent %d  lr %.4f  loss %.4f -> %.4f  cues recalled %.0f %%"
              % (i, agents.lr[i], first[i], last[i], 100 * recalled[i]))
