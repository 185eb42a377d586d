"""A population of agents with memory: python -m paper_2206_08888_amd.recall [--agents N] [--updates N] [--memory attention]

Every agent sees a cue at the first step of an episode, noise from then on, and has to name the cue at the last step.
Its network is one recurrent layer (candidate and gate from one projection, Recurrence, a linear read-out of the last
state); the weight matrices are trained by Muon with a learning rate per agent, the gate's bias by plain gradient steps.
All agents advance together: stacked weights [P, in, out], one call per layer and update.  Afterwards the trained agents
act step by step from a state table, as a simulator would have them, over episodes that start at resets.

With --memory attention the layer is linear attention with a decay for each head (queries, keys and values from one
projection, the read-out from its output at the last step), and gradients are clipped by every agent's norm before Muon
has them.
"""
import argparse

import torch

from .operators import GradientClip, LinearAttention, Muon, Recurrence

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

    RATES = -1.5, -0.9                                            # learning rates of a population, powers of ten

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


class AttentionAgents:
    """P agents with HEADS memories of width / HEADS times width / HEADS.  Observations have a constant for a last channel, which the query at
    the last step is made from; memories last for half an episode and longer ones."""

    HEADS, RATES = 2, (-2.0, -1.3)

    def __init__(self, P, width, T, batch, lr, device="cuda", seed=0, max_norm=1.0):
        if width < 1 or width % self.HEADS:
            raise ValueError("width must be a positive multiple of %d, not %d" % (self.HEADS, width))
        gen = torch.Generator(device=device)
        gen.manual_seed(seed)
        I = CUES + NOISE + 1
        self.P, self.width, self.batch = P, width, batch
        self.w_in = torch.randn((P, I, 3 * width), generator=gen, device=device) * I ** -0.5
        self.w_out = torch.randn((P, width, CUES), generator=gen, device=device) * width ** -0.5
        self.momenta = [torch.zeros_like(self.w_in), torch.zeros_like(self.w_out)]
        self.lr = torch.as_tensor(lr, dtype=torch.float32, device=device)
        self.hparams = torch.stack([self.lr, torch.full_like(self.lr, 0.95), torch.full_like(self.lr, 0.01)], 1).contiguous()
        self.max_norm = torch.full((P,), max_norm, device=device)
        self.log_decay = -torch.tensor([2.0, 0.5], device=device).expand(P, self.HEADS).contiguous() / T
        shapes = [(I, 3 * width), (width, CUES)]
        self.attention = LinearAttention(P, batch, T, self.HEADS, width // self.HEADS, width // self.HEADS, device=device)
        self.clip, self.muon = GradientClip(P, shapes, device=device), Muon(P, shapes, device=device)

    def _project(self, obs):
        """Observations with the constant [P, B * T, I + 1], and queries, keys and values as they lie in the projection."""
        P, B, T, _ = obs.shape
        x = torch.nn.functional.pad(obs, (0, 1), value=1.0).view(P, B * T, -1)
        qkv = torch.bmm(x, self.w_in).view(P, B, T, 3, self.HEADS, self.width // self.HEADS)
        return x, qkv.unbind(3)

    def gradients(self, obs, cue):
        """Losses [P], and the gradients of the mean squared error of the read-out at the last step."""
        P, B, T, _ = obs.shape
        x, (q, k, v) = self._project(obs)
        o, _ = self.attention.forward(q, k, v, self.log_decay)
        last = o[:, :, -1].reshape(P, B, self.width)
        error = torch.bmm(last, self.w_out) - torch.nn.functional.one_hot(cue, CUES).float()
        d_out = error * (2.0 / (B * CUES))
        d_o = torch.zeros_like(o)
        d_o[:, :, -1] = torch.bmm(d_out, self.w_out.transpose(1, 2).contiguous()).view(P, B, self.HEADS, -1)
        dq, dk, dv, _ = self.attention.backward(q, k, v, d_o, self.log_decay)
        d_qkv = torch.stack([dq, dk, dv], 3).view(P, B * T, 3 * self.width)
        d_w_in = torch.bmm(x.transpose(1, 2).contiguous(), d_qkv)
        return error.square().mean((1, 2)), [d_w_in, torch.bmm(last.transpose(1, 2).contiguous(), d_out)]

    def update(self, obs, cue):
        """One step; the agents' losses."""
        loss, grads = self.gradients(obs, cue)
        self.clip(grads, self.max_norm, out=grads)
        self.muon.step([self.w_in, self.w_out], self.momenta, grads, self.hparams)
        return loss

    def act(self, obs):
        """As Agents.act."""
        P, B, T, _ = obs.shape
        D = self.width // self.HEADS
        state = torch.zeros((P, B, self.HEADS, D, D), device=obs.device)
        reset = torch.zeros((P, B), dtype=torch.bool, device=obs.device)
        answers = []
        for episode in range(2):
            for t in range(T):
                _, (q, k, v) = self._project(obs[:, :, t:t + 1])
                o = self.attention.step(q[:, :, 0], k[:, :, 0], v[:, :, 0], state, self.log_decay, reset=reset if t else ~reset)
            answers.append(torch.bmm(o.view(P, B, self.width), self.w_out).argmax(2))
        assert torch.equal(answers[0], answers[1])                # the reset cut the first episode off
        return answers[1]


MEMORIES = {"recurrence": Agents, "attention": AttentionAgents}


def train(P=8, width=64, T=40, batch=32, updates=150, lr=None, device="cuda", seed=0, memory="recurrence"):
    """(losses of the first and of the last update, share of cues recalled per agent, agents)."""
    if updates < 1:
        raise ValueError("updates must be positive, not %d" % updates)
    if memory not in MEMORIES:
        raise ValueError("memory must be one of %s, not %s" % (", ".join(MEMORIES), memory))
    lr = torch.logspace(*MEMORIES[memory].RATES, P) if lr is None else lr
    agents, gen = MEMORIES[memory](P, width, T, batch, lr, device, seed), torch.Generator(device=device)
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
    p.add_argument("--memory", choices=sorted(MEMORIES), default="recurrence")
    a = p.parse_args()
    first, last, recalled, agents = train(P=a.agents, updates=a.updates, memory=a.memory)
    for i in range(a.agents):
        print("agent %d  lr %.4f  loss %.4f -> %.4f  cues recalled %.0f %%"
              % (i, agents.lr[i], first[i], last[i], 100 * recalled[i]))
