"""Peers that train small language-model policies together: Moshpit SGD with gradients of its own.

N = M^d peers, each a policy whose parameters are a row of the state X:

    x = embedding(context) * sqrt(width)      [vocab, width]
    a = relu(x W1^T)                          [hidden, width]
    logits = a W2^T                           [vocab, hidden]

An iteration draws contexts, samples an action from every peer's policy, rewards the one that a fixed rule asks
for, and takes a few steps on that sample: forward pass with the activations saved in 8 bits, clipped policy loss
with a KL term to the policy it started from, backward pass into the rows of G, then one averaging round
(theta - gamma g averaged within the groups of peers that are present).

    python examples/local_step.py [--iterations 60]
"""
from __future__ import annotations

import argparse
import math
import os
import sys
from dataclasses import dataclass

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2103_03239_amd import binding  # noqa: E402


@dataclass(frozen=True)
class Sizes:
    M: int = 4
    d: int = 2
    vocab: int = 64
    width: int = 32
    hidden: int = 96
    tokens: int = 512                  # places of a peer in an iteration

    @property
    def N(self) -> int:
        return self.M ** self.d

    @property
    def w1(self) -> int:               # where W1 begins in a peer's row; the embedding table begins it
        return self.vocab * self.width

    @property
    def w2(self) -> int:
        return self.w1 + self.hidden * self.width

    @property
    def P(self) -> int:
        return self.w2 + self.vocab * self.hidden


class Peers:
    """The peers' policies and one local step of all of them."""

    def __init__(self, sizes: Sizes, seed: int = 0, device: str = "cuda:0"):
        s = self.sizes = sizes
        self.rng = torch.Generator(device=device)
        self.rng.manual_seed(seed)
        first = torch.empty((1, s.P), device=device).normal_(generator=self.rng)      # all peers start alike
        first[:, : s.w1] *= s.width ** -0.5
        first[:, s.w1: s.w2] *= (2.0 / s.width) ** 0.5
        first[:, s.w2:] *= 0.1 * s.hidden ** -0.5
        self.X = first.repeat(s.N, 1)
        self.G = torch.zeros_like(self.X)
        self.handle = binding.Moshpit(s.N, s.P, s.M, s.d, binding.F32)
        self.handle.bind_state(self.X)

    def weights(self, X):
        s = self.sizes
        return X[:, s.w1: s.w2].view(s.N, s.hidden, s.width), X[:, s.w2:].view(s.N, s.vocab, s.hidden)

    def forward(self, contexts):
        """Logits, and what the backward pass needs of the activations: their 8-bit forms."""
        s, h = self.sizes, self.handle
        W1, W2 = self.weights(self.X)
        x = h.embed(contexts, 0, s.vocab, s.width, scale=math.sqrt(s.width))
        saved_x = h.checkpoint(x)
        a = torch.bmm(x, W1.transpose(1, 2)).relu_()
        saved_a = h.checkpoint(a)
        return torch.bmm(a, W2.transpose(1, 2)), saved_x, saved_a

    def gradients(self, contexts, actions, old_logp, ref_logp, advantage, weight, kl_coef: float = 0.01):
        """One forward and backward pass: the rows of G, and the loss's statistics per peer."""
        s, h = self.sizes, self.handle
        W1, W2 = self.weights(self.X)
        logits, saved_x, saved_a = self.forward(contexts)
        stats, _ = h.policy_loss(logits, actions, old_logp, advantage, weight, ref_logp=ref_logp, clip_low=0.2, clip_high=0.28, kl_coef=kl_coef)
        dlogits = logits                                             # (the gradient took their place)
        h.weight_grad(dlogits, *saved_a, self.G, s.w2)
        dy = torch.bmm(dlogits, W2)
        dy *= h.checkpoint_restore(*saved_a) > 0
        h.weight_grad(dy, *saved_x, self.G, s.w1)
        h.embed_grad(torch.bmm(dy, W1), contexts, self.G, 0, s.vocab, scale=math.sqrt(s.width))
        return stats

    def sample(self, contexts):
        """An action for every context, its log-probability, and the policy's probabilities."""
        logits, _, _ = self.forward(contexts)
        noise = torch.empty_like(logits).exponential_(generator=self.rng)
        actions = (logits - noise.log()).argmax(-1).int()
        return actions, self.handle.token_logp(logits, actions)


def train(sizes: Sizes, iterations: int, steps: int = 4, gamma: float = 0.2, absent: float = 0.1, seed: int = 0, say=print):
    """Rewards per iteration (mean over the peers) and the peers' distortion at the end."""
    p = Peers(sizes, seed)
    s, dev = sizes, p.X.device
    wanted = torch.randperm(s.vocab, generator=p.rng, device=dev).int()          # the rule: context -> action
    host = np.random.default_rng(seed)
    rewards, t = [], 0
    for it in range(iterations):
        contexts = torch.randint(0, s.vocab, (s.N, s.tokens), generator=p.rng, device=dev, dtype=torch.int32)
        contexts[:, s.tokens - it % 7:] = -1                                       # sequences end earlier now and then
        actions, old = p.sample(contexts)
        reward = (actions == wanted[contexts.clamp(min=0).long()]).float()
        live = (contexts >= 0).float()
        mean = (reward * live).sum(1, keepdim=True) / live.sum(1, keepdim=True)
        weight = live / live.sum(1, keepdim=True)
        rewards.append(float(mean.mean()))
        for _ in range(steps):
            alive = (host.random(s.N) >= absent).astype(np.uint8)
            p.gradients(contexts, actions, old, old, (reward - mean) * 4.0, weight)
            p.handle.sgd_round(t, p.G, gamma, alive)
            t += 1
        if say and it % 10 == 0:
            say(f"iteration {it}: reward {rewards[-1]:.3f}")
    return rewards, p.handle.dist_to_mean()


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    ap.add_argument("--iterations", type=int, default=60)
    got, spread = train(Sizes(), ap.parse_args().iterations)
    print(f"reward {got[0]:.3f} at the start, {got[-1]:.3f} at the end; distortion of the peers {spread:.3g}")
