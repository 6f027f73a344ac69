"""Peers that train small transformers together: Moshpit SGD with the operators of a transformer block.

N = M^d peers, each a transformer of one block whose parameters are a row of the state X; its tokens come as packed sequences.

    x = embedding(token) * sqrt(width)
    x = x + dropout(attention(norm(x) Wqkv^T) Wo^T)
    x = x + dropout(relu(norm(x) W1^T) W2^T)
    logits = norm(x) Wv^T

An iteration draws sequences, samples an action at every place, rewards the one that the sequence's first token asks for (which a
place only learns by attention), and takes a few steps on that sample: forward pass with the layers' inputs saved in 8 bits, clipped
policy loss, backward pass into the rows of G, then one averaging round.

    python examples/block_step.py [--iterations 80]
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
    vocab: int = 8
    width: int = 64
    heads: int = 4
    kv_heads: int = 2
    depth: int = 16
    hidden: int = 128
    tokens: int = 512                  # places of a peer in an iteration
    dropout: float = 0.02

    @property
    def N(self) -> int:
        return self.M ** self.d

    def layers(self):
        """name -> (first parameter, shape); gains are rows of one."""
        shapes = dict(embedding=(self.vocab, self.width), gain1=(1, self.width), qkv=((self.heads + 2 * self.kv_heads) * self.depth, self.width),
                      out=(self.width, self.heads * self.depth), gain2=(1, self.width), up=(self.hidden, self.width), down=(self.width, self.hidden),
                      gain3=(1, self.width), head=(self.vocab, self.width))
        at, found = 0, {}
        for name, shape in shapes.items():
            found[name] = (at, shape)
            at += shape[0] * shape[1]
        return found, at


class Peers:
    """The peers' transformers and one local step of all of them."""

    def __init__(self, sizes: Sizes, seed: int = 0, device: str = "cuda:0"):
        s = self.sizes = sizes
        self.layers, self.P = s.layers()
        self.rng = torch.Generator(device=device)
        self.rng.manual_seed(seed)
        first = torch.empty((1, self.P), device=device).normal_(generator=self.rng)     # all peers start alike
        for name, (at, (outs, ins)) in self.layers.items():
            part = first[:, at: at + outs * ins]
            if name.startswith("gain"):
                part.fill_(1.0)
            else:
                part.mul_((0.3 if name in ("out", "down", "head") else 1.0) * ins ** -0.5)
        self.X = first.repeat(s.N, 1)
        self.G = torch.zeros_like(self.X)
        self.handle = binding.Moshpit(s.N, self.P, s.M, s.d, binding.F32)
        self.handle.bind_state(self.X)
        self.step = torch.zeros(1, dtype=torch.int64, device=device)                    # masks of dropout follow from it

    def weights(self, X, name):
        at, (outs, ins) = self.layers[name]
        return X[:, at: at + outs * ins].view(self.sizes.N, outs, ins)

    def at(self, name) -> int:
        return self.layers[name][0]

    def linear(self, x, name):
        return torch.bmm(x, self.weights(self.X, name).transpose(1, 2))

    def split(self, qkv):
        s = self.sizes
        a, b = s.heads * s.depth, s.kv_heads * s.depth
        return qkv[..., :a], qkv[..., a: a + b], qkv[..., a + b:]

    def forward(self, tokens, first):
        """Logits, and what the backward pass needs."""
        s, h = self.sizes, self.handle
        x0 = h.embed(tokens, self.at("embedding"), s.vocab, s.width, scale=math.sqrt(s.width))
        y1, _, saved1 = h.norm(x0, self.at("gain1"), saved=True)
        qkv = self.linear(y1, "qkv")
        o, lse = h.attention(*self.split(qkv), first, s.heads, s.kv_heads)
        x1 = h.dropout(self.linear(o, "out"), s.dropout, 1, step=self.step, residual=x0)
        y2, _, saved2 = h.norm(x1, self.at("gain2"), saved=True)
        u = self.linear(y2, "up").relu_()
        x2 = h.dropout(self.linear(u, "down"), s.dropout, 2, step=self.step, residual=x1)
        y3, _, saved3 = h.norm(x2, self.at("gain3"), saved=True)
        return self.linear(y3, "head"), (x0, saved1, qkv, o, lse, h.checkpoint(o), x1, saved2, u > 0, h.checkpoint(u), x2, saved3)

    def gradients(self, tokens, first, actions, old_logp, advantage, weight):
        """One forward and backward pass: the rows of G, and the loss's statistics per peer."""
        s, h, G = self.sizes, self.handle, self.G
        logits, (x0, saved1, qkv, o, lse, saved_o, x1, saved2, live, saved_u, x2, saved3) = self.forward(tokens, first)
        stats, _ = h.policy_loss(logits, actions, old_logp, advantage, weight, clip_low=0.2, clip_high=0.28)

        def back(dy, saved, name):                                       # a linear layer's: its weights' into G, its input's returned
            h.weight_grad(dy, *saved, G, self.at(name))
            return torch.bmm(dy, self.weights(self.X, name))
        dx = h.norm_grad(back(logits, saved3, "head"), x2, G, self.at("gain3"))         # (the logits' gradient took their place)
        du = back(h.dropout(dx, s.dropout, 2, step=self.step), saved_u, "down").mul_(live)
        dx = h.norm_grad(back(du, saved2, "up"), x1, G, self.at("gain2"), dtotal=dx, out=dx)
        do = back(h.dropout(dx, s.dropout, 1, step=self.step), saved_o, "out")
        dqkv = torch.empty_like(qkv)
        dq, dk, dv = self.split(dqkv)
        h.attention_grad(do, *self.split(qkv), o, lse, first, s.heads, s.kv_heads, dq=dq, dk=dk, dv=dv)
        dx = h.norm_grad(back(dqkv, saved1, "qkv"), x0, G, self.at("gain1"), dtotal=dx, out=dx)
        h.embed_grad(dx, tokens, G, self.at("embedding"), s.vocab, scale=math.sqrt(s.width))
        return stats

    def sample(self, tokens, first):
        """An action at every place and its log-probability."""
        logits, _ = self.forward(tokens, first)
        noise = torch.empty_like(logits).exponential_(generator=self.rng)
        actions = (logits - noise.log()).argmax(-1).int()
        return actions, self.handle.token_logp(logits, actions)


def sequences(sizes: Sizes, rng, device):
    """Packed sequences of 4 to 20 tokens: tokens, and where each token's sequence begins; the last places have none."""
    s = sizes
    tokens = torch.randint(0, s.vocab, (s.N, s.tokens), generator=rng, device=device, dtype=torch.int32)
    begins = torch.randint(4, 21, (s.N, s.tokens // 4), generator=rng, device=device).cumsum(1)
    begins = torch.cat([torch.zeros_like(begins[:, :1]), begins], 1)
    place = torch.arange(s.tokens, device=device).expand(s.N, -1).contiguous()
    first = begins.gather(1, torch.searchsorted(begins, place, right=True) - 1).int()
    tokens[:, s.tokens - 3:], first[:, s.tokens - 3:] = -1, -1
    return tokens, first


def train(sizes: Sizes, iterations: int, steps: int = 4, gamma: float = 0.2, absent: float = 0.1, seed: int = 0, say=print):
    """Rewards per iteration (mean over the peers) and the peers' distortion at the end."""
    p = Peers(sizes, seed)
    s, dev = sizes, p.X.device
    wanted = torch.randperm(s.vocab, generator=p.rng, device=dev).int()          # the rule: first token of a sequence -> action
    host = np.random.default_rng(seed)
    rewards, t = [], 0
    for it in range(iterations):
        tokens, first = sequences(s, p.rng, dev)
        live = (tokens >= 0).float()
        actions, old = p.sample(tokens, first)
        begin = tokens.gather(1, first.clamp(min=0).long()).clamp(min=0).long()
        reward = (actions == wanted[begin]).float()
        mean = (reward * live).sum(1, keepdim=True) / live.sum(1, keepdim=True)
        weight = live / live.sum(1, keepdim=True)
        rewards.append(float(mean.mean()))
        for _ in range(steps):
            alive = (host.random(s.N) >= absent).astype(np.uint8)
            p.gradients(tokens, first, actions, old, (reward - mean) * 4.0, weight)
            p.handle.sgd_round(t, p.G, gamma, alive)
            p.step += 1
            t += 1
        if say and it % 10 == 0:
            say(f"iteration {it}: reward {rewards[-1]:.3f}")
    return rewards, p.handle.dist_to_mean()


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    ap.add_argument("--iterations", type=int, default=80)
    got, spread = train(Sizes(), ap.parse_args().iterations)
    print(f"reward {got[0]:.3f} at the start, {got[-1]:.3f} at the end; distortion of the peers {spread:.3g}")
