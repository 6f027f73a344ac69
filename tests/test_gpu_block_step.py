"""The operators of a transformer block together: gradients of whole transformers by the library against automatic differentiation in 64 bits,
and a few iterations of training with them."""
import math
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


def dropped(x, p, keep, residual):
    return residual + torch.where(keep, x * (65536.0 / (65536 - math.floor(p * 65536 + 0.5))), 0.0)


def test_gradients_against_automatic_differentiation():
    import block_step
    s = block_step.Sizes(M=2, d=2, vocab=40, width=48, heads=4, kv_heads=2, depth=20, hidden=72, tokens=90, dropout=0.1)
    p = block_step.Peers(s, seed=3)
    h, dev = p.handle, p.X.device
    p.X.add_(torch.empty_like(p.X).normal_(0.0, 0.02, generator=p.rng))
    tokens, first = block_step.sequences(s, p.rng, dev)
    tokens[0, 60:], first[0, 60:] = -1, -1
    live = tokens >= 0
    actions = torch.randint(0, s.vocab, tokens.shape, generator=p.rng, device=dev, dtype=torch.int32)
    advantage = torch.empty(tokens.shape, device=dev).normal_(generator=p.rng)
    weight = live.float() / s.tokens
    logits, _ = p.forward(tokens, first)
    old = h.token_logp(logits, actions) + 0.1                            # ratios of exp(-0.1), off the kinks
    p.G.fill_(7.0)                                                       # every element is written
    stats = p.gradients(tokens, first, actions, old, advantage, weight)
    ones = torch.ones((s.N, s.tokens, s.width), device=dev)
    keep1, keep2 = (h.dropout(ones, s.dropout, seed, step=p.step) != 0 for seed in (1, 2))
    h.sync()

    X = p.X.double().requires_grad_()
    kept = {}

    def linear(x, name):
        y = torch.bmm(x, p.weights(X, name).transpose(1, 2).contiguous())
        y.retain_grad()
        kept[name] = (x.detach(), y)
        return y

    def norm(x, name):
        return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6) * p.weights(X, name)
    E = p.weights(X, "embedding")
    x = torch.where(live[..., None], E[torch.arange(s.N, device=dev)[:, None], tokens.clamp(min=0).long()] * math.sqrt(s.width), 0.0)
    q, k, v = p.split(linear(norm(x, "gain1"), "qkv"))
    q = q.unflatten(2, (s.heads, s.depth)).transpose(1, 2)
    k, v = (t.unflatten(2, (s.kv_heads, s.depth)).transpose(1, 2).repeat_interleave(s.heads // s.kv_heads, 1) for t in (k, v))
    place = torch.arange(s.tokens, device=dev)
    seen = (first[:, :, None] <= place) & (place <= place[:, None]) & live[:, :, None] & live[:, None, :]
    z = (q.contiguous() @ k.transpose(2, 3).contiguous() * s.depth ** -0.5).masked_fill(~seen[:, None], -math.inf)
    z = torch.where(live[:, None, :, None], z, 0.0)
    o = torch.where(live[:, None, :, None], z.softmax(-1) @ v.contiguous(), 0.0).transpose(1, 2).flatten(2)
    x = dropped(linear(o, "out"), s.dropout, keep1, x)
    u = linear(norm(x, "gain2"), "up").relu()
    x = dropped(linear(u, "down"), s.dropout, keep2, x)
    lp = linear(norm(x, "gain3"), "head").log_softmax(-1).gather(2, actions.long()[..., None])[..., 0]
    ratio = (lp - old.double()).exp()
    loss = -weight.double() * torch.minimum(advantage * ratio, advantage * ratio.clamp(0.8, 1.28))
    loss.sum().backward()
    assert torch.allclose(stats[:, 0].double(), loss.sum(1).detach(), rtol=1e-4, atol=1e-5)

    # Weights meet their layer's input as it was saved: off by half a step, at most the group's largest / 128, which a gradient meets with |dy|; all
    # else is binary32: a few hundred roundings of 2^-24 one after the other, over sums of up to 90 terms: within 1e-4 of the magnitudes' sums.
    small = 1e-4
    for name, (at, (outs, ins)) in p.layers.items():
        got, want = (t[:, at: at + outs * ins].double().view(s.N, outs, ins) for t in (p.G, X.grad))
        if name in kept:
            inp, y = kept[name]
            most = torch.nn.functional.pad(inp.abs(), (0, -ins % 32)).unflatten(-1, (-1, 32)).amax(-1)
            step = (most / 128.0).repeat_interleave(32, -1)[..., :ins]
            bound = torch.bmm(y.grad.abs().transpose(1, 2).contiguous(), step + small * inp.abs()) + small * want.abs().amax()
        else:
            bound = small * (want.abs() + want.abs().amax())
        assert ((got - want).abs() <= bound).all(), (name, float(((got - want).abs() / bound).max()))


def test_training():
    import block_step
    rewards, spread = block_step.train(block_step.Sizes(M=2, d=2, tokens=64), 4, say=None)
    assert len(rewards) == 4 and all(0.0 <= r <= 1.0 for r in rewards) and math.isfinite(spread)
