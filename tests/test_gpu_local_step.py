"""The local step as a whole: gradients of a small policy by the library's operators against automatic
differentiation in 64 bits, and training by Moshpit SGD with them."""
import math
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


def test_gradients_against_automatic_differentiation():
    import local_step
    s = local_step.Sizes(M=2, d=2, vocab=50, width=40, hidden=72, tokens=60)
    p = local_step.Peers(s, seed=3)
    p.X.add_(torch.empty_like(p.X).normal_(0.0, 0.02, generator=p.rng))
    contexts = torch.randint(0, s.vocab, (s.N, s.tokens), generator=p.rng, device=p.X.device, dtype=torch.int32)
    contexts[0, 50:] = -1
    actions, old = p.sample(contexts)
    advantage = torch.empty((s.N, s.tokens), device=p.X.device).normal_(generator=p.rng)
    weight = (contexts >= 0).float() / s.tokens
    old = old + 0.1                                                   # ratios of exp(-0.1), off the kinks
    p.G.fill_(7.0)                                                    # every element is written
    stats = p.gradients(contexts, actions, old, old - 0.05, advantage, weight)
    p.handle.sync()

    X = p.X.double().requires_grad_()
    W1, W2 = p.weights(X)
    E = X[:, : s.w1].view(s.N, s.vocab, s.width)
    at = contexts.long()
    x = torch.where((at >= 0)[..., None], E[torch.arange(s.N, device=X.device)[:, None], at.clamp(min=0)] * math.sqrt(s.width), 0.0)
    pre = torch.bmm(x, W1.transpose(1, 2).contiguous())
    a = pre.relu()
    logits = torch.bmm(a, W2.transpose(1, 2).contiguous())
    logits.retain_grad()
    pre.retain_grad()
    lp = logits.log_softmax(-1).gather(2, actions.long()[..., None])[..., 0]
    ratio, off = (lp - old.double()).exp(), old.double() - 0.05 - lp
    loss = weight.double() * (0.01 * (off.exp() - off - 1) - torch.minimum(advantage * ratio, advantage * ratio.clamp(0.8, 1.28)))
    loss.sum().backward()
    assert torch.allclose(stats[:, 0].double(), loss.sum(1).detach(), rtol=1e-4, atol=1e-5)

    # Saved elements are off by half a step, at most the group's largest / 128, which a weight's gradient meets with |dy|; and a
    # positive pre-activation below half a step is saved as zero, whose slope is lost.  The rest is binary32.
    def half_step(v):
        most = torch.nn.functional.pad(v.abs(), (0, -v.shape[-1] % 32)).unflatten(-1, (-1, 32)).amax(-1)
        return (most / 128.0).repeat_interleave(32, -1)[..., : v.shape[-1]]

    def product(y, v):
        return torch.bmm(y.transpose(1, 2).contiguous(), v)
    dz, dy = logits.grad.abs(), pre.grad.abs()
    lost = torch.where((a > 0) & (a < half_step(a.detach())), torch.bmm(dz, W2.abs().detach()), 0.0).detach()
    small = 1e-5
    want = X.grad
    bound2 = product(dz, half_step(a.detach())) + small * product(dz, a.detach())
    bound1 = product(dy, half_step(x.detach())) + product(lost, x.abs().detach()) + small * product(dy, x.abs().detach())
    in_x = torch.bmm(lost, W1.abs().detach()) + small * torch.bmm(dy, W1.abs().detach())
    bound0 = torch.zeros((s.N, s.vocab, s.width), dtype=torch.float64, device=X.device)
    for i in range(s.N):
        bound0[i].index_add_(0, at[i].clamp(min=0), in_x[i] * math.sqrt(s.width))
    bound = torch.cat([bound0.flatten(1), bound1.flatten(1), bound2.flatten(1)], 1) + 1e-9
    assert ((p.G.double() - want).abs() <= bound).all()


def test_training_raises_the_reward():
    """A policy that answers at random is right once in `vocab` times; after training it is right more than ten times as often."""
    import local_step
    s = local_step.Sizes(M=2, d=2, vocab=16, width=32, hidden=64, tokens=512)
    rewards, spread = local_step.train(s, 40, say=None)
    assert rewards[0] < 2.0 / s.vocab
    assert sum(rewards[-5:]) / 5 > 10.0 / s.vocab
    assert math.isfinite(spread)
