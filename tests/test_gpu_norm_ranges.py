"""Root-mean-square norms over the whole range of their values: rows whose squares pass binary32 or vanish in it, with eps from nothing to
numbers near the largest.  Bounds as in test_gpu_norm_dropout.py; U = 2^-24 of a result for each binary32 operation."""
import pytest
import torch

from test_gpu_local_ops import DEV, TINY, TYPES, U, close, handle, normal, rng
from test_gpu_norm_dropout import depth, f32, gains, normed

pytestmark = pytest.mark.gpu

# Sizes of a row's elements.  2^122: squares pass binary32 also where elements are taken times 2^-64; 2^127: the largest; 2^64: their mean, but not
# the sum of few; 2^-140: below the normal numbers (bfloat16 has such down to 2^-133).
SIZES = [2.0 ** e for e in (127, 122, 100, 64, 30, 0, -30, -49, -51, -64, -100, -126, -130)]


def spread(shape, dtype, g):
    """Values of both signs between a half and 1, off the largest finite ones."""
    x = torch.rand(shape, generator=g, device=DEV) * 0.48 + 0.5
    return torch.where(torch.rand(shape, generator=g, device=DEV) < 0.5, -x, x).to(dtype)


@pytest.mark.parametrize("eps", [1e-6, 0.0, 1e-30, 2e38])
@pytest.mark.parametrize("act", ["f32", "bf16"])
@pytest.mark.parametrize("W", [2, 40, 500, 1_000, 3_000, 9_000, 20_000])
def test_norms_of_rows_of_all_sizes(act, eps, W):
    g, T, dtype = rng(W), 2 * len(SIZES) + 1, TYPES[act][0]
    X = gains(2, 0, W, "f32", g)
    x, dY = spread((2, T, W), dtype, g), normal((2, T, W), dtype, g)
    for n, size in enumerate(SIZES):
        x[:, 2 * n] *= size
        x[:, 2 * n + 1, : W // 2] *= size                             # beside elements of about 1
        # (a size of dx that is neither too large nor too small)
        dY[:, 2 * n] *= min(max(size, 2.0 ** -40), 2.0 ** 60)
    x[:, T - 1] = 0.0
    live = slice(0, T if eps else T - 1)                               # (a row of zeros without eps: 0 / 0)
    before = dY.clone()
    if not eps:
        dY[:, T - 1] = 0.0
    G = torch.zeros_like(X)
    with handle(X, 2, 1) as m:
        print("norms of all sizes", act, eps, W, flush=True)
        y, _, (codes, scales) = m.norm(x, 0, eps=eps, saved=True)
        dx = m.norm_grad(dY, x, G, 0, eps=eps)
        again = m.checkpoint(y)
        m.norm_grad(dY[:, live].contiguous(), x[:, live].contiguous(), G, 0, eps=eps)      # the gain's: without the row of no answer
        m.sync()
    assert torch.equal(dY[:, live], before[:, live])
    gain, h = X[:, :W].double(), x.double()
    unit, want = normed(h, gain, f32(eps))
    k = depth(W)
    close(y[:, live], want[:, live], (((k + 6) / 2 + 9) * U * want.abs() + TYPES[act][2] * want.abs() * 1.01 + TINY)[:, live])
    u = dY.double() * gain[:, None]
    inverse = (h.square().mean(-1, keepdim=True) + f32(eps)).rsqrt()
    grad = inverse * (u - unit * (u * unit).mean(-1, keepdim=True))
    size = inverse * ((k / 2 + 14) * U * u.abs() + (2 * k + 28) * U * unit.abs() * (u * unit).abs().mean(-1, keepdim=True)) + (U + TYPES[act][2]) * grad.abs()
    close(dx[:, live], grad[:, live], (size * 1.01 + TINY)[:, live])
    terms = (dY.double() * unit)[:, live]
    close(G[:, :W], terms.sum(1), ((T + k / 2 + 14) * U * terms.abs().sum(1)) * 1.01 + TINY)
    assert torch.equal(again[0], codes) and torch.equal(again[1], scales)
