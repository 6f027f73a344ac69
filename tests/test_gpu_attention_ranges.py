"""Attention over the whole range of its values: values near the largest finite ones, keys with infinities among those that a token sees, many
tiles and many blocks.  Plain forms and bounds as in test_gpu_attention.py; U = 2^-24."""
import math

import pytest
import torch

from test_gpu_attention import Want, cached_want, firsts, make, merge, peers, seen_of, split
from test_gpu_local_ops import DEV, TINY, TYPES, U, close, normal, rng

pytestmark = pytest.mark.gpu


def large_values(shape, H, g, dtype):
    """[N, rows, H * D]: peer 0: elements of one sign and of both, up to 6e37; peer 1: all 3.3e38 (the largest finite value is 3.4e38)."""
    v = torch.rand(shape, generator=g, device=DEV) * 3e37 + 3e37
    v[..., 1::3] *= -1
    v[..., 2::3] *= torch.where(torch.rand(v[..., 2::3].shape, generator=g, device=DEV) < 0.5, -1.0, 1.0)
    v[1] = 3.3e38
    return v.to(dtype)


def equal_scores(N, queries, keys, H, K, D, dtype, grow):
    """Scores of 0, and of the second half of the keys of `grow`."""
    q, k = torch.zeros((N, queries, H, D), dtype=dtype, device=DEV), torch.zeros((N, keys, K, D), dtype=dtype, device=DEV)
    q[..., 0] = 1.0
    k[:, keys // 2:, :, 0] = grow
    return q.flatten(2), k.flatten(2)


@pytest.mark.parametrize("act", ["f32", "bf16"])
@pytest.mark.parametrize("grow", [0.0, 5.375])                        # e^5.375 = 2^7.75: below what running sums are rescaled for
@pytest.mark.parametrize("S,new,keys,H,K,D", [(1, 1, 33, 2, 1, 16), (1, 1, 64, 2, 1, 64), (3, 4, 300, 4, 2, 40), (1, 1, 9_000, 2, 1, 128), (2, 3, 2_500, 16, 2, 128),
                                              (1, 1, 700, 1, 1, 200), (2, 1, 1_500, 2, 1, 256)])
def test_cached_values_near_the_largest(act, grow, S, new, keys, H, K, D):
    """Weights pass 1 within a running sum, and sums over thousands of keys the largest value; outputs lie between the values."""
    g, N, dtype = rng(keys + D), 2, TYPES[act][0]
    q, k = equal_scores(N, S * new, keys, H, K, D, dtype, grow)
    v = large_values((N, keys, K * D), K, g, dtype)
    spans = torch.tensor([0, keys], dtype=torch.int32, device=DEV).expand(N, S, 2).contiguous()
    want, _ = cached_want(q, k, v, spans, new, H, K, 1.0, act)
    with peers(2, 1) as m:
        print("large values over a cache", act, grow, S, new, keys, H, K, D, flush=True)
        out = m.attention_cached(q, k, v, spans, H, K, scale=1.0)
        m.sync()
    close(out, want.out, want.out_slack)


@pytest.mark.parametrize("act", ["f32", "bf16"])
@pytest.mark.parametrize("grow", [0.0, 5.375])
@pytest.mark.parametrize("T,H,K,D", [(33, 2, 1, 16), (300, 4, 2, 64), (260, 2, 1, 128), (150, 2, 1, 200)])
def test_values_near_the_largest(act, grow, T, H, K, D):
    g, N, dtype = rng(T + D), 2, TYPES[act][0]
    q, k = equal_scores(N, T, T, H, K, D, dtype, grow)
    v = large_values((N, T, K * D), K, g, dtype)
    first = torch.zeros((N, T), dtype=torch.int32, device=DEV)
    want = Want(q, k, v, seen_of(first), H, K, 1.0, act)
    with peers(2, 1) as m:
        print("large values", act, grow, T, H, K, D, flush=True)
        out, lse = m.attention(q, k, v, first, H, K, scale=1.0)
        m.sync()
    close(out, want.out, want.out_slack)
    close(lse, want.lse, want.lse_slack)


def spoil_keys(q, k, H, D, first_of, places):
    """Elements 0 of the queries' heads positive; the keys at `places` -inf there, so that their scores are: weights of 0."""
    q.view(*q.shape[:2], H, D)[..., 0].abs_().add_(0.5)
    for i, j in places:
        k[i, j].view(-1, D)[:, 0] = -math.inf


@pytest.mark.parametrize("act", ["f32", "bf16"])
@pytest.mark.parametrize("H,K,D", [(2, 1, 8), (4, 2, 64), (2, 1, 100), (32, 4, 128), (2, 1, 200)])
def test_scores_of_infinities(act, H, K, D):
    """A key whose score is -inf has no weight; one of +inf, or 0 times an infinity, leaves no number to those that see it."""
    g, N, T, cut = rng(D), 8, 200, 90
    q, k, v = make(N, T, H, K, D, act, g)
    first = torch.zeros((N, T), dtype=torch.int32, device=DEV)
    first[:, cut:], first[:, T - 4:] = cut, -1
    places = [(0, 0), (0, 20), (0, 37), (0, 38), (0, cut), (1, T - 5)] + [(2, j) for j in range(31, 85)] + [(3, cut + 1)]
    spoil_keys(q, k, H, D, first, places)
    dead = torch.zeros((N, T), dtype=torch.bool, device=DEV)
    for i, j in places:
        dead[i, j] = True
    seen = seen_of(first)
    want = Want(q, torch.where(dead[..., None], 0.0, k.float()).to(k.dtype), v, seen & ~dead[:, None, :], H, K, D ** -0.5, act)
    good = seen.any(2) & (seen & ~dead[:, None, :]).any(2)
    alone = seen.any(2) & ~good                                       # see nothing but scores of -inf
    assert int(alone.sum()) == 2
    k[1, 30].view(-1, D)[:, 0] = math.inf                             # sequence 0 of peer 1, from token 30 on
    good[1, 30:cut] = False
    q[3, cut + 50].view(-1, D)[:, 0] = 0.0                            # 0 times -inf
    good[3, cut + 50] = False
    q[4, 17].view(-1, D)[:, 0] = math.inf
    good[4, 17] = False
    with peers(2, 3) as m:
        print("scores of infinities", act, H, K, D, flush=True)
        out, lse = m.attention(q, k, v, first, H, K)
        m.sync()
    lse = lse.transpose(1, 2)
    close(out[good], want.out[good], want.out_slack[good])
    close(lse[good], want.lse.transpose(1, 2)[good], want.lse_slack.transpose(1, 2)[good])
    bad = seen.any(2) & ~good
    assert torch.isnan(out[bad]).all() and not torch.isfinite(lse[bad]).any()
    none = ~seen.any(2)
    assert not out[none].any() and not lse[none].any()


@pytest.mark.parametrize("act", ["f32", "bf16"])
@pytest.mark.parametrize("S,new,keys,H,K,D", [(1, 1, 40, 2, 1, 8), (2, 3, 300, 4, 2, 64), (1, 1, 9_000, 2, 1, 128), (2, 2, 900, 16, 1, 80), (1, 2, 700, 2, 1, 200)])
def test_cached_scores_of_infinities(act, S, new, keys, H, K, D):
    """The same over a cache: also where all keys that a wave or a share takes have scores of -inf."""
    g, N = rng(keys), 4
    q, = make(N, S * new, H, K, D, act, g, 0, 1)
    _, k, v = make(N, keys, H, K, D, act, g)
    spans = torch.tensor([0, keys], dtype=torch.int32, device=DEV).expand(N, S, 2).contiguous()
    places = [(0, 5), (0, keys - 1)] + [(1, j) for j in range(0, keys // 2)] + [(1, j) for j in range(keys // 2, keys - 3, 3)] + [(3, j) for j in range(keys)]
    dead = torch.zeros((N, keys), dtype=torch.bool, device=DEV)
    for i, j in places:
        dead[i, j] = True
    q.view(N, S * new, H, D)[..., 0].abs_().add_(0.5)
    clean = torch.where(dead[..., None], 0.0, k.float()).to(k.dtype)
    k.view(N, keys, K, D)[dead] = torch.cat([torch.full((K, 1), -math.inf, device=DEV), k[0, 0].view(K, D)[:, 1:].float()], 1).to(k.dtype)
    end = spans[..., 1].long().repeat_interleave(new, 1)[..., None]
    seen = torch.arange(keys, device=DEV) < end - (new - 1 - torch.arange(S * new, device=DEV)[None, :, None] % new)
    want = Want(q, clean, v, seen & ~dead[:, None, :], H, K, D ** -0.5, act)
    k[2, keys // 2].view(K, D)[:, 0] = math.inf
    with peers(2, 2) as m:
        print("scores of infinities over a cache", act, S, new, keys, H, K, D, flush=True)
        out = m.attention_cached(q, k, v, spans, H, K)
        m.sync()
    close(out[:2], want.out[:2], want.out_slack[:2])
    assert torch.isnan(out[2:]).all()
