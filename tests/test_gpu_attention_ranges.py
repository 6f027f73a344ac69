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
