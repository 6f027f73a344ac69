"""Attention over the whole range of its values: values near the largest finite ones, keys with infinities among those that a token sees, many
tiles and many blocks.  Plain forms and bounds as in test_gpu_attention.py; U = 2^-24."""
import math

import pytest
import torch

from paper_2103_03239_amd import binding
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


# ---- the backward pass ------------------------------------------------------------

def check_gradients(act, N, M, d, T, H, K, D, first, want=None):
    g = rng(T + D)
    q, k, v = make(N, T, H, K, D, act, g)
    dout = normal((N, T, H * D), TYPES[act][0], g, 0.1)
    want = Want(q, k, v, seen_of(first), H, K, D ** -0.5, act, dout) if want is None else want(q, k, v, dout)
    with peers(M, d) as m:
        print("attention_grad", act, N, T, H, K, D, flush=True)
        out, lse = m.attention(q, k, v, first, H, K)
        got = m.attention_grad(dout, q, k, v, out, lse, first, H, K)
        again = m.attention_grad(dout, q, k, v, out, lse, first, H, K)
        m.sync()
    for x, y, name in zip(got, again, ("dq", "dk", "dv")):
        assert torch.equal(x, y)
        close(x, getattr(want, name), getattr(want, name + "_slack"))


@pytest.mark.parametrize("act,T,D", [("f32", 2_200, 32), ("bf16", 2_200, 96), ("bf16", 4_200, 64), ("bf16", 2_100, 200)])
@pytest.mark.parametrize("kind", ["one", "padded", "far"])
def test_gradients_of_many_tiles(act, T, D, kind):
    """More than 64 tiles of queries, whose ranges a block of keys looks at 64 at a time: all of them see the first keys, or hardly any, or the last."""
    g, N = rng(T), 2
    if kind == "far":                                                 # tokens see themselves, the last 150 see everything
        first = torch.arange(T, dtype=torch.int32, device=DEV).expand(N, T).contiguous()
        first[:, T - 150:] = 0
    else:
        first = firsts(kind, N, T, g)
    check_gradients(act, N, 2, 1, T, 1, 1, D, first)


@pytest.mark.parametrize("act,M,T,H,K,D", [("f32", 4, 400, 16, 8, 20), ("f32", 4, 390, 16, 8, 96), ("f32", 4, 200, 8, 4, 200), ("bf16", 4, 500, 32, 16, 64),
                                           ("bf16", 4, 390, 32, 16, 100), ("bf16", 4, 500, 8, 4, 200)])
@pytest.mark.parametrize("kind", ["packed", "holes"])
def test_gradients_of_many_blocks(act, M, T, H, K, D, kind):
    """More blocks of keys than run at once, so that each goes over all queries and heads that see its keys and writes its sums itself: several tiles of
    queries for two heads, and depths that are cut into slices.  (A compute unit of 256 runs one of these blocks, or two of bfloat16 heads up to 128.)"""
    N, slices = M * M, 1 if D <= 128 else 2 if act == "bf16" else 4
    assert N * K * ((T + 127) // 128) * slices >= 2 * 256 * (2 if act == "bf16" and D <= 128 else 1)
    check_gradients(act, N, M, 2, T, H, K, D, firsts(kind, N, T, rng(T)))


class Corrected:
    """Gradients in 64 bits, with bounds for a delta that bfloat16 outputs put off and sum ds over the keys puts right.  With weights off by a share P of
    them, dp by e, out's inner product with dout by O: delta + drift is off by sum p P (|dp - delta| + O + e) + sum p e and its sums' roundings, which
    is what dk meets.  dq: ds, which O is still in, and p, which is taken from it drift times, are rounded to half a step b."""

    def __init__(self, q, k, v, dout, seen, H, K, scale):
        b, group = TYPES["bf16"][2], H // K
        plain = Want(q, k, v, seen, H, K, scale, "bf16", dout)
        self.dv, self.dv_slack, self.dk, self.dq = plain.dv, plain.dv_slack, plain.dk, plain.dq
        out, out_slack, lse, lse_slack = split(plain.out, H), split(plain.out_slack, H), plain.lse[..., None], plain.lse_slack[..., None]
        q, do = split(q, H), split(dout, H)
        k, v = (split(x, K).repeat_interleave(group, 1) for x in (k, v))
        D, n = q.shape[3], seen.sum(2)[:, None, :, None].double()
        kt, vt = k.transpose(2, 3).contiguous(), v.transpose(2, 3).contiguous()
        p = torch.where(seen[:, None], (scale * q @ kt - lse).exp(), 0.0)
        E = (2 * D + 16) * U * torch.where(seen[:, None], scale * q.abs() @ kt.abs(), 0.0).amax(-1, keepdim=True)
        P, dp, e = E + lse_slack + 8 * U, do @ vt, (2 * D + 8) * U * (do.abs() @ vt.abs())
        delta = (do * out).sum(-1, keepdim=True)
        O = (do.abs() * out_slack).sum(-1, keepdim=True) + (2 * D + 4) * U * (do * out).abs().sum(-1, keepdim=True)  # noqa: E741
        S, pe = (p * ((dp - delta).abs() + O + e)).sum(-1, keepdim=True), (p * e).sum(-1, keepdim=True)
        off = (P + (n + 8) * U) * S + pe * 1.01 + 2 * U * delta.abs()
        ds, m = p * (dp - delta), float(q.shape[2] * group)
        slack = p * ((dp - delta).abs() * (P + 3 * U) + e + off + 2 * U * delta.abs()) * 1.01
        mine = slack + b * ds.abs() * 1.01
        shared = lambda x: merge(x.unflatten(1, (-1, group)).sum(2))  # noqa: E731
        t = lambda x: x.transpose(2, 3).contiguous()  # noqa: E731
        self.dk_slack = scale * (shared(t(mine) @ q.abs()) + 2 * m * U * shared(t(ds.abs() + slack) @ q.abs()))
        both = ds.abs() + 2 * p * (O + off)
        self.dq_slack = scale * merge((mine + 2.02 * b * p * (O + off)) @ k.abs() + 2 * (n + 6) * U * (both @ k.abs()))
        for name in ("dk", "dq"):
            setattr(self, name + "_slack", (getattr(self, name + "_slack") + (4 * U + b) * getattr(self, name).abs()) * 1.01 + TINY)


@pytest.mark.parametrize("T,H,K,D", [(300, 4, 2, 64), (260, 4, 2, 96), (260, 2, 1, 128), (150, 4, 2, 20), (150, 2, 1, 200), (140, 2, 1, 256)])
@pytest.mark.parametrize("window", [1, 2, 4, 30, 1_000])
def test_delta_is_put_right(T, H, K, D, window):
    """What rounding a bfloat16 output puts delta off by reaches neither dk nor dq (left as it is, it would be up to 5 to 25 times dk's bound and 3 to 19
    times dq's in windows of 2 tokens)."""
    t = torch.arange(T, device=DEV)
    first = (t - window + 1).clamp(min=0).int().expand(4, T).contiguous()
    check_gradients("bf16", 4, 2, 2, T, H, K, D, first, lambda q, k, v, dout: Corrected(q, k, v, dout, seen_of(first), H, K, D ** -0.5))


@pytest.mark.parametrize("act", ["f32", "bf16"])
def test_the_largest_scale(act):
    """Scores of 0 by whatever scale are 0; one that is infinite times log2 e is refused."""
    g, N, T, H, D = rng(4), 2, 70, 2, 16
    q, k, v = make(N, T, H, H, D, act, g)
    k.zero_()
    first, spans = torch.zeros((N, T), dtype=torch.int32, device=DEV), torch.tensor([0, T], dtype=torch.int32, device=DEV).expand(N, T, 2).contiguous()
    want = Want(q, k, v, seen_of(first), H, H, 1.0, act)
    with peers(2, 1) as m:
        out, lse = m.attention(q, k, v, first, H, scale=2.0 ** 127)
        for scale in (2.5e38, 3.4e38):
            for call in (lambda: m.attention(q, k, v, first, H, scale=scale), lambda: m.attention_cached(q, k, v, spans, H, scale=scale),
                         lambda: m.attention_grad(out, q, k, v, out, lse, first, H, scale=scale)):
                with pytest.raises(binding.MoshpitError, match="scale"):
                    call()
        m.sync()
    close(out, want.out, want.out_slack)
    close(lse, want.lse, want.lse_slack)
