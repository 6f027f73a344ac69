"""Causal attention over packed sequences, its backward pass and attention over a cache, against plain forms in 64 bits.

Bounds (U = 2^-24; a matrix instruction's addition is allowed a whole unit in the last place, 2 U): a score is off by at most 2 (depth + 4) U of
the sum A of its terms' magnitudes, a weight relatively by the scores' largest error and by its exponential, a sum of n weighted rows by
2 n U of the magnitudes' sum; in bfloat16 a weight in a product is off by half a step, 2^-8, and so is each result that is stored."""
import math

import pytest
import torch

from paper_2103_03239_amd import binding
from test_gpu_local_ops import DEV, TINY, TYPES, U, close, handle, normal, rng, rows

pytestmark = pytest.mark.gpu


def peers(M, d):
    return handle(torch.zeros((M ** d, 8), device=DEV), M, d)


def firsts(kind, N, T, g):
    """Which token every token sees first."""
    t = torch.arange(T, device=DEV).expand(N, T)
    if kind == "one" or T == 0:
        return torch.zeros((N, T), dtype=torch.int32, device=DEV)
    if kind == "none":
        return torch.full((N, T), -1, dtype=torch.int32, device=DEV)
    cuts = torch.randint(0, T, (N, max(1, T // 40)), generator=g, device=DEV)
    cuts[:, 0] = 0
    cuts = cuts.sort(1).values
    f = cuts.gather(1, torch.searchsorted(cuts, t.contiguous(), right=True) - 1)
    if kind == "window":
        f = torch.maximum(f, t - 37)
    if kind == "padded":                                              # places behind the last sequence, a peer without tokens
        f[t >= T - T // 5] = -1
        f[-1] = -1
    if kind == "holes":                                               # and places without a token anywhere, by numbers of all kinds
        wild = torch.tensor([-1, -2 ** 31, 2 ** 31 - 1, T, -5], device=DEV)
        hole = torch.rand((N, T), generator=g, device=DEV) < 0.3
        f = torch.where(hole, wild[torch.randint(0, 5, (N, T), generator=g, device=DEV)], f)
        f[:, -1] = T - 1
    if kind == "any":                                                 # in no order at all
        f = (torch.rand((N, T), generator=g, device=DEV) * (t + 2)).long() - 1
    return f.int().contiguous()


def seen_of(first):
    """[N, T, T]: which token sees which."""
    T = first.shape[1]
    t, f = torch.arange(T, device=DEV), first.long()
    live = (f >= 0) & (f <= t)
    return (f[:, :, None] <= t) & (t <= t[:, None]) & live[:, :, None] & live[:, None, :]


def split(x, n):
    """[N, rows, n * depth] -> [N, n, rows, depth] in binary64."""
    return x.double().unflatten(2, (n, -1)).transpose(1, 2).contiguous()


def merge(x):
    return x.transpose(1, 2).flatten(2)


class Want:
    """Attention in 64 bits with the slack of every result; q, k, v [N, rows, heads * depth], seen [N, queries, keys]."""

    def __init__(self, q, k, v, seen, H, K, scale, act, dout=None):
        b = TYPES[act][2]
        self.group = H // K
        q = split(q, H)
        k, v = (split(x, K).repeat_interleave(self.group, 1) for x in (k, v))
        live = seen.any(2)
        alive = seen.any(1)
        q = torch.where(live[:, None, :, None], q, 0.0)
        k, v = (torch.where(alive[:, None, :, None], x, 0.0) for x in (k, v))
        D, n = q.shape[3], seen.sum(2)[:, None, :, None].double()
        s = scale * q @ k.transpose(2, 3).contiguous()
        A = scale * q.abs() @ k.abs().transpose(2, 3).contiguous()
        some = live[:, None, :, None]
        s = s.masked_fill(~seen[:, None], -math.inf)
        top = torch.where(some, s.amax(-1, keepdim=True), 0.0) if s.shape[3] else torch.zeros_like(s.sum(-1, keepdim=True))
        p = (s - top).exp()
        total = torch.where(some, p.sum(-1, keepdim=True), 1.0)
        p = p / total
        self.lse = (top + total.log())[..., 0]
        E = (2 * D + 16) * U * (torch.where(seen[:, None], A, 0.0).amax(-1, keepdim=True) if s.shape[3] else 0.0)
        size = p @ v.abs()
        out = p @ v
        self.out, self.out_slack = merge(out), merge((2 * E + (3 * n + 32) * U + b) * size * 1.01 + b * out.abs() * 1.01 + TINY)
        self.lse_slack = (E + (n + 32) * U)[..., 0] * 1.01 + 4 * U * self.lse.abs()
        if dout is None:
            return
        do = torch.where(some, split(dout, H), 0.0)
        vt = v.transpose(2, 3).contiguous()
        dp, dp_size = do @ vt, do.abs() @ vt.abs()
        delta = (do * out).sum(-1, keepdim=True)
        off = (do.abs() * split(self.out_slack, H)).sum(-1, keepdim=True) + (2 * D + 4) * U * (do * out).abs().sum(-1, keepdim=True)
        P = E + self.lse_slack[..., None] + 8 * U
        ds = p * (dp - delta)
        ds_slack = p * ((dp - delta).abs() * (P + 3 * U + b) + (2 * D + 8) * U * dp_size + off + 2 * U * delta.abs())
        m = float(q.shape[2] * self.group)
        pt, dst, slt = (x.transpose(2, 3).contiguous() for x in (p, ds, ds_slack))
        Pt = ((P + b) * p).transpose(2, 3).contiguous()
        shared = lambda x: merge(x.unflatten(1, (-1, self.group)).sum(2))  # noqa: E731
        self.dv, self.dk, self.dq = shared(pt @ do), scale * shared(dst @ q), scale * merge(ds @ k)
        self.dv_slack = shared(Pt @ do.abs()) + 2 * m * U * shared(pt @ do.abs())
        self.dk_slack = scale * (shared(slt @ q.abs()) + 2 * m * U * shared(dst.abs() @ q.abs()))
        self.dq_slack = scale * merge(ds_slack @ k.abs() + 2 * (n + 4) * U * (ds.abs() @ k.abs()))
        for name in ("dv", "dk", "dq"):
            x = getattr(self, name)
            setattr(self, name + "_slack", (getattr(self, name + "_slack") + 4 * U * x.abs() + b * x.abs()) * 1.01 + TINY)


def make(N, T, H, K, D, act, g, pad=0, count=3):
    q = rows(N, T, H * D, TYPES[act][0], g, pad, pad % 2, 1.5)
    return [q] + [rows(N, T, K * D, TYPES[act][0], g, pad, pad % 2) for _ in range(count - 1)]


def spoil(first, *matrices):
    """Rows of places without a token may hold anything."""
    t = torch.arange(first.shape[1], device=DEV)
    empty = (first < 0) | (first > t)
    for x in matrices:
        x[empty] = math.nan


# kind, M, d, T, query heads, key heads, depth, pad: lengths about the tiles' ends, depths about the widths and odd ones
SHAPES = [
    ("one", 2, 1, 0, 1, 1, 8, 0), ("one", 2, 1, 1, 1, 1, 1, 0), ("one", 2, 2, 1, 4, 2, 64, 0), ("one", 2, 1, 2, 3, 1, 5, 1), ("one", 2, 1, 31, 2, 2, 16, 0),
    ("one", 2, 1, 33, 2, 1, 20, 1), ("padded", 3, 3, 77, 3, 1, 20, 0), ("packed", 2, 1, 64, 2, 2, 32, 0), ("packed", 2, 1, 65, 2, 1, 33, 2),
    ("holes", 2, 2, 129, 4, 2, 64, 0), ("one", 2, 1, 200, 2, 1, 96, 0), ("window", 2, 1, 300, 2, 2, 128, 0), ("packed", 2, 1, 260, 6, 2, 80, 3), ("any", 2, 1, 150, 2, 1, 64, 0),
    ("padded", 2, 2, 130, 8, 1, 100, 0), ("none", 2, 1, 40, 2, 2, 16, 0), ("one", 2, 1, 140, 2, 1, 192, 0), ("holes", 2, 1, 97, 3, 3, 200, 1), ("packed", 2, 1, 128, 1, 1, 256, 0),
    ("one", 2, 1, 600, 1, 1, 64, 0), ("packed", 2, 1, 515, 4, 4, 128, 0), ("any", 2, 1, 270, 4, 1, 130, 0), ("window", 2, 1, 1_100, 2, 1, 48, 0),
]


@pytest.mark.parametrize("act", ["f32", "bf16"])
@pytest.mark.parametrize("kind,M,d,T,H,K,D,pad", SHAPES)
def test_attention(act, kind, M, d, T, H, K, D, pad):
    N, g = M ** d, rng(T + D)
    q, k, v = make(N, T, H, K, D, act, g, pad)
    first = firsts(kind, N, T, g)
    want = Want(q, k, v, seen_of(first), H, K, D ** -0.5, act)
    spoil(first, q, k, v)
    out = rows(N, T, H * D, TYPES[act][0], g, pad, pad % 2)
    fence = out._base.clone()
    with peers(M, d) as m:
        print("attention", act, kind, N, T, H, K, D, pad, flush=True)
        got, lse = m.attention(q, k, v, first, H, K, out=out)
        new, lse2 = m.attention(q, k, v, first, H, K)
        m.sync()
    assert got is out and torch.equal(new, out) and torch.equal(lse, lse2)
    close(out, want.out, want.out_slack)
    close(lse, want.lse, want.lse_slack)
    none = ~seen_of(first).any(2)
    assert not out[none].any() and not lse.transpose(1, 2)[none].any()
    out.copy_(fence[pad % 2:].view(N, T, H * D + pad)[..., : H * D])
    assert torch.equal(out._base, fence)


@pytest.mark.parametrize("act", ["f32", "bf16"])
@pytest.mark.parametrize("kind,M,d,T,H,K,D,pad", SHAPES)
def test_attention_grad(act, kind, M, d, T, H, K, D, pad):
    N, g = M ** d, rng(T + D)
    q, k, v = make(N, T, H, K, D, act, g, pad)
    dout = rows(N, T, H * D, TYPES[act][0], g, pad, pad % 2, 0.1)
    first = firsts(kind, N, T, g)
    want = Want(q, k, v, seen_of(first), H, K, D ** -0.5, act, dout)
    spoil(first, q, k, v, dout)
    into = make(N, T, H, K, D, act, g, pad)
    fences = [x._base.clone() for x in into]
    with peers(M, d) as m:
        print("attention_grad", act, kind, N, T, H, K, D, pad, flush=True)
        out, lse = m.attention(q, k, v, first, H, K)
        got = m.attention_grad(dout, q, k, v, out, lse, first, H, K, dq=into[0], dk=into[1], dv=into[2])
        again = m.attention_grad(dout, q, k, v, out, lse, first, H, K)
        m.sync()
    assert all(a is b for a, b in zip(got, into))
    for a, b in zip(got, again):
        assert torch.equal(a, b)                                      # repeats to the bit
    close(got[2], want.dv, want.dv_slack)
    close(got[1], want.dk, want.dk_slack)
    close(got[0], want.dq, want.dq_slack)
    none = ~seen_of(first).any(2)
    for x, fence in zip(got, fences):
        assert not x[none].any()
        x.copy_(fence[pad % 2:].view(N, T, x.shape[2] + pad)[..., : x.shape[2]])
        assert torch.equal(x._base, fence)


def test_attention_grad_against_differences():
    """Central differences of <out, dout> along directions of q, k and v, attention taken in 64 bits, binary32 gradients."""
    g = rng(3)
    N, T, H, K, D = 2, 70, 4, 2, 24
    q, k, v = make(N, T, H, K, D, "f32", g)
    dout = normal((N, T, H * D), torch.float32, g)
    first = firsts("padded", N, T, g)
    with peers(2, 1) as m:
        out, lse = m.attention(q, k, v, first, H, K)
        grads = m.attention_grad(dout, q, k, v, out, lse, first, H, K)
        m.sync()
    seen, step = seen_of(first), 2.0 ** -12
    for n in range(3):
        e = normal((q, k, v)[n].shape, torch.float32, g).double()

        def value(s):
            x = [t.double() for t in (q, k, v)]
            x[n] = x[n] + s * e
            return (Want(*x, seen, H, K, D ** -0.5, "f32").out * dout.double()).sum()
        slope, got = (value(step) - value(-step)) / (2 * step), (grads[n].double() * e).sum()
        size = (grads[n].double() * e).abs().sum()
        # their own error: step^2 / 6 times a third derivative, of which each order brings at most a factor of a few (|scores'| slopes)
        assert abs(float(slope - got)) <= (50 * step ** 2 + 1_000 * U) * float(size)


@pytest.mark.parametrize("act", ["f32", "bf16"])
def test_heads_of_one_row(act):
    """Queries, keys and values as slices of one product's rows, their gradients into slices of another's."""
    g, N, T, H, K, D = rng(6), 4, 190, 4, 2, 64
    qkv = normal((N, T, (H + 2 * K) * D), TYPES[act][0], g)
    parts = [qkv[..., : H * D], qkv[..., H * D: (H + K) * D], qkv[..., (H + K) * D:]]
    dqkv = torch.empty_like(qkv)
    into = [dqkv[..., : H * D], dqkv[..., H * D: (H + K) * D], dqkv[..., (H + K) * D:]]
    dout, first = normal((N, T, H * D), TYPES[act][0], g, 0.1), firsts("packed", N, T, g)
    want = Want(*parts, seen_of(first), H, K, 0.3, act, dout)
    with peers(2, 2) as m:
        out, lse = m.attention(*parts, first, H, K, scale=0.3)
        m.attention_grad(dout, *parts, out, lse, first, H, K, scale=0.3, dq=into[0], dk=into[1], dv=into[2])
        m.sync()
    close(out, want.out, want.out_slack)
    for x, name in zip(into, ("dq", "dk", "dv")):
        close(x, getattr(want, name), getattr(want, name + "_slack"))


@pytest.mark.parametrize("act", ["f32", "bf16"])
@pytest.mark.parametrize("D", [40, 64, 128])
def test_spoilt_tokens_reach_only_those_that_see_them(act, D):
    """Infinities and NaN in one sequence's rows, and in a token's that earlier ones do not see, in tiles shared with others."""
    g, N, T, H, K = rng(D), 2, 150, 2, 1
    q, k, v = make(N, T, H, K, D, act, g)
    first = torch.zeros((N, T), dtype=torch.int32, device=DEV)
    first[:, 40:90], first[:, 90:] = 40, 90
    clean = Want(q, k, v, seen_of(first), H, K, D ** -0.5, act)
    v[0, 60, 3], v[0, 61, 4], k[0, 70, 5] = math.inf, math.nan, math.nan
    v[1, 149, 0] = -math.inf
    with peers(2, 1) as m:
        out, lse = m.attention(q, k, v, first, H, K)
        m.sync()
    good = torch.ones((N, T), dtype=torch.bool, device=DEV)
    good[0, 60:90] = False
    good[1, 149] = False
    close(out[good], clean.out[good], clean.out_slack[good])
    close(lse.transpose(1, 2)[good], clean.lse.transpose(1, 2)[good], clean.lse_slack.transpose(1, 2)[good])
    heads = out.view(N, T, H, D)
    assert torch.isinf(heads[0, 60:70, :, 3]).all() and torch.isnan(heads[0, 61:70, :, 4]).all() and torch.isnan(heads[0, 70:90]).all()
    assert (heads[1, 149, :, 0] == -math.inf).all()
    others = [d for d in range(D) if d not in (3, 4)]                 # the values' other elements are what they were
    close(heads[0, 60:70][:, :, others].flatten(1), clean.out.view(N, T, H, D)[0, 60:70][:, :, others].flatten(1),
          clean.out_slack.view(N, T, H, D)[0, 60:70][:, :, others].flatten(1))
    close(heads[1, 149, :, 1:].flatten(), clean.out.view(N, T, H, D)[1, 149, :, 1:].flatten(), clean.out_slack.view(N, T, H, D)[1, 149, :, 1:].flatten())


@pytest.mark.parametrize("act", ["f32", "bf16"])
def test_scores_far_apart(act):
    """Largest scores that grow along the keys by thousands, and equal ones."""
    N, T, H, D = 2, 300, 1, 16
    q, k, v = (torch.zeros((N, T, D), dtype=TYPES[act][0], device=DEV) for _ in range(3))
    q[..., 0] = 1.0
    k[0, :, 0] = torch.arange(T, device=DEV).to(k.dtype) * 64          # whole numbers of up to 8 bits times 64
    k[1] = -2.0 ** 60
    v.normal_(generator=rng(1))
    first = torch.zeros((N, T), dtype=torch.int32, device=DEV)
    want = Want(q, k, v, seen_of(first), H, H, 1.0, act)
    with peers(2, 1) as m:
        out, lse = m.attention(q, k, v, first, H, scale=1.0)
        m.sync()
    # The last key's score is 64 above the others' (e^-64 < 2^-92 of it): out = (w v) (1 / w).  The product, the quotient and their product are
    # rounded, and the quotient's reciprocal may be off by another: 4 U of v.  w itself cancels, but is not 1 (the scores, up to 2^14.6, are taken
    # from a largest one that is rounded after its product with log2 e), so in bfloat16 its product takes it with half a step.
    last = v[0, :256].double()
    close(out[0, :256], last, (4 * U + 2 * TYPES[act][2]) * 1.01 * last.abs())
    close(out[1], want.out[1], (16 + 3 * T) * U * v[1].double().abs().amax() + 2 * TYPES[act][2] * v[1].double().abs().amax())
    assert torch.allclose(lse[0, 0, :256].double(), want.lse[0, 0, :256], rtol=4 * U, atol=0)


# ---- over a cache ---------------------------------------------------------------

def cached_want(q, k, v, spans, new, H, K, scale, act):
    N, S = spans.shape[:2]
    keys = k.shape[1]
    begin = spans[..., 0].long().clamp(0, keys).repeat_interleave(new, 1)[..., None]
    end = spans[..., 1].long().clamp(max=keys).repeat_interleave(new, 1)[..., None]
    later = new - 1 - torch.arange(S * new, device=DEV)[None, :, None] % new
    j = torch.arange(keys, device=DEV)
    seen = (j >= begin) & (j < end - later)
    return Want(q, k, v, seen, H, K, scale, act), seen


# M, d, sequences, new tokens, rows of the cache, query heads, key heads, depth, pad
CACHED = [
    (2, 1, 1, 1, 1, 1, 1, 8, 0), (2, 2, 1, 1, 300, 8, 2, 64, 0), (2, 1, 3, 1, 200, 4, 1, 20, 1), (2, 1, 5, 2, 333, 6, 2, 128, 0), (3, 2, 2, 5, 64, 8, 1, 33, 2),
    (2, 1, 9, 1, 1_000, 8, 8, 80, 0), (2, 1, 2, 9, 700, 8, 2, 100, 0), (2, 1, 1, 1, 5_000, 2, 1, 64, 0), (2, 1, 4, 3, 3_000, 16, 1, 256, 0), (2, 1, 3, 40, 500, 2, 1, 192, 0),
    (2, 1, 0, 1, 10, 2, 1, 16, 0), (2, 1, 3, 1, 0, 2, 1, 16, 0), (2, 1, 200, 1, 4_000, 2, 2, 32, 0), (2, 1, 2, 1, 9_000, 40, 1, 128, 0),
]


@pytest.mark.parametrize("act", ["f32", "bf16"])
@pytest.mark.parametrize("M,d,S,new,keys,H,K,D,pad", CACHED)
def test_attention_cached(act, M, d, S, new, keys, H, K, D, pad):
    N, g = M ** d, rng(keys + D)
    q, = make(N, S * new, H, K, D, act, g, pad, 1)
    _, k, v = make(N, keys, H, K, D, act, g, pad)
    cap = max(1, keys // max(1, S))
    begin = (torch.arange(S, device=DEV) * cap).expand(N, S)
    spans = torch.stack([begin, begin + torch.randint(0, cap + 1, (N, S), generator=g, device=DEV)], 2).int().contiguous()
    if S >= 3:                                                        # spans of all kinds: they may share rows, be empty, or reach out of the cache
        spans[0, 0] = torch.tensor([0, keys])
        spans[0, 1] = torch.tensor([keys // 2, keys // 3])
        spans[1, 1] = torch.tensor([-7, keys // 2])
        spans[1, 2] = torch.tensor([keys // 3, 2 ** 31 - 1])
        spans[0, 2] = torch.tensor([2 ** 31 - 1, -2 ** 31])
    elif S:
        spans[0, 0] = torch.tensor([0, keys])
    want, seen = cached_want(q, k, v, spans, new, H, K, D ** -0.5, act)
    read = torch.zeros((N, keys), dtype=torch.bool, device=DEV)
    for i in range(N):
        for b, e in spans[i].tolist():
            read[i, max(b, 0): max(e, 0)] = True
    k[~read], v[~read] = math.nan, math.nan                           # rows outside the spans may hold anything
    out = rows(N, S * new, H * D, TYPES[act][0], g, pad, pad % 2)
    fence = out._base.clone()
    with peers(M, d) as m:
        print("attention_cached", act, N, S, new, keys, H, K, D, pad, flush=True)
        assert m.attention_cached(q, k, v, spans, H, K, out=out) is out
        again = m.attention_cached(q, k, v, spans, H, K)
        m.sync()
    assert torch.equal(out, again)
    close(out, want.out, want.out_slack)
    assert not out[~seen.any(2)].any()
    out.copy_(fence[pad % 2:].view(N, S * new, H * D + pad)[..., : H * D])
    assert torch.equal(out._base, fence)


@pytest.mark.parametrize("act", ["f32", "bf16"])
def test_generation_goes_on_from_a_prompt(act):
    """A prompt at once, then token after token from the cache, is attention over the whole."""
    g, N, T, H, K, D, prompt = rng(2), 4, 150, 4, 2, 64, 131
    q, k, v = make(N, T, H, K, D, act, g)
    first = torch.zeros((N, T), dtype=torch.int32, device=DEV)
    want = Want(q, k, v, seen_of(first), H, K, D ** -0.5, act)
    cache_k, cache_v = torch.full_like(k, math.nan), torch.full_like(v, math.nan)
    with peers(2, 2) as m:
        cut = first.clone()
        cut[:, prompt:] = -1
        whole, _ = m.attention(q, k, v, cut, H, K)
        cache_k[:, :prompt], cache_v[:, :prompt] = k[:, :prompt], v[:, :prompt]
        for t in range(prompt, T):
            cache_k[:, t], cache_v[:, t] = k[:, t], v[:, t]
            spans = torch.tensor([0, t + 1], dtype=torch.int32, device=DEV).expand(N, 1, 2).contiguous()
            whole[:, t: t + 1] = m.attention_cached(q[:, t: t + 1].contiguous(), cache_k, cache_v, spans, H, K)
        m.sync()
    close(whole, want.out, want.out_slack)


def test_long_matrices():
    """Rows whose elements lie beyond 2^32 bytes and 2^31 elements of a matrix's start: a cache's, and a whole prompt's by a wide stride."""
    g, N, H, K, D, keys = rng(7), 2, 2, 1, 128, 9_000_000
    k, v = (torch.empty((N, keys, K * D), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    spans = torch.tensor([[[keys - 700, keys], [0, 300]], [[keys // 2, keys // 2 + 40], [keys - 9, keys]]], dtype=torch.int32, device=DEV)
    q = normal((N, 2, H * D), torch.bfloat16, g)
    small = []
    for i in range(N):
        for b, e in spans[i].tolist():
            k[i, b:e], v[i, b:e] = normal((e - b, D), torch.bfloat16, g), normal((e - b, D), torch.bfloat16, g)
            small.append((k[i, b:e].clone(), v[i, b:e].clone()))
    with peers(2, 1) as m:
        out = m.attention_cached(q, k, v, spans, H, K)
        m.sync()
        for n, (a, b) in enumerate(small):
            want, _ = cached_want(q[n // 2: n // 2 + 1, n % 2: n % 2 + 1], a[None], b[None], torch.tensor([[[0, len(a)]]], device=DEV), 1, H, K, D ** -0.5, "bf16")
            close(out[n // 2, n % 2], want.out[0, 0], want.out_slack[0, 0])
        del k, v
        T, stride = 260, 12_000_000
        flat = torch.empty(N * T * stride, dtype=torch.bfloat16, device=DEV)
        x = flat.as_strided((N, T, 6 * 64), (T * stride, stride, 1))
        x.normal_(generator=g)
        first, dout = firsts("packed", N, T, g), normal((N, T, 2 * 64), torch.bfloat16, g)
        parts = x[..., :128], x[..., 128:256], x[..., 256:]
        want = Want(*parts, seen_of(first), 2, 2, 0.125, "bf16", dout)
        out, lse = m.attention(*parts, first, 2)
        grads = m.attention_grad(dout, *parts, out, lse, first, 2)
        m.sync()
    close(out, want.out, want.out_slack)
    for got, name in zip(grads, ("dq", "dk", "dv")):
        close(got, getattr(want, name), getattr(want, name + "_slack"))


def test_another_stream_and_replays():
    """A captured pass, replayed with other inputs between eager calls of other sizes that use the same workspace."""
    g, N, T, H, K, D = rng(5), 2, 200, 4, 1, 64
    q, k, v = make(N, T, H, K, D, "bf16", g)
    dout, first = normal((N, T, H * D), torch.bfloat16, g), firsts("packed", N, T, g)
    spans = torch.tensor([[[0, 200]], [[7, 150]]], dtype=torch.int32, device=DEV)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream), peers(2, 1) as m:
        def pass_():
            out, lse = m.attention(q, k, v, first, H, K)
            return [out, lse, *m.attention_grad(dout, q, k, v, out, lse, first, H, K), m.attention_cached(q[:, :1].contiguous(), k, v, spans, H, K)]
        pass_()
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            held = pass_()
        for n in range(4):
            q.normal_(generator=g)
            graph.replay()
            got = [x.clone() for x in held]
            want = pass_()
            big = make(N, 700, H, K, D, "bf16", g)
            m.attention_cached(big[0][:, :1].contiguous(), big[1], big[2], spans, H, K)
            o, ls = m.attention(*big, firsts("one", N, 700, g), H, K)
            m.attention_grad(o, *big, o, ls, firsts("one", N, 700, g), H, K)
            stream.synchronize()
            for a, b in zip(got, want):
                assert torch.equal(a, b)


def test_refusals():
    g = rng(1)
    q, k, v = make(2, 6, 4, 2, 16, "f32", g)
    first = firsts("one", 2, 6, g)
    spans = torch.zeros((2, 3, 2), dtype=torch.int32, device=DEV)
    with binding.Moshpit(2, 8, 2, 1, binding.F32) as m:
        with pytest.raises(binding.MoshpitError, match="no state bound"):
            m.attention(q, k, v, first, 4, 2)
    with peers(2, 1) as m:
        out, lse = m.attention(q, k, v, first, 4, 2)
        for scale in (0.0, -1.0, math.nan, math.inf):
            for call in (lambda: m.attention(q, k, v, first, 4, 2, scale=scale), lambda: m.attention_grad(out, q, k, v, out, lse, first, 4, 2, scale=scale),
                         lambda: m.attention_cached(q, k, v, spans, 4, 2, scale=scale)):
                with pytest.raises(binding.MoshpitError, match="scale"):
                    call()
        wide = normal((2, 6, 257 * 2), torch.float32, g)
        with pytest.raises(binding.MoshpitError, match="1 .. 256"):
            m.attention(wide, wide, wide, first, 2)
        three = normal((2, 6, 48), torch.float32, g)
        with pytest.raises(binding.MoshpitError, match="multiple"):
            m.attention(q, three, three, first, 4, 3)
        for call in (lambda: m.attention(q, k, v.bfloat16(), first, 4, 2), lambda: m.attention(q, k, v, first.long(), 4, 2), lambda: m.attention(q, k, v, first[:, :5], 4, 2),
                     lambda: m.attention(q, k, v, first, 5, 2), lambda: m.attention(q, k, v, first, 4, 4), lambda: m.attention(q, k[:, :5].contiguous(), v[:, :5].contiguous(), first, 4, 2),
                     lambda: m.attention(q, k, v, first, 4, 2, out=k), lambda: m.attention(q, k, v, first, 0, 2), lambda: m.attention(q, k, v, first, 4, 0),
                     lambda: m.attention_grad(out, q, k, v, out, lse[:, :3], first, 4, 2), lambda: m.attention_grad(out, q, k, v, out, lse, first, 4, 2, dk=q),
                     lambda: m.attention_cached(q, k, v, spans[:, :, :1], 4, 2), lambda: m.attention_cached(q[:, :5].contiguous(), k, v, spans, 4, 2),
                     lambda: m.attention_cached(q, k, v, spans.long(), 4, 2), lambda: m.attention_cached(q[:, :0].contiguous(), k, v, spans, 4, 2)):
            with pytest.raises(ValueError):
                call()


def test_attention_of_many_blocks():
    """Deep binary32 heads with more blocks than run at once (another form of the kernel than few take)."""
    test_attention("f32", "packed", 2, 3, 300, 32, 4, 128, 0)


@pytest.mark.parametrize("act", ["f32", "bf16"])
@pytest.mark.parametrize("D,keys", [(40, 90), (128, 2_500), (200, 300)])
def test_spoilt_new_tokens(act, D, keys):
    """Infinities and NaN in a new token's value reach it and later ones; queries that are no numbers, and scores of -inf alone, give NaN, not zeros."""
    g, N, S, new, H, K = rng(D), 2, 3, 4, 4, 2
    q, = make(N, S * new, H, K, D, act, g, 0, 1)
    _, k, v = make(N, keys * S, H, K, D, act, g)
    spans = torch.tensor([[keys * s, keys * (s + 1)] for s in range(S)], dtype=torch.int32, device=DEV).expand(N, S, 2).contiguous()
    clean, _ = cached_want(q, k, v, spans, new, H, K, D ** -0.5, act)
    q[0, 2 * new + 1] = math.nan                                      # sequence 2: one query
    q[1, :new] = 1.0                                                  # sequence 0 of peer 1: scores of -inf
    k[1, :keys] = -math.inf
    v[0, keys - 2, 3], v[0, keys - 1, D + 4] = math.inf, math.nan     # sequence 0: the third new token's first head, the last one's second
    v[0, keys + 5, 1] = -math.inf                                     # sequence 1: an old token
    with peers(2, 1) as m:
        out = m.attention_cached(q, k, v, spans, H, K)
        m.sync()
    heads = out.view(N, S, new, H, D)
    assert torch.isnan(heads[0, 2, 1]).all() and torch.isnan(heads[1, 0]).all()
    assert (heads[0, 0, 2:, :2, 3] == math.inf).all() and torch.isnan(heads[0, 0, 3, 2:, 4]).all() and (heads[0, 1, :, :2, 1] == -math.inf).all()
    good = torch.ones_like(heads, dtype=torch.bool)
    good[0, 2, 1] = good[1, 0] = False
    good[0, 0, 2:, :2, 3] = good[0, 0, 3, 2:, 4] = good[0, 1, :, :2, 1] = False
    good = good.view_as(out)
    close(out[good], clean.out[good], clean.out_slack[good])


def test_results_apart():
    """Results in the place of what is read, or of each other, are refused."""
    g = rng(8)
    q, k, v = make(2, 6, 2, 2, 16, "f32", g)
    first, spans = firsts("one", 2, 6, g), torch.zeros((2, 6, 2), dtype=torch.int32, device=DEV)
    with peers(2, 1) as m:
        out, lse = m.attention(q, k, v, first, 2)
        dout, dk = torch.ones_like(out), torch.empty_like(k)
        for call in (lambda: m.attention(q, k, v, first, 2, out=q), lambda: m.attention(q, k, v, first, 2, out=v),
                     lambda: m.attention_cached(q, k, v, spans, 2, out=k), lambda: m.attention_grad(dout, q, k, v, out, lse, first, 2, dq=dout),
                     lambda: m.attention_grad(dout, q, k, v, out, lse, first, 2, dk=k), lambda: m.attention_grad(dout, q, k, v, out, lse, first, 2, dk=dk, dv=dk),
                     lambda: m.attention_grad(dout, q, k, v, out, lse, first, 2, dv=out)):
            with pytest.raises(binding.MoshpitError, match="cannot take the place"):
                call()


@pytest.mark.parametrize("D", [64, 96, 128, 256])
def test_queries_of_one_key(D):
    """A token that sees itself alone: ds, and so dq, is 0.  delta is off by half a step of out's elements; what that brings, ds k, is taken off again as
    ds p k.  There ds is rounded to bfloat16, and p, which is 1 but for binary32 roundings, at most as much: two half steps of it are left."""
    g, N, T, H, K = rng(D), 2, 140, 4, 2
    q, k, v = make(N, T, H, K, D, "bf16", g)
    first = torch.arange(T, dtype=torch.int32, device=DEV).expand(N, T).contiguous()
    dout = normal((N, T, H * D), torch.bfloat16, g)
    with peers(2, 1) as m:
        out, lse = m.attention(q, k, v, first, H, K)
        dq, _, _ = m.attention_grad(dout, q, k, v, out, lse, first, H, K)
        m.sync()
    step = 2.0 ** -8
    off = (step + (4 * D + 16) * U) * (split(dout, H) * split(out, H)).abs().sum(-1, keepdim=True)
    bound = D ** -0.5 * merge(off * split(k, K).abs().repeat_interleave(H // K, 1)) * 2 * step * 1.05 + TINY
    assert (dq.double().abs() <= bound).all()
