"""The operators of a peer's local step against plain forms in 64 bits: embeddings and their gradient, 8-bit
checkpoints, weight gradients, the clipped policy loss.  Bounds follow from the operations: a binary32 operation
is off by 2^-24 of its result, a stored bfloat16 value (8 significant bits) by 2^-8, a sum of n terms by n roundings of the sum of their
magnitudes, in whatever order; the matrix instructions' additions are allowed a whole unit in the last place, 2^-23."""
import math

import numpy as np
import pytest
import torch

from paper_2103_03239_amd import binding

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
TYPES = {"f32": (torch.float32, binding.F32, 0.0), "bf16": (torch.bfloat16, binding.BF16, 2.0 ** -8)}
U = 2.0 ** -24
TINY = 2.0 ** -126                       # below the normal numbers an error is absolute


def rng(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def normal(shape, dtype, g, scale=1.0):
    return torch.empty(shape, dtype=dtype, device=DEV).normal_(0.0, scale, generator=g)


def handle(X, M, d):
    m = binding.Moshpit(X.shape[0], X.shape[1], M, d, binding.F32 if X.dtype == torch.float32 else binding.BF16)
    m.bind_state(X)
    return m


def rows(N, T, W, dtype, g, pad=0, off=0, scale=1.0):
    """[N, T, W] with `pad` unused elements after every row, starting `off` elements into the buffer."""
    buf = normal((N * T * (W + pad) + off,), dtype, g, scale)
    return buf[off: off + N * T * (W + pad)].view(N, T, W + pad)[..., :W]


def close(got, want, bound):
    got, want = got.double(), want.double()
    bad = ~((got - want).abs() <= bound)
    assert not bad.any(), (int(bad.sum()), float(((got - want).abs() / bound).nan_to_num().max()), bad.nonzero()[:3].tolist())


# ---- embeddings ---------------------------------------------------------------

def lookup_want(X, tokens, column, V, D, scale):
    out = torch.zeros((*tokens.shape, D), dtype=torch.float64, device=DEV)
    for i in range(tokens.shape[0]):
        ok = (tokens[i] >= 0) & (tokens[i] < V)
        table = X[i, column: column + V * D].double().view(V, D)
        out[i, ok] = table[tokens[i, ok].long()] * float(np.float32(scale))
    return out


@pytest.mark.parametrize("state,act", [("f32", "f32"), ("f32", "bf16"), ("bf16", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("M,d,T,V,D,column,pad", [
    (2, 1, 1, 1, 1, 0, 0), (2, 2, 1, 500, 512, 0, 0), (2, 1, 5, 7, 7, 3, 1), (3, 2, 33, 100, 9, 1, 0), (2, 2, 130, 50, 1_003, 5, 3),
    (2, 1, 3, 11, 8, 0, 8), (2, 1, 17, 40, 2_048, 64, 0), (3, 3, 64, 1_001, 100, 7, 4), (2, 1, 700, 3, 16, 0, 1),
])
def test_embed(state, act, M, d, T, V, D, column, pad):
    N, g = M ** d, rng(T + V + D)
    X = normal((N, column + V * D + 3), TYPES[state][0], g)
    tokens = torch.randint(-1, V + 1, (N, T), generator=g, device=DEV, dtype=torch.int32)      # -1 and V: no token
    out = rows(N, T, D, TYPES[act][0], g, pad, pad % 2)
    fence = out._base.clone() if pad else None
    with handle(X, M, d) as m:
        print("embed", state, act, N, T, V, D, column, pad, flush=True)
        assert m.embed(tokens, column, V, D, scale=1.75, out=out) is out
        m.sync()
    want = lookup_want(X, tokens, column, V, D, 1.75)
    close(out, want, (U + TYPES[act][2]) * want.abs() * 1.01 + TINY)
    if pad:                                                                                    # nothing beside the rows was written
        out.copy_(fence[pad % 2:].view(N, T, D + pad)[..., :D])
        assert torch.equal(out._base, fence)


def grad_want(dY, tokens, V, scale):
    """The gradient, the sum of its terms' magnitudes, and how many they are."""
    N, T, D = dY.shape
    want = torch.zeros((N, V, D), dtype=torch.float64, device=DEV)
    size, count = torch.zeros_like(want), torch.zeros((N, V, 1), dtype=torch.float64, device=DEV)
    for i in range(N):
        ok = (tokens[i] >= 0) & (tokens[i] < V)
        t, y = tokens[i, ok].long(), dY[i, ok].double() * scale
        want[i].index_add_(0, t, y)
        size[i].index_add_(0, t, y.abs())
        count[i].index_add_(0, t, torch.ones((len(t), 1), dtype=torch.float64, device=DEV))
    return want, size, count


def some_tokens(kind, N, T, V, g):
    if kind == "zipf":
        tok = ((torch.rand((N, T), generator=g, device=DEV) * math.log(V + 1.0)).exp().long() - 1).clamp(0, V - 1).int()
        tok[:, T - T // 5:] = -1
        tok[-1] = -1                                               # a peer without tokens
    elif kind == "same":
        tok = torch.full((N, T), V // 2, dtype=torch.int32, device=DEV)
    elif kind == "few":
        tok = torch.randint(0, min(V, 4), (N, T), generator=g, device=DEV, dtype=torch.int32) * max(1, V // 4) % V
    else:
        tok = torch.randint(-1, V + 1, (N, T), generator=g, device=DEV, dtype=torch.int32)
    return tok.contiguous()


@pytest.mark.parametrize("state,act", [("f32", "f32"), ("f32", "bf16"), ("bf16", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("kind,M,d,T,V,D,column,pad", [
    ("any", 2, 1, 0, 5, 16, 0, 0), ("any", 2, 1, 1, 1, 1, 0, 0), ("any", 3, 2, 40, 64, 3, 1, 1), ("any", 2, 2, 63, 9, 33, 0, 0),
    ("same", 2, 2, 64, 3, 33, 2, 0), ("same", 2, 1, 63, 300, 128, 0, 0), ("same", 2, 1, 9_000, 255, 40, 0, 3), ("few", 2, 1, 1_024, 256, 260, 1, 0),
    ("few", 2, 2, 1_025, 257, 64, 0, 0), ("zipf", 2, 2, 8_192, 1_000, 100, 7, 4), ("zipf", 3, 1, 8_193, 70_001, 24, 0, 0),
    ("zipf", 2, 1, 20_011, 300, 513, 0, 0), ("zipf", 3, 3, 77, 1_001, 100, 7, 4), ("any", 2, 1, 257, 5_000, 1_030, 0, 2),
])
@pytest.mark.parametrize("accumulate", [False, True])
def test_embed_grad(state, act, kind, M, d, T, V, D, column, pad, accumulate):
    N, g = M ** d, rng(T + V + D)
    X = torch.zeros((N, column + V * D + 5), dtype=TYPES[state][0], device=DEV)
    G = normal(X.shape, X.dtype, g, 0.1)
    before = G.clone()
    dY = rows(N, T, D, TYPES[act][0], g, pad, pad % 2)
    tokens = some_tokens(kind, N, T, V, g)
    dY[(tokens < 0) | (tokens >= V)] = math.nan                     # places without a token may hold anything
    with handle(X, M, d) as m:
        print("embed_grad", state, act, kind, N, T, V, D, column, pad, accumulate, flush=True)
        m.embed_grad(dY, tokens, G, column, V, scale=0.375, accumulate=accumulate)
        m.sync()
        first = G.clone()
        G.copy_(before)
        m.embed_grad(dY, tokens, G, column, V, scale=0.375, accumulate=accumulate)
        m.sync()
    assert torch.equal(first, G)                                    # repeats to the bit
    want, size, count = grad_want(dY, tokens, V, 0.375)
    got = G[:, column: column + V * D].reshape(N, V, D)
    if accumulate:
        old = before[:, column: column + V * D].reshape(N, V, D).double()
        untouched = (count == 0).expand_as(want)
        assert torch.equal(got.double()[untouched], old[untouched])
        want, size = want + old, size + old.abs()
    close(got, want, (count + 3) * U * size + TYPES[state][2] * want.abs() * 1.01 + TINY)
    G[:, column: column + V * D] = before[:, column: column + V * D]
    assert torch.equal(G, before)                                   # nothing beside the table was written


def test_embed_grad_is_the_lookups_slope():
    """The lookup is linear in the table: a step of 2^-3 along D changes <lookup, dY> by 2^-3 <gradient, D>."""
    g = rng(5)
    N, T, V, D = 4, 300, 90, 48
    X, step = normal((N, V * D), torch.float32, g), normal((N, V * D), torch.float32, g)
    dY, tokens = normal((N, T, D), torch.float32, g), some_tokens("any", N, T, V, g)
    G = torch.zeros_like(X)
    with handle(X, 2, 2) as m:
        m.embed_grad(dY, tokens, G, 0, V, scale=2.0)
        a = m.embed(tokens, 0, V, D, scale=2.0)
        moved = X + 0.125 * step
        m.bind_state(moved)
        b = m.embed(tokens, 0, V, D, scale=2.0)
        m.sync()
    change = ((b.double() - a.double()) * dY.double()).sum()
    slope = 0.125 * (G.double() * step.double()).sum()
    size = ((a.double().abs() + b.double().abs()) * dY.double().abs()).sum() + 0.125 * (T + 3) * (G.double().abs() * step.double().abs()).sum()
    assert abs(float(change - slope)) <= 4 * U * float(size)


def test_embeddings_far_into_long_rows():
    """Tables whose elements lie beyond 2^31 of the state's start."""
    N, V, D = 4, 100, 640
    P = 750_000_000
    X = torch.zeros((N, P), dtype=torch.bfloat16, device=DEV)
    G = torch.zeros((N, P), dtype=torch.bfloat16, device=DEV)
    column, g = P - V * D, rng(9)
    X[:, column:] = normal((N, V * D), torch.bfloat16, g)
    tokens = some_tokens("any", N, 50, V, g)
    dY = normal((N, 50, D), torch.bfloat16, g)
    with handle(X, 2, 2) as m:
        out = m.embed(tokens, column, V, D)
        m.embed_grad(dY, tokens, G, column, V)
        m.sync()
    assert torch.equal(out.double(), lookup_want(X, tokens, column, V, D, 1.0))
    want, size, count = grad_want(dY, tokens, V, 1.0)
    close(G[:, column:].view(N, V, D), want, (count + 3) * U * size + 2.0 ** -8 * want.abs() * 1.01 + TINY)
    assert not G[:, : column].any()


# ---- checkpoints ----------------------------------------------------------------

def codes_want(x):
    """Codes and scale bytes of x (numpy, binary64, [rows, width]) from their definition."""
    R, W = x.shape
    groups = -(-W // 32)
    q, s = np.zeros((R, W), np.int8), np.zeros((R, groups), np.uint8)
    for a in range(groups):
        v = x[:, 32 * a: 32 * a + 32]
        most = np.abs(v).max(1)
        bad = ~np.isfinite(most)
        most = np.where(bad, 0.0, most)
        e = np.full(R, -126)
        for k in range(-125, 129):
            e = np.where(np.rint(np.ldexp(most, -e)) > 127, k, e)
        s[:, a] = np.where(bad, 255, e + 127)
        q[:, 32 * a: 32 * a + 32] = np.where(bad[:, None], 0, np.rint(np.ldexp(np.where(bad[:, None], 0.0, v), -e[:, None])))
    return q, s


@pytest.mark.parametrize("act", ["f32", "bf16"])
@pytest.mark.parametrize("T,W,pad", [(1, 1, 0), (3, 7, 1), (2, 8, 0), (5, 31, 2), (4, 32, 0), (4, 33, 3), (3, 1_003, 0), (200, 96, 0), (67, 100, 4), (9, 4_096, 0)])
def test_checkpoint(act, T, W, pad):
    N, g = 4, rng(T + W)
    X = torch.zeros((N, 8), device=DEV)
    x = rows(N, T, W, TYPES[act][0], g, pad, pad % 2)
    x.mul_(torch.empty(W, device=DEV).normal_(0, 3, generator=g).exp_())
    flat = x.reshape(-1)
    n = flat.numel()
    special = [0.0, -0.0, 127.5, 127.0, 63.75, 63.5, 1.0, 2.0 ** -126, 2.0 ** -133, -2.0 ** -126 * 127.5, 3.3e38, 1e-30, -126.5, 0.5]
    for k, v in enumerate(special):
        x.view(N, T, W)[k % N, (k * 7) % T, (k * 13) % W] = v
    if T * W > 500:
        x[1, 0, : min(W, 32)] = 0.0                                  # an empty group
        x[2, 1, W // 2], x[3, 1, W - 1], x[0, 1, 0] = math.inf, math.nan, -math.inf
    with handle(X, 2, 2) as m:
        print("checkpoint", act, N, T, W, pad, flush=True)
        codes, scales = m.checkpoint(x)
        back = m.checkpoint_restore(codes, scales, dtype=x.dtype)
        wide = m.checkpoint_restore(codes, scales)
        out = rows(N, T, W, torch.bfloat16, g, pad, pad % 2)
        m.checkpoint_restore(codes, scales, out=out)
        m.sync()
    q, s = codes_want(x.cpu().double().numpy().reshape(N * T, W))
    assert np.array_equal(scales.cpu().numpy().reshape(N * T, -1), s)
    assert np.array_equal(codes.cpu().numpy().reshape(N * T, W), q)
    value = np.where(s[:, np.arange(W) // 32] == 255, np.nan, np.ldexp(q.astype(np.float64), s[:, np.arange(W) // 32].astype(int) - 127))
    for y in (back, wide, out):
        assert np.array_equal(y.cpu().double().numpy().reshape(N * T, W), value, equal_nan=True)


# ---- weight gradients -------------------------------------------------------------

@pytest.mark.parametrize("state,act", [("f32", "f32"), ("f32", "bf16"), ("bf16", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("M,d,T,O,I,column,pad", [
    (2, 1, 0, 5, 7, 0, 0), (2, 1, 1, 1, 1, 0, 0), (2, 2, 3, 130, 33, 3, 1), (2, 1, 32, 128, 128, 0, 0), (3, 2, 33, 8, 200, 1, 0),
    (2, 1, 500, 129, 257, 0, 2), (2, 2, 1_000, 64, 96, 5, 0), (2, 1, 4_100, 31, 40, 0, 0), (2, 1, 260, 700, 300, 0, 0),
    (3, 1, 129, 256, 512, 0, 0), (2, 2, 700, 384, 1_000, 0, 0), (2, 1, 2_500, 520, 264, 0, 0),
])
@pytest.mark.parametrize("accumulate", [False, True])
def test_weight_grad(state, act, M, d, T, O, I, column, pad, accumulate):
    N, g = M ** d, rng(T + O + I)
    X = torch.zeros((N, column + O * I + 3), dtype=TYPES[state][0], device=DEV)
    G = normal(X.shape, X.dtype, g)
    before = G.clone()
    dY = rows(N, T, O, TYPES[act][0], g, pad, pad % 2, 0.1)
    x = rows(N, T, I, TYPES[act][0], g)
    with handle(X, M, d) as m:
        print("weight_grad", state, act, N, T, O, I, column, pad, accumulate, flush=True)
        codes, scales = m.checkpoint(x)
        m.weight_grad(dY, codes, scales, G, column, accumulate=accumulate)
        m.sync()
        first = G.clone()
        G.copy_(before)
        m.weight_grad(dY, codes, scales, G, column, accumulate=accumulate)
        value = m.checkpoint_restore(codes, scales).double()
        m.sync()
    assert torch.equal(first, G)
    y = dY.double().transpose(1, 2).contiguous()
    want, size = torch.bmm(y, value), torch.bmm(y.abs(), value.abs())
    if accumulate:
        old = before[:, column: column + O * I].reshape(N, O, I).double()
        want, size = want + old, size + old.abs()
    terms = 3 * T if act == "f32" else T
    close(G[:, column: column + O * I].reshape(N, O, I), want, (terms + 8) * 2 * U * size + TYPES[state][2] * want.abs() * 1.01 + TINY)
    G[:, column: column + O * I] = before[:, column: column + O * I]
    assert torch.equal(G, before)


@pytest.mark.parametrize("state,act", [("f32", "f32"), ("f32", "bf16"), ("bf16", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("M,d,T,O,I,column,pad", [
    (4, 2, 1, 1_024, 1_024, 0, 0), (4, 2, 31, 1_000, 1_008, 3, 24), (4, 2, 63, 1_016, 912, 0, 8), (8, 2, 64, 512, 512, 0, 0),
    (8, 2, 65, 392, 400, 1, 8), (4, 2, 128, 1_000, 1_008, 0, 24), (4, 2, 129, 1_024, 1_003, 0, 0), (8, 2, 192, 510, 496, 0, 2),
    (4, 2, 193, 1_024, 912, 0, 8), (4, 2, 300, 1_001, 1_003, 1, 1), (8, 2, 321, 400, 496, 5, 16),
])
def test_weight_grad_of_many_large_matrices(state, act, M, d, T, O, I, column, pad):
    """Enough of them for the large tiles: rows on and off 16-byte boundaries, steps that end inside, an infinity in the last token,
    NaN in the columns between the rows."""
    N, g, accumulate = M ** d, rng(T + O + I), T % 2 == 1
    X = torch.zeros((N, column + O * I + 3), dtype=TYPES[state][0], device=DEV)
    G = normal(X.shape, X.dtype, g)
    before = G.clone()
    dY = rows(N, T, O, TYPES[act][0], g, pad, 0, 0.1)
    if pad:
        dY._base.view(N, T, O + pad)[..., O:] = math.nan
    dY[0, T - 1, 1] = math.inf
    x = rows(N, T, I, TYPES[act][0], g)
    with handle(X, M, d) as m:
        print("weight_grad", state, act, N, T, O, I, column, pad, accumulate, flush=True)
        codes, scales = m.checkpoint(x)
        m.weight_grad(dY, codes, scales, G, column, accumulate=accumulate)
        m.sync()
        first = G.clone()
        G.copy_(before)
        m.weight_grad(dY, codes, scales, G, column, accumulate=accumulate)
        value = m.checkpoint_restore(codes, scales).double()
        m.sync()
    assert torch.equal(first.nan_to_num(7.0), G.nan_to_num(7.0))
    got = G[:, column: column + O * I].reshape(N, O, I)
    row = got[0, 1].double()
    assert torch.equal(row.nan_to_num(7.0), (math.inf * value[0, T - 1]).nan_to_num(7.0))     # (of an infinity: +-inf, NaN by x = 0)
    y = dY.double()
    y[0, T - 1, 1] = 0.0
    y = y.transpose(1, 2).contiguous()
    want, size = torch.bmm(y, value), torch.bmm(y.abs(), value.abs())
    if accumulate:
        old = before[:, column: column + O * I].reshape(N, O, I).double()
        want, size = want + old, size + old.abs()
    terms = 3 * T if act == "f32" else T
    bound = (terms + 8) * 2 * U * size + TYPES[state][2] * want.abs() * 1.01 + TINY
    bound[0, 1] = math.inf
    close(torch.where(torch.isinf(bound), want, got.double()), want, bound)
    G[:, column: column + O * I] = before[:, column: column + O * I]
    assert torch.equal(G, before)


def test_weight_grad_of_extreme_values():
    """binary32 factors near the ends of the range are not lost by their parts; a group that is NaN is NaN in its columns only."""
    N, T, O, I = 2, 40, 24, 70
    X, G = torch.zeros((N, O * I), device=DEV), torch.zeros((N, O * I), device=DEV)
    dY = torch.zeros((N, T, O), device=DEV)
    x = torch.zeros((N, T, I), device=DEV)
    big = torch.tensor(3.4028234e38, device=DEV)
    dY[0, 0], x[0, 0] = big, 0.5
    dY[1, 3] = 2.0 ** -100 * 1.2345678
    x[1, 3] = 3.0
    with handle(X, 2, 1) as m:
        m.weight_grad(dY, *m.checkpoint(x), G, 0)
        m.sync()
        want = torch.bmm(dY.double().transpose(1, 2).contiguous(), x.double())
        close(G.view(N, O, I), want, 8 * 2 * U * want.abs() + TINY)
        x[1, 3, 40] = math.nan
        m.weight_grad(dY, *m.checkpoint(x), G, 0)
        m.sync()
    nan = torch.isnan(G.view(N, O, I)[1])
    assert nan[:, 32:64].all() and not nan[:, :32].any() and not nan[:, 64:].any() and not torch.isnan(G[0]).any()


def test_weight_grad_is_the_layers_slope():
    """The layer y = x W^T is linear in W: <y(W + D) - y(W), dY> = <gradient, D> for the x that was saved."""
    g = rng(6)
    N, T, O, I = 2, 90, 50, 70
    X, G = torch.zeros((N, O * I), device=DEV), torch.zeros((N, O * I), device=DEV)
    dY, x, step = normal((N, T, O), torch.float32, g), normal((N, T, I), torch.float32, g), normal((N, O, I), torch.float32, g)
    with handle(X, 2, 1) as m:
        codes, scales = m.checkpoint(x)
        m.weight_grad(dY, codes, scales, G, 0)
        saved = m.checkpoint_restore(codes, scales).double()
        m.sync()
    change = (torch.bmm(saved, step.double().transpose(1, 2).contiguous()) * dY.double()).sum()
    slope = (G.double() * step.double().flatten(1)).sum()
    size = (torch.bmm(saved.abs(), step.double().abs().transpose(1, 2).contiguous()) * dY.double().abs()).sum()
    assert abs(float(change - slope)) <= (3 * T + 8) * 2 * U * float(size)


# ---- policy loss --------------------------------------------------------------------

def policy_case(N, T, V, dtype, g, pad=0):
    z = rows(N, T, V, dtype, g, pad, pad % 2, 2.0)
    tokens = torch.randint(0, V, (N, T), generator=g, device=DEV)
    z.scatter_add_(2, tokens[..., None], torch.full((N, T, 1), 5.0, dtype=dtype, device=DEV))
    lp = z.double().log_softmax(-1).gather(2, tokens[..., None])[..., 0]
    ratio = torch.empty((N, T), device=DEV).normal_(0, 0.3, generator=g).exp_()
    for edge in (0.8, 1.3):                                          # off the kinks by more than rounding
        ratio = torch.where((ratio / edge - 1).abs() < 2e-3, ratio * 1.01, ratio)
    c = {"z": z, "tokens": tokens.int(), "old": (lp - ratio.log()).float(), "ref": (lp + torch.empty((N, T), device=DEV).normal_(0, 0.4, generator=g)).float()}
    c["adv"] = torch.empty((N, T), device=DEV).normal_(generator=g)
    c["w"] = (torch.rand((N, T), generator=g, device=DEV) < 0.8).float() * torch.rand((N, T), generator=g, device=DEV)
    return c


def policy_want(c, kl, low=0.2, high=0.3, ref=True):
    """In binary64: gradient, stats, lp; and how far binary32 may be off each."""
    z, V = c["z"].double(), c["z"].shape[2]
    tok = c["tokens"].long()
    live = (c["w"] != 0) & (tok >= 0) & (tok < V)
    tok = tok.clamp(0, V - 1)[..., None]
    z = torch.where(live[..., None], z, torch.zeros_like(z))
    m, lse = z.amax(-1), torch.logsumexp(z, -1)
    lp = z.gather(2, tok)[..., 0] - lse
    p = (z - lse[..., None]).exp()
    w, A, old, rf = (c[k].double() for k in ("w", "adv", "old", "ref"))
    low, high = 1.0 - float(np.float32(low)), 1.0 + float(np.float32(high))
    kl = float(np.float32(kl))
    r = (lp - old).exp()
    gain, held = A * r, A * r.clamp(low, high)
    e = (rf - lp).exp() if ref else torch.ones_like(lp)
    k = e - (rf - lp) - 1 if ref else torch.zeros_like(lp)
    clipped = gain > held
    loss = w * (kl * k - torch.minimum(gain, held))
    slope = w * (kl * (1 - e) - torch.where(clipped, torch.zeros_like(gain), gain))
    zero = torch.zeros_like(lp)
    loss, slope, lp_out = (torch.where(live, x, zero) for x in (loss, slope, lp))
    wk, wc = torch.where(live, w * k, zero), torch.where(live & clipped, w, zero)
    grad = -slope[..., None] * p
    grad.scatter_add_(2, tok, slope[..., None])
    # binary32: x - m and its product with log2 e are off by 2^-24 each, exp2 by 2^-23, the sum by an addition per element of a
    # thread and one per exchange
    finite = torch.where(z == -math.inf, m[..., None], z)
    d = (m[..., None] - finite)
    n = max(128, V / 256) + 32
    s_off = U * (n + 4 + 3 * (p * d).sum(-1))
    lp_off = 4 * U * (m.abs() + lp.abs() + lse.abs() + 1) + s_off
    r_off = lp_off + U * (lp.abs() + old.abs() + 4)
    e_off = lp_off + U * (lp.abs() + rf.abs() + 4)
    slope_off = w * (abs(kl) * (e * e_off + 2 * U * (1 + e)) + gain.abs() * (r_off + 4 * U)) + 4 * U * slope.abs()
    loss_off = w * (abs(kl) * (e * e_off + lp_off + 4 * U * (e + (rf - lp).abs() + 1)) + gain.abs() * (r_off + 4 * U)) + 4 * U * loss.abs()
    grad_off = slope_off[..., None] * (p + torch.zeros_like(p).scatter_(2, tok, 1.0)) + slope.abs()[..., None] * p * (U * (3 * d + 8) + s_off[..., None]) \
        + 2 * U * grad.abs()
    stats = torch.stack([loss.sum(1), wk.sum(1), wc.sum(1)], 1)
    k_off = w * (e * e_off + lp_off + 4 * U * (e + (rf - lp).abs() + 1)) if ref else zero
    off = torch.stack([loss_off.sum(1) + 2 * U * loss.abs().sum(1), k_off.sum(1) + 2 * U * wk.abs().sum(1), 2 * U * wc.sum(1)], 1)
    return grad, stats, lp_out, grad_off, off, lp_off


@pytest.mark.parametrize("act", ["f32", "bf16"])
@pytest.mark.parametrize("M,d,T,V,pad,kl", [
    (2, 1, 0, 9, 0, 0.1), (2, 1, 1, 1, 0, 0.1), (2, 1, 1, 2, 1, 0.0), (2, 2, 5, 7, 0, 0.1), (3, 2, 3, 63, 3, 0.05), (2, 2, 9, 1_000, 1, 0.1),
    (2, 1, 4, 4_096, 0, 0.0), (2, 1, 3, 4_097, 0, 0.1), (2, 2, 40, 8_200, 2, 0.1), (2, 1, 7, 16_500, 1, 0.02), (2, 1, 2, 33_001, 0, 0.1),
    (2, 2, 30, 50_001, 0, 0.1), (2, 1, 3, 65_600, 1, 0.1), (2, 1, 1, 131_072, 0, 0.1), (2, 1, 2, 200_003, 5, 0.1), (2, 2, 300, 70_000, 0, 0.1),
    (2, 2, 1_100, 300, 1, 0.1), (2, 2, 1_030, 7, 0, 0.1), (3, 2, 500, 512, 3, 0.05), (8, 4, 1, 100, 0, 0.1), (2, 3, 700, 1_024, 0, 0.0),     # many short rows
])
@pytest.mark.parametrize("in_place", [False, True])
def test_policy_loss(act, M, d, T, V, pad, kl, in_place):
    N, g = M ** d, rng(T + V)
    dtype, _, u = TYPES[act]
    c = policy_case(N, T, V, dtype, g, pad)
    if V > 60 and T:
        c["z"][..., 11:14] = -math.inf                               # never sampled ...
        hit = (c["tokens"] >= 11) & (c["tokens"] < 14)
        c["tokens"][hit] = 3                                         # ... so not among the tokens
    if T > 2:
        c["tokens"][0, 1], c["tokens"][1, 2] = -1, V                 # places without a token
        c["w"][-1] = 0                                               # a peer whose mask leaves nothing
        c["z"][-1, 0] = math.nan
        c["z"][0, 1] = math.inf
    X = torch.zeros((N, 16), device=DEV)
    z = c["z"].clone() if not in_place else c["z"]
    want = policy_want({**c, "z": c["z"].clone()}, kl)
    grad = z if in_place else torch.full_like(rows(N, T, V, dtype, g, pad, pad % 2), 7.0)
    with handle(X, M, d) as m:
        print("policy", act, N, T, V, pad, kl, in_place, flush=True)
        scored = m.token_logp(c["z"], c["tokens"])
        stats, logp = m.policy_loss(z, c["tokens"], c["old"], c["adv"], c["w"], ref_logp=c["ref"], clip_low=0.2, clip_high=0.3, kl_coef=kl,
                                    grad=None if in_place else grad)
        m.sync()
    w_grad, w_stats, w_lp, grad_off, stats_off, lp_off = want
    live = (c["w"] != 0) & (c["tokens"] >= 0) & (c["tokens"] < V)
    close(logp, w_lp, lp_off)
    close(stats, w_stats, stats_off + TINY)
    close(grad, w_grad, grad_off + u * w_grad.abs() * 1.01 + TINY)
    assert not grad[~live].any()
    close(scored[live], w_lp[live], lp_off[live])
    assert not scored[(c["tokens"] < 0) | (c["tokens"] >= V)].any()


def test_policy_loss_without_reference():
    g = rng(3)
    c = policy_case(2, 20, 700, torch.float32, g)
    X, grad = torch.zeros((2, 16), device=DEV), torch.empty_like(c["z"])
    want = policy_want(c, 0.0, ref=False)
    with handle(X, 2, 1) as m:
        stats, logp = m.policy_loss(c["z"], c["tokens"], c["old"], c["adv"], c["w"], clip_low=0.2, clip_high=0.3, grad=grad)
        m.sync()
    close(grad, want[0], want[3] + TINY)
    close(stats, want[1], want[4] + TINY)
    assert not stats[:, 1].any()


def test_policy_gradient_is_the_losss_slope():
    """The loss along a line, five points: the central difference of two steps, extrapolated, against <gradient, direction>."""
    g = rng(4)
    N, T, V = 2, 6, 40
    c = policy_case(N, T, V, torch.float32, g)
    X, grad, line = torch.zeros((N, 16), device=DEV), torch.empty_like(c["z"]), normal((N, T, V), torch.float32, g)
    args = dict(ref_logp=c["ref"], clip_low=8.0, clip_high=8.0, kl_coef=0.2)     # no kink on the way
    with handle(X, 2, 1) as m:
        m.policy_loss(c["z"], c["tokens"], c["old"], c["adv"], c["w"], grad=grad, **args)

        def loss(h):
            s, _ = m.policy_loss(c["z"] + h * line, c["tokens"], c["old"], c["adv"], c["w"], grad=torch.empty_like(grad), **args)
            m.sync()
            return s[:, 0].double()
        h = 2.0 ** -5
        near, far = (loss(h) - loss(-h)) / (2 * h), (loss(2 * h) - loss(-2 * h)) / (4 * h)
    slope = (grad.double() * line.double()).sum((1, 2))
    # what the extrapolation leaves is h^4 times a fifth derivative: of terms w (|A| r + kl e) that move by up to 2 |line| per unit
    _, _, _, _, off, _ = policy_want(c, 0.2, 8.0, 8.0)
    lp = c["z"].double().log_softmax(-1).gather(2, c["tokens"].long()[..., None])[..., 0]
    size = (c["w"].double() * (c["adv"].double().abs() * (lp - c["old"].double()).exp() + 0.2 * (c["ref"].double() - lp).exp())).sum(1)
    reach = 2.0 * float(line.abs().max())
    bound = 2.0 * off[:, 0] / h + size * 4.0 * h ** 4 / 120.0 * reach ** 5 * 52.0       # (52: ways to take five derivatives of an exponential of a function)
    assert ((near + (near - far) / 3.0 - slope).abs() <= bound).all()


def test_logits_beyond_32_bits_of_offset():
    N, T, V = 4, 6_000, 100_000                                      # 2.4e9 logits
    z = torch.zeros((N, T, V), dtype=torch.bfloat16, device=DEV)
    g = rng(8)
    last = policy_case(1, 2, V, torch.bfloat16, g)
    z[-1, -2:] = last["z"][0]
    c = {k: torch.zeros((N, T), device=DEV) for k in ("old", "ref", "adv", "w")}
    tokens = torch.zeros((N, T), dtype=torch.int32, device=DEV)
    for k in c:
        c[k][-1, -2:] = last[k][0]
    tokens[-1, -2:] = last["tokens"][0]
    last["w"] = last["w"] + 0.25
    c["w"][-1, -2:] = last["w"][0]
    X = torch.zeros((N, 16), device=DEV)
    with handle(X, 2, 2) as m:
        stats, logp = m.policy_loss(z, tokens, c["old"], c["adv"], c["w"], ref_logp=c["ref"], clip_low=0.2, clip_high=0.3, kl_coef=0.1)
        m.sync()
    want = policy_want(last, 0.1)
    close(z[-1:, -2:], want[0], want[3] + 2.0 ** -8 * want[0].abs() * 1.01 + TINY)
    close(stats[-1:], want[1], want[4] + TINY)
    assert not stats[:-1].any() and not z[:-1].any()


# ---- use ------------------------------------------------------------------------------

def test_on_another_stream_and_in_a_graph():
    """Everything is queued on the bound stream, and a captured step replays with new inputs."""
    g = rng(7)
    N, T, V, D, I = 4, 200, 300, 64, 96
    X, G = normal((N, V * D + V * I), torch.float32, g), torch.zeros((N, V * D + V * I), device=DEV)
    tokens = some_tokens("any", N, T, V, g)
    x, z = normal((N, T, I), torch.float32, g), normal((N, T, V), torch.float32, g)
    old, adv, w = (torch.rand((N, T), generator=g, device=DEV) for _ in range(3))
    grad = torch.empty_like(z)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with binding.Moshpit(N, X.shape[1], 2, 2, binding.F32) as m, torch.cuda.stream(side):
        m.bind_state(X, side)
        out = torch.empty((N, T, D), device=DEV)

        def step():
            m.embed(tokens, 0, V, D, out=out)
            codes, scales = m.checkpoint(x)
            stats, logp = m.policy_loss(z, tokens, old, adv, w, grad=grad)
            m.weight_grad(grad, codes, scales, G, V * D)
            m.embed_grad(out, tokens, G, 0, V)
            return stats, logp, codes
        step()
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            held = step()
        for k in range(3):
            x.normal_(generator=g)
            z.normal_(generator=g)
            X.normal_(generator=g)
            G.fill_(9.0)
            graph.replay()
            side.synchronize()
            replayed = [t.clone() for t in (G, out, grad, *held)]
            G.fill_(9.0)
            eager = step()
            side.synchronize()
            for a, b in zip(replayed, (G, out, grad, *eager)):
                assert torch.equal(a, b), k


def test_new_tensors_belong_to_the_bound_stream():
    """Called with another stream current, the operators' new tensors are not out of blocks that stream still uses: here
    a block that a long queue of its work reads after it was freed."""
    g = rng(12)
    N, T, W = 4, 256, 1_024
    X, x = torch.zeros((N, 16), device=DEV), normal((N, T, W), torch.float32, g)
    big = normal((4_096, 4_096), torch.float32, g)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with binding.Moshpit(N, 16, 2, 2, binding.F32) as m:
        m.bind_state(X, side)
        want, scales = m.checkpoint(x)
        value = m.checkpoint_restore(want, scales)
        m.sync()                                                      # (the clones are the current stream's)
        want, value = want.clone(), value.clone()
        torch.cuda.synchronize()
        for _ in range(10):
            big = (big @ big).clamp_(-1, 1)
        held = value.clone()                                          # queued behind the products
        total = held.double().sum()
        del held                                                      # its block is free to this stream, and still to be read
        out = m.checkpoint_restore(want, scales)
        m.sync()
        assert torch.equal(out, value)
        torch.cuda.synchronize()
        assert float(total) == float(value.double().sum())
        assert torch.equal(out, value)


def test_refusals():
    X = torch.zeros((4, 1_000), device=DEV)
    G = torch.zeros_like(X)
    tokens = torch.zeros((4, 8), dtype=torch.int32, device=DEV)
    y, z = torch.zeros((4, 8, 10), device=DEV), torch.zeros((4, 8, 30), device=DEV)
    v = torch.zeros((4, 8), device=DEV)
    with binding.Moshpit(4, 1_000, 2, 2, binding.F32) as m:
        with pytest.raises(binding.MoshpitError, match="no state bound"):
            m.embed(tokens, 0, 100, 10)
        m.bind_state(X)
        for column, vocab, width in ((-1, 10, 10), (0, 101, 10), (901, 10, 10), (0, 0, 10), (0, 10, 0)):
            with pytest.raises((binding.MoshpitError, ValueError)):
                m.embed(tokens, column, vocab, width)
        for bad in (tokens.long(), tokens[:, ::2], tokens[:3], tokens.cpu()):
            with pytest.raises(ValueError):
                m.embed(bad, 0, 10, 10)
        with pytest.raises(ValueError):
            m.embed_grad(y.half(), tokens, G, 0, 100)
        with pytest.raises(ValueError):
            m.embed_grad(y.transpose(1, 2), tokens, G, 0, 100)
        with pytest.raises(ValueError):
            m.embed_grad(y, tokens, G.bfloat16(), 0, 100)
        with pytest.raises(binding.MoshpitError, match="do not fit"):
            m.embed_grad(y, tokens, G, 1, 100)
        codes, scales = m.checkpoint(y)
        with pytest.raises(ValueError):
            m.checkpoint_restore(codes, scales[:, :4])
        with pytest.raises(ValueError):
            m.weight_grad(y[:, :7], codes, scales, G, 0)
        with pytest.raises(binding.MoshpitError, match="do not fit"):
            m.weight_grad(y, codes, scales, G, 901)
        with pytest.raises(binding.MoshpitError, match="KL term"):
            m.policy_loss(z, tokens, v, v, v, kl_coef=0.1)
        with pytest.raises(binding.MoshpitError, match="clip range"):
            m.policy_loss(z, tokens, v, v, v, clip_low=math.nan)
        with pytest.raises(binding.MoshpitError, match="KL coefficient"):
            m.policy_loss(z, tokens, v, v, v, ref_logp=v, kl_coef=math.inf)
        with pytest.raises(ValueError):
            m.policy_loss(z, tokens, v, v, v, grad=z.bfloat16())
        with pytest.raises(ValueError):
            m.policy_loss(z, tokens, v.double(), v, v)
        m.sync()
    lib = binding.load_library()
    assert lib.moshpit_embed(None, 0, 1, 1, None, 0, 1.0, None, 0, 1) == -1
    assert not X.any() and not G.any() and not z.any()
