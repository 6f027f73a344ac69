"""Root-mean-square norms, their backward pass and dropout against plain forms in 64 bits.  Bounds follow from the operations (U = 2^-24 of a
result for each of binary32).  A norm's sum of squares: a thread adds up at most 32 elements of a row that registers hold and width / 1024 of a
longer one, then 6 steps over lanes and 15 over waves follow, all of positive terms."""
import math

import numpy as np
import pytest
import torch

from paper_2103_03239_amd import binding
from test_gpu_local_ops import DEV, TINY, TYPES, U, close, handle, normal, rng, rows

pytestmark = pytest.mark.gpu


def depth(W):
    return 64 + W / 1024


def gains(N, column, W, state, g, after=3):
    return normal((N, column + W + after), torch.float32, g, 0.3).add_(1.0).to(TYPES[state][0])


def normed(h, gain, eps):
    """x^ and y of rows h [N, T, W] and gains [N, W], binary64."""
    unit = h / (h.square().mean(-1, keepdim=True) + eps).sqrt()
    return unit, unit * gain[:, None]


def f32(x):
    return float(np.float32(x))


# one token to many, rows of one element to rows that registers do not hold, every number of threads a row takes
SHAPES = [(2, 1, 1, 1, 0, 0), (2, 2, 1, 512, 0, 0), (2, 1, 5, 7, 3, 1), (3, 2, 33, 100, 1, 0), (2, 1, 40, 130, 2, 3), (2, 1, 70, 256, 0, 0), (3, 3, 77, 1_003, 7, 5),
          (2, 1, 130, 520, 1, 2), (2, 1, 9, 2_048, 0, 8), (2, 1, 300, 4_096, 0, 0), (2, 2, 3, 4_097, 1, 1), (2, 1, 5, 8_192, 0, 0), (2, 1, 3, 16_384, 0, 0),
          (2, 1, 5, 16_385, 3, 1), (2, 1, 2, 40_000, 0, 0), (4, 2, 1_025, 64, 0, 0), (2, 1, 0, 33, 0, 0)]


@pytest.mark.parametrize("state,act", [("f32", "f32"), ("f32", "bf16"), ("bf16", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("M,d,T,W,column,pad", SHAPES)
def test_norm(state, act, M, d, T, W, column, pad):
    N, g, eps = M ** d, rng(T + W), 1e-5
    X = gains(N, column, W, state, g)
    x = rows(N, T, W, TYPES[act][0], g, pad, pad % 2, 3.0)
    r = rows(N, T, W, TYPES[act][0], g, pad, pad % 2)
    if T > 2:
        x[0, 1], r[0, 1] = 0.0, 0.0                                  # a row of zeros
        r[1, 2] = -x[1, 2]
    out, total = (rows(N, T, W, TYPES[act][0], g, pad, pad % 2) for _ in range(2))
    fences = [v._base.clone() for v in (out, total)]
    with handle(X, M, d) as m:
        print("norm", state, act, N, T, W, column, pad, flush=True)
        y0, h0, s0 = m.norm(x, column, eps=eps)
        y1, h1, s1 = m.norm(x, column, residual=r, eps=eps, saved=True, out=out, total=total)
        y2, h2, s2 = m.norm(x, column, residual=r, eps=eps)
        again = m.checkpoint(y1)
        m.sync()
    assert h0 is x and s0 is None and s2 is None and y1 is out and h1 is total
    assert torch.equal(y1, y2) and torch.equal(h1, h2)
    assert torch.equal(s1[0], again[0]) and torch.equal(s1[1], again[1])         # the 8-bit form of what is stored
    gain = X[:, column: column + W].double()
    for y, h in ((y0, x.double()), (y1, x.double() + r.double())):
        _, want = normed(h, gain, f32(eps))
        # h U (its own rounding, once in the element and within the squares'), squares and their sum, mean and eps 3, root 2, three products
        close(y, want, ((depth(W) + 6) / 2 + 7) * U * want.abs() + TYPES[act][2] * want.abs() * 1.01 + TINY)
    close(h1, x.double() + r.double(), (U + TYPES[act][2]) * (x.double() + r.double()).abs() * 1.01 + TINY)
    for v, fence in zip((out, total), fences):                                    # nothing beside the rows was written
        v.copy_(fence[pad % 2:].view(N, T, W + pad)[..., :W])
        assert torch.equal(v._base, fence)


@pytest.mark.parametrize("state,act", [("f32", "f32"), ("f32", "bf16"), ("bf16", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("M,d,T,W,column,pad", SHAPES)
@pytest.mark.parametrize("residual,accumulate", [(False, False), (True, True)])
def test_norm_grad(state, act, M, d, T, W, column, pad, residual, accumulate):
    N, g, eps = M ** d, rng(T + W), 1e-5
    X = gains(N, column, W, state, g)
    G = normal(X.shape, X.dtype, g)
    before = G.clone()
    x, dY, dt, out = (rows(N, T, W, TYPES[act][0], g, pad, pad % 2, s) for s in (3.0, 0.1, 0.1, 1.0))
    if T > 2:
        x[0, 1] = 0.0
    fence = out._base.clone()
    with handle(X, M, d) as m:
        print("norm_grad", state, act, N, T, W, column, pad, residual, accumulate, flush=True)
        got = m.norm_grad(dY, x, G, column, eps=eps, dtotal=dt if residual else None, accumulate=accumulate, out=out)
        m.sync()
        first, dx = G.clone(), out.clone()
        G.copy_(before)
        m.norm_grad(dY, x, G, column, eps=eps, dtotal=dt if residual else None, accumulate=accumulate, out=out)
        m.sync()
    assert got is out and torch.equal(first, G) and torch.equal(dx, out)          # repeats to the bit
    gain, h, dy = X[:, column: column + W].double(), x.double(), dY.double()
    unit, _ = normed(h, gain, f32(eps))
    inverse = (h.square().mean(-1, keepdim=True) + f32(eps)).rsqrt()
    u, k = dy * gain[:, None], depth(W)
    mean, size = (u * unit).mean(-1, keepdim=True), (u * unit).abs().mean(-1, keepdim=True)
    want = inverse * (u - unit * mean) + (dt.double() if residual else 0.0)
    slack = inverse * ((k / 2 + 12) * U * u.abs() + (2 * k + 24) * U * unit.abs() * size) + U * (want.abs() + (dt.double().abs() if residual else 0.0))
    close(dx, want, slack * 1.01 + TYPES[act][2] * want.abs() * 1.01 + TINY)
    want, size = (dy * unit).sum(1), (dy * unit).abs().sum(1)
    if accumulate:
        old = before[:, column: column + W].double()
        want, size = want + old, size + old.abs()
    close(G[:, column: column + W], want, (T + k / 2 + 12) * U * size + TYPES[state][2] * want.abs() * 1.01 + TINY)
    G[:, column: column + W] = before[:, column: column + W]
    assert torch.equal(G, before)                                                 # nothing beside the gain was written
    out.copy_(fence[pad % 2:].view(N, T, W + pad)[..., :W])
    assert torch.equal(out._base, fence)


def test_norm_grad_against_differences():
    """Central differences of <y, dY> + <h, dt> along directions of x and of the gain, the norm taken in 64 bits at the operator's results."""
    g = rng(4)
    N, T, W = 4, 9, 96
    X, x, dY, dt = normal((N, W), torch.float32, g), normal((N, T, W), torch.float32, g), normal((N, T, W), torch.float32, g), normal((N, T, W), torch.float32, g)
    G = torch.zeros_like(X)
    with handle(X, 2, 2) as m:
        dx = m.norm_grad(dY, x, G, 0, dtotal=dt)
        m.sync()
    ex, eg, step = normal(x.shape, torch.float32, g).double(), normal(X.shape, torch.float32, g).double(), 2.0 ** -10

    def value(s):
        h = x.double() + s * ex
        return (normed(h, X.double() + s * eg, f32(1e-6))[1] * dY.double()).sum() + (h * dt.double()).sum()
    slope = (value(step) - value(-step)) / (2 * step)
    got = (dx.double() * ex).sum() + (G.double() * eg).sum()
    size = (dx.double() * ex).abs().sum() + (G.double() * eg).abs().sum()
    # the differences' own error: step^2 / 6 of the third derivative, which for a norm of W = 96 is within a few times the slopes' size
    assert abs(float(slope - got)) <= (step ** 2 * 4 + 200 * U) * float(size)


@pytest.mark.parametrize("act", ["f32", "bf16"])
@pytest.mark.parametrize("W", [40, 1_000, 3_000, 20_000])
def test_norms_of_large_small_and_spoilt_rows(act, W):
    """Rows whose squares pass binary32 or vanish in it, and rows with an infinity or a NaN, which stay by themselves."""
    g, T = rng(W), 8
    X = gains(2, 0, W, "f32", g)
    x, dY = normal((2, T, W), TYPES[act][0], g), normal((2, T, W), TYPES[act][0], g)
    x[:, 1] *= 1e25
    x[:, 2] *= 1e-25
    x[:, 3, W // 2] = math.inf
    x[:, 4, W - 1] = math.nan
    x[:, 5] *= 2.0 ** 64
    G = torch.zeros_like(X)
    with handle(X, 2, 1) as m:
        y, _, (codes, scales) = m.norm(x, 0, saved=True)
        dx = m.norm_grad(dY, x, G, 0)
        again = m.checkpoint(y)
        m.sync()
    gain, h = X[:, :W].double(), x.double()
    unit, want = normed(h, gain, f32(1e-6))
    good = torch.tensor([0, 1, 2, 5, 6, 7], device=DEV)
    k = depth(W)
    close(y[:, good], want[:, good], ((k + 6) / 2 + 9) * U * want[:, good].abs() + TYPES[act][2] * want[:, good].abs() * 1.01 + TINY)
    u = dY.double() * gain[:, None]
    inverse = (h.square().mean(-1, keepdim=True) + f32(1e-6)).rsqrt()
    grad = inverse * (u - unit * (u * unit).mean(-1, keepdim=True))
    size = inverse * ((k / 2 + 14) * U * u.abs() + (2 * k + 28) * U * unit.abs() * (u * unit).abs().mean(-1, keepdim=True)) + (U + TYPES[act][2]) * grad.abs()
    close(dx[:, good], grad[:, good], size[:, good] * 1.01 + TINY)
    assert torch.isnan(y[:, 4]).all() and torch.isnan(dx[:, 4]).all()
    assert torch.isnan(y[:, 3, W // 2]).all() and not torch.isfinite(dx[:, 3]).all()
    assert torch.equal(again[0], codes) and torch.equal(again[1], scales)
    assert not torch.isfinite(G[:, :W]).all()                                     # the sum takes every row


def test_norms_in_place():
    g = rng(11)
    for act, W in (("f32", 200), ("bf16", 1_000), ("bf16", 20_000)):
        X = gains(2, 0, W, "f32", g)
        x, r, dY, dt = (normal((2, 6, W), TYPES[act][0], g) for _ in range(4))
        G, G2 = torch.zeros_like(X), torch.zeros_like(X)
        with handle(X, 2, 1) as m:
            y, h, _ = m.norm(x, 0, residual=r)
            a, b = x.clone(), r.clone()
            m.norm(a, 0, residual=b, out=a, total=b)
            m.sync()
            assert torch.equal(a, y) and torch.equal(b, h)
            a, b = x.clone(), r.clone()
            m.norm(a, 0, residual=b, out=b, total=a)
            m.sync()
            assert torch.equal(b, y) and torch.equal(a, h)
            dx = m.norm_grad(dY, h, G, 0, dtotal=dt)
            for k in range(3):
                place = [dY.clone(), h.clone(), dt.clone()]
                m.norm_grad(place[0], place[1], G2, 0, dtotal=place[2], out=place[k])
                m.sync()
                assert torch.equal(place[k], dx) and torch.equal(G, G2)


# ---- dropout ------------------------------------------------------------------

def kept(rows, W, p, seed, step):
    """The mask from its definition, in whole numbers."""
    mask = (1 << 64) - 1

    def mix(x):
        x ^= x >> 32
        x = x * 0x9E3779B97F4A7C15 & mask
        x ^= x >> 29
        x = x * 0x6A09E667F3BCC909 & mask
        return x ^ x >> 32
    cut = math.floor(p * 65536 + 0.5)
    base = mix(seed + 0xE7037ED1A0B428DB * (step + 1) & mask)
    out = np.zeros((len(rows), W), bool)
    for n, row in enumerate(rows):
        key = mix(base + 0x8EBC6AF09C88C6E3 * (row + 1) & mask)
        for c in range(0, W, 4):
            word = mix(key ^ c // 4)
            for k in range(min(4, W - c)):
                out[n, c + k] = (word >> 16 * k & 0xffff) >= cut
    return out, 65536.0 / (65536 - cut)


@pytest.mark.parametrize("act", ["f32", "bf16"])
@pytest.mark.parametrize("M,d,T,W,pad,p,seed,step", [
    (2, 1, 1, 1, 0, 0.5, 0, None), (2, 2, 1, 512, 0, 0.1, 7, 0), (2, 1, 5, 7, 1, 0.3, 1 << 63, 5), (3, 2, 33, 100, 0, 0.9, (1 << 64) - 1, (1 << 62) + 3),
    (2, 1, 40, 1_003, 3, 0.0, 3, 1), (2, 1, 3, 5_000, 0, 1e-6, 3, -1), (2, 1, 9, 33, 0, 65_535 / 65_536, 12, 2), (2, 1, 0, 5, 0, 0.5, 1, None), (4, 2, 100, 8, 8, 0.25, 9, 4),
])
@pytest.mark.parametrize("residual", [False, True])
def test_dropout(act, M, d, T, W, pad, p, seed, step, residual):
    N, g = M ** d, rng(T + W)
    X = torch.zeros((N, 8), device=DEV)
    x, r, out = (rows(N, T, W, TYPES[act][0], g, pad, pad % 2) for _ in range(3))
    fence = out._base.clone()
    s = None if step is None else torch.tensor([step], dtype=torch.int64, device=DEV)
    keep, factor = kept(range(N * T), W, p, seed, 0 if step is None else step)
    keep = torch.from_numpy(keep).view(N, T, W).to(DEV)
    x[~keep] = math.nan                                                           # what is dropped may be anything
    with handle(X, M, d) as m:
        print("dropout", act, N, T, W, pad, p, seed, step, residual, flush=True)
        assert m.dropout(x, p, seed, step=s, residual=r if residual else None, out=out) is out
        new = m.dropout(x, p, seed, step=s, residual=r if residual else None)
        place = x.clone()
        m.dropout(place, p, seed, step=s, residual=r.contiguous() if residual else None, out=place)
        m.sync()
    assert torch.equal(out, new) and torch.equal(out, place)
    term = torch.where(keep, x.double() * factor, 0.0)
    want = term + (r.double() if residual else 0.0)
    close(out, want, 3 * U * (term.abs() + want.abs()) + TYPES[act][2] * want.abs() * 1.01 + TINY)
    assert torch.equal(out[~keep], r[~keep] if residual else torch.zeros_like(out[~keep]))
    out.copy_(fence[pad % 2:].view(N, T, W + pad)[..., :W])
    assert torch.equal(out._base, fence)


def test_dropout_far_into_many_rows():
    """Elements beyond 2^32 of the matrix's start, the mask of a few rows there."""
    N, T, W = 2, 300_000, 8_192
    X = torch.zeros((N, 8), device=DEV)
    x = torch.ones((N, T, W), dtype=torch.bfloat16, device=DEV)
    with handle(X, 2, 1) as m:
        m.dropout(x, 0.5, 77, out=x)
        m.sync()
    for n in (0, 262_145, 2 * T - 1):
        keep, _ = kept([n], W, 0.5, 77, 0)
        assert np.array_equal((x.view(-1, W)[n] == 2.0).cpu().numpy(), keep[0])


def test_dropout_is_even_and_unlike_from_seed_to_seed():
    """Shares of kept elements by column of four, by row and in all, and of agreement between seeds, steps and neighbouring rows: each within six
    standard deviations of independent draws."""
    N, T, W, p = 4, 256, 1_024, 0.25
    X, x = torch.zeros((N, 8), device=DEV), torch.ones((N, T, W), device=DEV)
    with handle(X, 2, 2) as m:
        a, b = (m.dropout(x, p, seed) != 0 for seed in (1, 2))
        c = m.dropout(x, p, 1, step=torch.ones(1, dtype=torch.int64, device=DEV)) != 0
        m.sync()
    q = 1 - p
    same = q * q + p * p

    def near(v, share):
        n = v.numel()
        assert abs(float(v.double().mean()) - share) <= 6 * math.sqrt(share * (1 - share) / n)
    near(a, q)
    for k in range(4):
        near(a[..., k::4], q)
    share = a.double().mean(2)
    assert float((share - q).abs().max()) <= 6 * math.sqrt(q * p / W)
    for other in (b, c):
        near(a == other, same)
    near(a[:, 1:] == a[:, :-1], same)
    near(a[..., 1:] == a[..., :-1], same)
    near(a[1:] == a[:-1], same)


def test_dropout_replayed_with_another_step():
    """A captured call reads the step when it runs; norms beside it, with eager work between the replays."""
    N, T, W = 4, 50, 96
    g = rng(8)
    X, x, r, dY = gains(N, 0, W, "f32", g), normal((N, T, W), torch.bfloat16, g), normal((N, T, W), torch.bfloat16, g), normal((N, T, W), torch.bfloat16, g)
    G, step = torch.zeros_like(X), torch.zeros(1, dtype=torch.int64, device=DEV)
    total, y, dx = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream), handle(X, 2, 2) as m:
        def pass_():
            m.dropout(x, 0.2, 5, step=step, residual=r, out=total)
            m.norm(total, 0, out=y)
            m.norm_grad(dY, total, G, 0, out=dx)
        pass_()
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            pass_()
        seen = []
        for k in (0, 1, 2, 1):
            step.fill_(k)
            for v in (total, y, dx, G):
                v.fill_(7.0)
            graph.replay()
            stream.synchronize()
            got = [v.clone() for v in (total, y, dx, G)]
            pass_()                                                               # the eager result, the handle's workspace used in between
            m.norm_grad(dY[:, : 1].contiguous(), total[:, : 1].contiguous(), torch.empty_like(G), 0)
            stream.synchronize()
            for a, b in zip(got, (total, y, dx, G)):
                assert torch.equal(a[..., :W], b[..., :W])
            seen.append(got[0])
        assert torch.equal(seen[1], seen[3]) and not torch.equal(seen[0], seen[1]) and not torch.equal(seen[1], seen[2])


def test_refusals():
    g = rng(1)
    X = gains(2, 4, 32, "f32", g, after=0)
    x = normal((2, 3, 32), torch.float32, g)
    G = torch.zeros_like(X)
    with binding.Moshpit(2, 36, 2, 1, binding.F32) as m:
        with pytest.raises(binding.MoshpitError, match="no state bound"):
            m.norm(x, 0)
    with handle(X, 2, 1) as m:
        for call in (lambda: m.norm(x, 5), lambda: m.norm(x, -1), lambda: m.norm_grad(x, x, G, 5)):
            with pytest.raises(binding.MoshpitError, match="do not fit"):
                call()
        for eps in (-1e-6, math.nan, math.inf):
            with pytest.raises(binding.MoshpitError, match="eps"):
                m.norm(x, 0, eps=eps)
            with pytest.raises(binding.MoshpitError, match="eps"):
                m.norm_grad(x, x, G, 0, eps=eps)
        for p in (-0.1, 1.0, math.nan):
            with pytest.raises(binding.MoshpitError, match="probability"):
                m.dropout(x, p, 1)
        with pytest.raises(binding.MoshpitError, match="drops everything"):
            m.dropout(x, 1 - 2.0 ** -18, 1)
        for call in (lambda: m.norm(x, 0, residual=x.bfloat16()), lambda: m.norm(x, 0, out=x[..., :31]), lambda: m.norm(x, 0, total=x),
                     lambda: m.norm(x[:1], 0), lambda: m.norm(x.half(), 0), lambda: m.norm_grad(x, x[:, :2], G, 0), lambda: m.norm_grad(x, x, G[:, :5], 0),
                     lambda: m.dropout(x, 0.1, -1), lambda: m.dropout(x, 0.1, 1 << 64), lambda: m.dropout(x, 0.1, 1, step=torch.zeros(2, dtype=torch.int64, device=DEV)),
                     lambda: m.dropout(x, 0.1, 1, step=torch.zeros(1, device=DEV)), lambda: m.dropout(x, 0.1, 1, out=x.bfloat16())):
            with pytest.raises(ValueError):
                call()


def test_places_of_other_strides():
    """A result that begins where an input does, by another stride, would be written over rows that are not yet read."""
    g = rng(2)
    X = gains(2, 4, 32, "f32", g, after=0)
    G, flat = torch.zeros_like(X), normal((2 * 3 * 64,), torch.float32, g)
    x, close_by = flat.as_strided((2, 3, 32), (3 * 64, 64, 1)), flat.as_strided((2, 3, 32), (3 * 32, 32, 1))
    y = normal((2, 3, 32), torch.float32, g)
    with handle(X, 2, 1) as m:
        for call in (lambda: m.norm(x, 0, out=close_by), lambda: m.norm(y, 0, residual=x, out=close_by), lambda: m.norm(x, 0, residual=y, total=close_by),
                     lambda: m.norm_grad(x, y, G, 0, out=close_by), lambda: m.norm_grad(y, x, G, 0, out=close_by), lambda: m.norm_grad(y, y, G, 0, dtotal=x, out=close_by),
                     lambda: m.dropout(x, 0.1, 1, out=close_by), lambda: m.dropout(y, 0.1, 1, residual=x, out=close_by)):
            with pytest.raises(binding.MoshpitError, match="only with its row stride"):
                call()
        with pytest.raises(binding.MoshpitError, match="cannot take the place"):
            m.norm(x, 0, residual=y, out=x, total=x)
