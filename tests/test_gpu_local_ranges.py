"""The local step's operators over the whole range of their values: masks of the type's lowest value, common offsets, saved groups at
the top of the range.  Bounds follow from the operations as in test_gpu_local_ops.py; a binary32 operation is off by U = 2^-24 of its result."""
import math

import pytest
import torch

from test_gpu_local_ops import DEV, TINY, TYPES, U, close, handle, normal, rng, rows

pytestmark = pytest.mark.gpu


# ---- policy loss ------------------------------------------------------------------

def loss_inputs(z, tokens, g):
    """Old and reference log-probabilities around the policy's, advantages and weights; off the kinks by more than rounding."""
    lp = z.double().log_softmax(-1).gather(2, tokens.long()[..., None])[..., 0]
    ratio = torch.empty(lp.shape, device=DEV).normal_(0, 0.3, generator=g).exp_()
    for edge in (0.8, 1.3):
        ratio = torch.where((ratio / edge - 1).abs() < 2e-3, ratio * 1.01, ratio)
    return {"z": z, "tokens": tokens, "old": (lp - ratio.log()).float(), "ref": (lp + torch.empty(lp.shape, device=DEV).normal_(0, 0.4, generator=g)).float(),
            "adv": torch.empty(lp.shape, device=DEV).normal_(generator=g), "w": 0.25 + torch.rand(lp.shape, generator=g, device=DEV)}


def loss_want(c, kl):
    """In binary64: gradient, stats, lp, and how far binary32 may be off each where a row's largest value is taken from every value first.  Then
    z - m, its product with log2 e and exp2 are off by U (m - z), U (m - z) and 2 U, the sum of n terms by n U, and the log-probability
    (z_a - m) - log sum by what its terms are, whatever m is."""
    z, tok = c["z"].double(), c["tokens"].long()[..., None]
    V = z.shape[2]
    m, z_a = z.amax(-1), z.gather(2, tok)[..., 0]
    above = torch.logsumexp(z - m[..., None], -1)
    lp = (z_a - m) - above
    p = (z - m[..., None] - above[..., None]).exp()
    d = torch.where(p == 0.0, 0.0, m[..., None] - z)
    w, A, old, rf = (c[k].double() for k in ("w", "adv", "old", "ref"))
    low, high = 1.0 - float(torch.tensor(0.2)), 1.0 + float(torch.tensor(0.3))
    kl = float(torch.tensor(kl))
    r, e = (lp - old).exp(), (rf - lp).exp()
    gain, held, k = A * r, A * r.clamp(low, high), e - (rf - lp) - 1
    clipped = gain > held
    loss = w * (kl * k - torch.minimum(gain, held))
    slope = w * (kl * (1 - e) - torch.where(clipped, torch.zeros_like(gain), gain))
    grad = -slope[..., None] * p
    grad.scatter_add_(2, tok, slope[..., None])
    n = max(128, V / 256) + 32
    s_off = U * (n + 4 + 3 * (p * d).sum(-1))
    lp_off = 4 * U * ((m - z_a) + above + lp.abs()) + s_off
    r_off, e_off = lp_off + U * (lp.abs() + old.abs() + 4), lp_off + U * (lp.abs() + rf.abs() + 4)
    slope_off = w * (abs(kl) * (e * e_off + 2 * U * (1 + e)) + gain.abs() * (r_off + 4 * U)) + 4 * U * slope.abs()
    k_off = w * (e * e_off + lp_off + 4 * U * (e + (rf - lp).abs() + 1))
    loss_off = abs(kl) * k_off + w * gain.abs() * (r_off + 4 * U) + 4 * U * loss.abs()
    grad_off = slope_off[..., None] * (p + torch.zeros_like(p).scatter_(2, tok, 1.0)) + slope.abs()[..., None] * p * (U * (3 * d + 8) + s_off[..., None]) \
        + 2 * U * grad.abs()
    wk, wc = w * k, torch.where(clipped, w, 0.0)
    off = torch.stack([loss_off.sum(1) + 2 * U * loss.abs().sum(1), k_off.sum(1) + 2 * U * wk.abs().sum(1), 2 * U * wc.sum(1)], 1)
    return grad, torch.stack([loss.sum(1), wk.sum(1), wc.sum(1)], 1), lp, grad_off, off, lp_off


def check_loss(c, act, kl, M, d):
    X = torch.zeros((M ** d, 16), device=DEV)
    grad = torch.full_like(c["z"], 7.0)
    want = loss_want(c, kl)
    with handle(X, M, d) as m:
        scored = m.token_logp(c["z"], c["tokens"])
        stats, logp = m.policy_loss(c["z"], c["tokens"], c["old"], c["adv"], c["w"], ref_logp=c["ref"], clip_low=0.2, clip_high=0.3, kl_coef=kl, grad=grad)
        m.sync()
    close(scored, want[2], want[5])
    close(logp, want[2], want[5])
    close(stats, want[1], want[4] + TINY)
    close(grad, want[0], want[3] + TYPES[act][2] * want[0].abs() * 1.01 + TINY)


# rows by 64 .. 1024 threads, in slices, many short ones, many that one block each scores
LOGITS = [(10, 2), (10, 7), (10, 512), (10, 3_000), (10, 6_000), (10, 12_000), (10, 24_000), (10, 50_001), (10, 100_000), (8, 140_003), (2_100, 300), (2_100, 512), (600, 6_001)]


@pytest.mark.parametrize("act", ["f32", "bf16"])
@pytest.mark.parametrize("T,V", LOGITS)
def test_masks_of_the_types_lowest_value(act, T, V):
    """Excluded tokens as the type's lowest value: most of a row, all but its token, its first or last part, all of it (every token alike),
    and beside -inf."""
    g, dtype = rng(T + V), TYPES[act][0]
    low = torch.finfo(dtype).min
    z = rows(2, T, V, dtype, g, scale=2.0).contiguous()
    tokens = torch.randint(0, V, (2, T), generator=g, device=DEV, dtype=torch.int32)
    at, kind = torch.arange(V, device=DEV), torch.arange(T, device=DEV) % 6
    few = torch.rand((2, T, V), generator=g, device=DEV) < 100.0 / V
    masked = torch.stack([~few, torch.ones_like(few), (at < V * 3 // 4).expand_as(few), (at >= V - 16).expand_as(few), torch.ones_like(few), torch.ones_like(few)])
    masked = masked[kind, :, torch.arange(T, device=DEV)].transpose(0, 1)
    masked = masked.scatter(2, tokens.long()[..., None], ((kind == 4) | (kind == 5))[None, :, None].expand(2, T, 1))
    z[masked] = low
    z.masked_fill_((kind == 5)[None, :, None] & (at % 3 == 0) & (at != tokens[..., None]), -math.inf)
    print("lowest", act, T, V, flush=True)
    check_loss(loss_inputs(z, tokens, g), act, 0.1, 2, 1)


@pytest.mark.parametrize("act", ["f32", "bf16"])
@pytest.mark.parametrize("T,V", LOGITS)
@pytest.mark.parametrize("offset", [1_024.0, -16_384.0])
def test_an_offset_common_to_a_row_is_no_error(act, T, V, offset):
    """The loss does not change when a row's logits move together: nor do its errors, however far."""
    g, dtype = rng(T + V), TYPES[act][0]
    spacing = 2.0 ** -7 * abs(offset) if act == "bf16" else 0.25
    z = (offset - spacing * torch.randint(0, 3 if act == "bf16" else 40, (2, T, V), generator=g, device=DEV)).to(dtype)
    tokens = torch.randint(0, V, (2, T), generator=g, device=DEV, dtype=torch.int32)
    c = loss_inputs(z, tokens, g)
    print("offset", act, T, V, offset, flush=True)
    check_loss(c, act, 0.1, 2, 1)


# ---- weight gradients -------------------------------------------------------------

@pytest.mark.parametrize("state,act", [("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16")])
@pytest.mark.parametrize("M,d,T,O,I", [(2, 1, 50, 3, 40), (2, 1, 100, 24, 70), (2, 1, 700, 128, 128), (8, 2, 65, 392, 400), (4, 2, 40, 1_001, 1_003)])
def test_weight_grad_of_every_power_of_two(state, act, M, d, T, O, I):
    """Codes count as code * 2^e for every scale byte whose values are finite, up to the largest: groups of 2^122 and of codes -1 .. 1 of 2^127
    beside small ones."""
    N, g = M ** d, rng(T + O + I)
    X, G = torch.zeros((N, O * I), dtype=TYPES[state][0], device=DEV), torch.zeros((N, O * I), dtype=TYPES[state][0], device=DEV)
    dY = rows(N, T, O, TYPES[act][0], g, scale=2.0 ** -60).contiguous()
    groups = -(-I // 32)
    codes = torch.randint(-127, 128, (N, T, I), generator=g, device=DEV)
    byte = torch.tensor([1, 100, 127, 200, 246, 247, 248, 249, 254], device=DEV)[torch.randint(0, 9, (N, T, groups), generator=g, device=DEV)]
    wide = byte.repeat_interleave(32, -1)[..., :I]
    codes = torch.where(wide == 249, codes.clamp(-63, 63), torch.where(wide == 254, codes.clamp(-1, 1), codes))
    value = codes.double() * torch.exp2(wide.double() - 127.0)
    assert float(value.abs().max()) <= torch.finfo(torch.float32).max
    with handle(X, M, d) as m:
        print("powers", state, act, N, T, O, I, flush=True)
        m.weight_grad(dY, codes.to(torch.int8), byte.to(torch.uint8), G, 0)
        back = m.checkpoint_restore(codes.to(torch.int8), byte.to(torch.uint8))
        m.sync()
    assert torch.equal(back.double(), value)
    y = dY.double().transpose(1, 2).contiguous()
    want, size = torch.bmm(y, value), torch.bmm(y.abs(), value.abs())
    terms = 3 * T if act == "f32" else T
    close(G.view(N, O, I), want, (terms + 8) * 2 * U * size + TYPES[state][2] * want.abs() * 1.01 + TINY)


# ---- checkpoints ------------------------------------------------------------------

@pytest.mark.parametrize("act", ["f32", "bf16"])
@pytest.mark.parametrize("T,W", [(40, 32), (7, 100), (3, 1_003)])
def test_checkpoint_of_the_largest_values(act, T, W):
    """Finite elements restore as finite ones, in both types: by the definition with e at most 121 and codes of at most 127, so that elements from
    127.5 * 2^121 on are off by up to a step and all others by half of one."""
    g, dtype = rng(T + W), TYPES[act][0]
    top = torch.finfo(dtype).max
    x = normal((4, T, W), dtype, g, 2.0 ** 126).clamp_(-top, top)
    x[0], x[1] = -top, normal((T, W), dtype, g, 2.0 ** 100)
    x[1, :, ::32] = top
    edge = [127.5 * 2.0 ** 121, 127.5 * 2.0 ** 121 * (1 - 2.0 ** -24 * 2), 127.25 * 2.0 ** 121, 127.0 * 2.0 ** 121, 126.5 * 2.0 ** 121, 126.0 * 2.0 ** 121, top, 127.5 * 2.0 ** 120]
    for t in range(T):                                               # a row for each, the group's largest element, beside small ones
        x[2, t] = normal((W,), dtype, g, 2.0 ** 110)
        x[2, t, ::32] = min(edge[t % len(edge)], top) * (-1) ** t
    with handle(torch.zeros((4, 8), device=DEV), 2, 2) as m:
        print("largest", act, T, W, flush=True)
        codes, scales = m.checkpoint(x)
        back, narrow = m.checkpoint_restore(codes, scales), m.checkpoint_restore(codes, scales, dtype=torch.bfloat16)
        m.sync()
    v = torch.nn.functional.pad(x.double(), (0, -W % 32)).unflatten(-1, (-1, 32))
    e = torch.full(v.shape[:-1], -126.0, dtype=torch.float64, device=DEV)
    for k in range(-125, 122):
        e = torch.where((v.abs().amax(-1) * 2.0 ** (1 - k)).round() > 127.0, float(k), e)
    step = torch.exp2(e)[..., None]
    q = (v / step).round().clamp(-127, 127)
    assert torch.equal(scales.double(), e + 127.0)
    assert torch.equal(codes.double(), q.flatten(-2)[..., :W])
    want = (q * step).flatten(-2)[..., :W]
    assert torch.equal(back.double(), want) and torch.equal(narrow.double(), want) and bool(torch.isfinite(narrow).all())
    off, step = (want - x.double()).abs(), step.expand_as(v).flatten(-2)[..., :W]
    assert bool((off <= torch.where(x.double().abs() >= 127.5 * 2.0 ** 121, step, 0.5 * step)).all())


@pytest.mark.parametrize("act", ["f32", "bf16"])
@pytest.mark.parametrize("M,d,V", [(8, 4, 2), (16, 2, 2), (16, 2, 70_002)])
def test_kl_term_near_the_reference(act, M, d, V):
    """k = exp(x) - 1 - x and its slope for x = ref - lp down to 2^-16, relatively as exact as for large ones, and never negative.  Logits of 0 and -200
    give the second token the log-probability -200 to the bit (exp(-200) is far below a binary32 rounding of 1), and x is exact."""
    N, g, dtype = M ** d, rng(V + d), TYPES[act][0]
    z = torch.full((N, 1, V), -math.inf, dtype=dtype, device=DEV)
    z[..., 0], z[..., 1] = 0.0, -200.0
    x = torch.exp2(torch.empty((N, 1), device=DEV).uniform_(-16.0, 2.5, generator=g)) * torch.randint(0, 2, (N, 1), generator=g, device=DEV).mul(2).sub(1)
    x = (x * 2.0 ** 16).round().div(2.0 ** 16)
    x[0], x[1], x[2], x[3], x[4] = 0.0, 0.5, -0.5, 2.0 ** -16, -2.0 ** -16
    tokens, v, grad = torch.ones((N, 1), dtype=torch.int32, device=DEV), torch.full((N, 1), -200.0, device=DEV), torch.empty_like(z)
    with handle(torch.zeros((N, 16), device=DEV), M, d) as m:
        print("near", act, N, V, flush=True)
        stats, logp = m.policy_loss(z, tokens, v, torch.zeros_like(v), torch.ones_like(v), ref_logp=v + x, kl_coef=1.0, grad=grad)
        m.sync()
    assert bool((logp == -200.0).all()) and torch.equal((v + x) - v, x)
    y = x.double()[:, 0]
    e1 = torch.expm1(y)
    terms = [y ** n / math.factorial(n) for n in range(2, 20)]       # (taken for |y| < 1: the rest is below 2^-53 of the sum)
    k = torch.where(y.abs() < 1.0, sum(terms), e1 - y)
    # within 1/2 a series: squares, sums and products, 8 U of it at most; beyond, expm1 (2 U) less x, each up to 4.5 times the result: 12 U
    close(stats[:, 1], k, 12 * U * k)
    close(stats[:, 0], k, 13 * U * k)
    assert bool((stats[:, 1] >= 0).all()) and float(stats[0, 1]) == 0.0
    for j, want in ((0, e1), (1, -e1)):
        close(grad[:, 0, j], want, (6 * U + TYPES[act][2]) * want.abs())
    assert not grad[..., 2:].any()


@pytest.mark.parametrize("act", ["f32", "bf16"])
@pytest.mark.parametrize("T,V", [(10, 300), (10, 100_000), (1, 300), (2_100, 300)])
def test_kl_as_a_statistic_does_not_reach_the_gradient(act, T, V):
    """With a coefficient of 0 loss and gradient are those without a reference, whatever the reference holds; the statistic tells."""
    g, dtype = rng(T + V), TYPES[act][0]
    c = loss_inputs(rows(4, T, V, dtype, g), torch.randint(0, V, (4, T), generator=g, device=DEV, dtype=torch.int32), g)
    grad, plain = torch.empty_like(c["z"]), torch.empty_like(c["z"])
    c["ref"][1, 0], c["ref"][2, 0], c["ref"][3, 0] = c["ref"][1, 0] + 100.0, math.nan, -math.inf
    args = c["z"], c["tokens"], c["old"], c["adv"], c["w"]
    with handle(torch.zeros((4, 16), device=DEV), 2, 2) as m:
        stats, logp = m.policy_loss(*args, ref_logp=c["ref"], grad=grad)
        without, logp_without = m.policy_loss(*args, grad=plain)
        m.sync()
    assert torch.equal(grad, plain) and torch.equal(logp, logp_without) and torch.equal(stats[:, 0], without[:, 0]) and torch.equal(stats[:, 2], without[:, 2])
    assert bool(torch.isfinite(stats[:, 0]).all()) and bool(torch.isfinite(grad).all())
    assert math.isfinite(float(stats[0, 1])) and float(stats[1, 1]) == math.inf and math.isnan(float(stats[2, 1])) and float(stats[3, 1]) == math.inf
