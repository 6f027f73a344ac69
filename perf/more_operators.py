"""The operators of a transformer block in a peer's local step, as timed cases.

The peers of this framework are rows of one matrix X, their gradients rows of a matrix G like it.  When they are
transformers, these operators lie between the token embeddings and the loss, for all N peers at once:

  norm       root-mean-square norm of x + residual with the gain that lies in the peer's row of X; the output also in 8 bits,
             as the weight gradients take it
  norm_grad  its backward pass: the input's gradient, and the gain's into the rows of G
  dropout    out = residual + dropout(x), the mask from a counter-based generator
  attention  causal attention over packed sequences with grouped heads
  train      the same and its backward pass
  cached     new tokens of sequences against the keys and values of the tokens before them
"""
import math
import types

import numpy as np
import torch

own = False

DEV = "cuda:0"
DTYPES = {"f32": (torch.float32, 4), "bf16": (torch.bfloat16, 2)}
GROUP = 32                         # elements that share a scale in the 8-bit form
EPS = 1e-6


def listed():
    return [
        # 16 peers generate, one token each: launch latency
        dict(name="norm_single_bf16", op="norm", M=4, d=2, T=1, width=512, state="bf16", act="bf16", before=1_000, after=24, residual=True, saved=False),
        # 16 peers, 4096 tokens of a wide layer each, the output saved in 8 bits for the backward pass
        dict(name="norm_16_bf16", op="norm", M=4, d=2, T=4_096, width=4_096, state="f32", act="bf16", before=0, after=0, residual=True, saved=True),
        # 27 small peers of odd sizes, one short sequence each
        dict(name="norm_grad_odd_f32", op="norm_grad", M=3, d=3, T=77, width=1_003, state="f32", act="f32", before=7, after=5, residual=False),
        # the backward pass of norm_16_bf16
        dict(name="norm_grad_16_bf16", op="norm_grad", M=4, d=2, T=4_096, width=4_096, state="f32", act="bf16", before=0, after=0, residual=True),
        # a few rows of odd length
        dict(name="dropout_small_f32", op="dropout", M=2, d=2, T=3, width=1_003, act="f32", p=0.1, residual=False),
        # after a wide layer of 16 peers, onto the residual stream
        dict(name="dropout_16_bf16", op="dropout", M=4, d=2, T=4_096, width=4_096, act="bf16", p=0.1, residual=True),
        # 27 small peers, short packed sequences, an odd head width
        dict(name="attention_small_f32", op="attention", M=3, d=3, T=77, heads=3, group=3, depth=20, act="f32", docs=4, window=0),
        # 2 peers with long documents
        dict(name="attention_long_bf16", op="attention", M=2, d=1, T=8_192, heads=16, group=4, depth=128, act="bf16", docs=2, window=0),
        # 4 peers in binary32, packed sequences of odd lengths
        dict(name="train_4_f32", op="train", M=2, d=2, T=1_500, heads=8, group=2, depth=80, act="f32", docs=5, window=0),
        # 16 peers, 8 sequences each
        dict(name="train_16_bf16", op="train", M=4, d=2, T=4_096, heads=8, group=2, depth=64, act="bf16", docs=8, window=0),
        # 16 peers generate, one token of one sequence each, a short prompt: latency
        dict(name="cached_single_bf16", op="cached", M=4, d=2, seqs=1, new=1, cap=300, heads=8, group=4, depth=64, act="bf16"),
        # 4 peers, 8 sequences of up to 16384 tokens each
        dict(name="cached_long_bf16", op="cached", M=2, d=2, seqs=8, new=1, cap=16_384, heads=16, group=4, depth=128, act="bf16"),
    ]


def _spread(rng, low, high):
    """A whole number, even over its logarithm."""
    return int(round(math.exp(rng.uniform(math.log(low), math.log(max(low, high))))))


def _tokens(rng, most):
    """From one to `most`; the long ones, where the time goes, as often as all."""
    return _spread(rng, rng.choice([1, max(1, most / 10)]), max(2, most))


def _others(rng):
    """Parameters before and after the ones that the operator is about: as a rule they keep the rows on 256-byte boundaries."""
    return rng.choice([dict(before=0, after=0), dict(before=128, after=1_024), dict(before=rng.randint(1, 999), after=rng.randint(0, 99))])


def draw(rng):
    op = rng.choice(["norm", "norm_grad", "dropout", "attention", "attention", "train", "train", "cached", "cached"])
    M, d = rng.choice([(2, 1), (2, 2), (3, 2), (4, 2), (3, 3), (8, 2)])
    N = M ** d
    case = dict(op=op, M=M, d=d, act=rng.choice(["f32", "bf16", "bf16"]))
    if op in ("norm", "norm_grad", "dropout"):
        width = _spread(rng, 16, 20_000)
        if rng.random() < 0.6:
            width = max(64, width // 64 * 64)
        case.update(width=width, T=_tokens(rng, min(65_536, 1.2e8 / N / width)), residual=rng.random() < 0.6)
        if op == "dropout":
            case["p"] = rng.choice([0.1, 0.1, 0.05, 0.5, 0.0])
        else:
            case.update(state=rng.choice(["f32", "bf16"]), **_others(rng))
        if op == "norm":
            case["saved"] = rng.random() < 0.7
        return case
    group = rng.choice([1, 2, 4, 8])
    case.update(group=group, heads=group * rng.choice([1, 2, 3, 4] if group < 8 else [1, 2]),
                depth=rng.choice([32, 64, 64, 64, 80, 96, 128, 128, 128, 192, 256, rng.randint(5, 140)]))
    if op == "cached":
        case.update(seqs=_spread(rng, 1, 40), new=rng.choice([1, 1, 1, 1, 2, 5]))
        row = case["heads"] // group * case["depth"] * DTYPES[case["act"]][1]
        # (the plain form compares every query with every key of its peer)
        cap = min(16_384, 4e8 / N / case["seqs"] / row, 1e9 / N / (case["seqs"] ** 2 * case["new"] * case["heads"]))
        case["cap"] = _tokens(rng, cap)
        return case
    pairs = 1.2e9 if op == "attention" else 6e8
    if case["act"] == "f32":
        pairs /= 4
    T = _tokens(rng, min(8_192, (pairs * 128 / max(128, case["depth"]) / N / case["heads"]) ** 0.5))
    case.update(T=T, docs=_spread(rng, 1, max(1, min(60, T // 8))), window=rng.choice([0, 0, 0, rng.randint(1, 500)]))
    return case


# ---- inputs -----------------------------------------------------------------

def _rng(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _normal(shape, dtype, g, scale=1.0):
    return torch.empty(shape, dtype=dtype, device=DEV).normal_(0.0, scale, generator=g)


def _activations(case, g):
    """[N, T, width], some channels larger than others."""
    x = _normal((case["M"] ** case["d"], case["T"], case["width"]), DTYPES[case["act"]][0], g)
    return x.mul_(torch.empty(case["width"], device=DEV).normal_(0.0, 0.5, generator=g).exp_())


def _first(case, g):
    """Where the sequence of every place begins (a window: where the part of it that the place sees), -1 behind the last sequence."""
    N, T = case["M"] ** case["d"], case["T"]
    t = torch.arange(T, device=DEV).expand(N, T).contiguous()
    cuts = torch.randint(0, T, (N, case["docs"]), generator=g, device=DEV)
    cuts[:, 0] = 0
    cuts = cuts.sort(1).values
    first = cuts.gather(1, torch.searchsorted(cuts, t, right=True) - 1)
    if case["window"]:
        first = torch.maximum(first, t - case["window"] + 1)
    if T >= 8:
        first[t >= torch.randint(T - T // 8, T + 1, (N, 1), generator=g, device=DEV)] = -1
    return first.int()


def prepare(case, seed):
    s = types.SimpleNamespace(case=case)
    g = _rng(seed)
    op, N = case["op"], case["M"] ** case["d"]
    state, act = DTYPES[case.get("state", "f32")][0], DTYPES[case["act"]][0]
    if op in ("norm", "norm_grad", "dropout"):
        s.x = _activations(case, g)
        shape = s.x.shape
        s.residual = _normal(shape, act, g) if case["residual"] else None
        if op == "dropout":
            s.seed, s.step, s.out = seed, torch.full((1,), 3, dtype=torch.int64, device=DEV), torch.empty_like(s.x)
        else:
            s.X = _normal((N, case["before"] + case["width"] + case["after"]), torch.float32, g, 0.2).add_(1.0).to(state)
        if op == "norm":
            s.out = torch.empty_like(s.x)
            s.total = torch.empty_like(s.x) if case["residual"] else None
        elif op == "norm_grad":
            s.dY, s.dX, s.G = _normal(shape, act, g, 1e-2), torch.empty_like(s.x), torch.zeros_like(s.X)
    else:
        kv, D = case["heads"] // case["group"], case["depth"]
        rows = case["T"] if op != "cached" else case["seqs"] * case["new"]
        keys = case["T"] if op != "cached" else case["seqs"] * case["cap"]
        s.scale = D ** -0.5
        s.q = _normal((N, rows, case["heads"] * D), act, g, 1.5)
        s.k, s.v = _normal((N, keys, kv * D), act, g), _normal((N, keys, kv * D), act, g)
        s.out = torch.empty_like(s.q)
        if op == "cached":
            begin = torch.arange(case["seqs"], device=DEV) * case["cap"]
            n = torch.randint(max(1, case["cap"] // 2), case["cap"] + 1, (N, case["seqs"]), generator=g, device=DEV)
            if case["seqs"] >= 8:
                n[:, -1] = 0                                       # a slot that is free
            s.spans = torch.stack([begin.expand(N, -1), begin + n], 2).int().contiguous()
        else:
            s.first = _first(case, g)
        if op == "train":
            s.dout = _normal(s.q.shape, act, g, 1e-2)
            s.dq, s.dk, s.dv = torch.empty_like(s.q), torch.empty_like(s.k), torch.empty_like(s.v)
    if own:
        from paper_2103_03239_amd import binding
        if not hasattr(s, "X"):
            s.X = torch.zeros((N, 64), dtype=state, device=DEV)
        s.handle = binding.Moshpit(N, s.X.shape[1], case["M"], case["d"], binding.F32 if state == torch.float32 else binding.BF16)
        s.handle.bind_state(s.X)
    return s


# ---- one pass ---------------------------------------------------------------

def _own(s):
    case, h, op = s.case, s.handle, s.case["op"]
    if op == "norm":
        y, total, saved = h.norm(s.x, case["before"], residual=s.residual, eps=EPS, saved=case["saved"], out=s.out, total=s.total)
        got = {"y": y}
        if case["residual"]:
            got["total"] = total
        if case["saved"]:
            got["saved"] = h.checkpoint_restore(*saved, dtype=torch.bfloat16)
        return got
    if op == "norm_grad":
        dx = h.norm_grad(s.dY, s.x, s.G, case["before"], eps=EPS, dtotal=s.residual, out=s.dX)
        return {"dx": dx, "gain": s.G[:, case["before"]: case["before"] + case["width"]]}
    if op == "dropout":
        return {"out": h.dropout(s.x, case["p"], s.seed, step=s.step, residual=s.residual, out=s.out)}
    kv = case["heads"] // case["group"]
    if op == "cached":
        return {"out": h.attention_cached(s.q, s.k, s.v, s.spans, case["heads"], kv, scale=s.scale, out=s.out)}
    out, lse = h.attention(s.q, s.k, s.v, s.first, case["heads"], kv, scale=s.scale, out=s.out)
    if op == "attention":
        return {"out": out, "lse": lse}
    dq, dk, dv = h.attention_grad(s.dout, s.q, s.k, s.v, out, lse, s.first, case["heads"], kv, scale=s.scale, dq=s.dq, dk=s.dk, dv=s.dv)
    return {"out": out, "dq": dq, "dk": dk, "dv": dv}


def _power(e):
    """2^e in binary32 for whole -126 <= e <= 127."""
    return ((e + 127) << 23).view(torch.float32)


def _in_8_bits(x):
    """What the 8-bit form of x [..., width] stands for: groups of 32 of a row, codes x / 2^e rounded to even, e the smallest
    whole number (-126 or more) with which no code passes 127."""
    W = x.shape[-1]
    x = torch.nn.functional.pad(x.float(), (0, -W % GROUP)).unflatten(-1, (-1, GROUP))
    most = x.abs().amax(-1)
    e = (torch.frexp(most).exponent - 7).clamp(-126, 127)
    e = torch.where((most * _power(-e)).round() > 127, e + 1, e)
    e = torch.where(most == 0, torch.full_like(e, -126), e)
    return ((x * _power(-e)[..., None]).round() * _power(e)[..., None]).flatten(-2)[..., :W]


def _gain(X, case):
    return X[:, None, case["before"]: case["before"] + case["width"]]


def _plain_norm(s):
    case = s.case
    h = s.x.float() if s.residual is None else s.x.float() + s.residual.float()
    s.out.copy_(h * torch.rsqrt(h.square().mean(-1, keepdim=True) + EPS) * _gain(s.X, case).float())
    got = {"y": s.out}
    if case["residual"]:
        got["total"] = s.total.copy_(h)
    if case["saved"]:
        got["saved"] = _in_8_bits(s.out).bfloat16()
    return got


def _plain_norm_grad(s):
    case, h, dy = s.case, s.x.float(), s.dY.float()
    r = torch.rsqrt(h.square().mean(-1, keepdim=True) + EPS)
    u = dy * _gain(s.X, case).float()
    dx = r * (u - h * (r * r * (u * h).mean(-1, keepdim=True)))
    s.dX.copy_(dx if s.residual is None else dx + s.residual.float())
    gain = s.G[:, case["before"]: case["before"] + case["width"]]
    gain.copy_((dy * h * r).sum(1))
    return {"dx": s.dX, "gain": gain}


def _signed(k):
    return k - (1 << 64) if k >= 1 << 63 else k


def _mix(x):
    """The library's mixer on the bits of 64-bit integers."""
    x = (x ^ (x >> 32 & 0xffffffff)) * _signed(0x9E3779B97F4A7C15)
    x = (x ^ (x >> 29 & 0x7ffffffff)) * _signed(0x6A09E667F3BCC909)
    return x ^ (x >> 32 & 0xffffffff)


def _dropped(case, seed, step):
    """Which elements a mask leaves out, [N, T, width], and the factor of the others."""
    N, T, W = case["M"] ** case["d"], case["T"], case["width"]
    cut = math.floor(case["p"] * 65536 + 0.5)
    base = _mix(_signed(seed) + _signed(0xE7037ED1A0B428DB) * (step + 1))
    key = _mix(base + _signed(0x8EBC6AF09C88C6E3) * (torch.arange(N * T, device=DEV) + 1))
    word = _mix(key[:, None] ^ torch.arange(-(-W // 4), device=DEV))
    bits = torch.stack([word >> 16 * k & 0xffff for k in range(4)], -1).view(N, T, -1)[..., :W]
    return bits < cut, 65536.0 / (65536 - cut)


def _plain_dropout(s):
    gone, factor = _dropped(s.case, s.seed, s.step)
    y = torch.where(gone, 0.0, s.x.float() * factor)
    return {"out": s.out.copy_(y if s.residual is None else y + s.residual.float())}


def _heads(x, n):
    """[N, rows, n * depth] -> [N, n, rows, depth] in binary32."""
    return x.float().unflatten(2, (n, -1)).transpose(1, 2).contiguous()


def _rows(x):
    return x.transpose(1, 2).flatten(2)


def _softmax(s, q, seen):
    """Per head: queries, keys and values in binary32, the weights and log-sums of the keys that are seen; rows that see none have weights 0."""
    case = s.case
    q = _heads(q, case["heads"])
    k, v = (_heads(x, case["heads"] // case["group"]).repeat_interleave(case["group"], 1) for x in (s.k, s.v))
    z = (torch.matmul(q, k.transpose(2, 3)) * s.scale).masked_fill_(~seen[:, None], -math.inf)
    some = seen.any(-1)[:, None, :, None]
    top = torch.where(some, z.amax(-1, keepdim=True), 0.0)
    z.sub_(top).exp_()
    total = torch.where(some, z.sum(-1, keepdim=True), 1.0)
    return q, k, v, z.div_(total), (top + total.log())[..., 0]


def _plain_attention(s):
    case, t = s.case, torch.arange(s.first.shape[1], device=DEV)
    live = s.first >= 0
    seen = (t >= s.first[:, :, None]) & (t <= t[:, None]) & live[:, :, None] & live[:, None, :]
    q, k, v, p, lse = _softmax(s, s.q, seen)
    out = torch.matmul(p, v)
    s.out.copy_(_rows(out))
    if case["op"] == "attention":
        return {"out": s.out, "lse": lse}
    do = _heads(s.dout, case["heads"])
    dv = torch.matmul(p.transpose(2, 3), do)
    ds = torch.matmul(do, v.transpose(2, 3)).sub_((do * out).sum(-1, keepdim=True)).mul_(p).mul_(s.scale)
    dq, dk = torch.matmul(ds, k), torch.matmul(ds.transpose(2, 3), q)
    s.dq.copy_(_rows(dq))
    s.dk.copy_(_rows(dk.unflatten(1, (-1, case["group"])).sum(2)))
    s.dv.copy_(_rows(dv.unflatten(1, (-1, case["group"])).sum(2)))
    return {"out": s.out, "dq": s.dq, "dk": s.dk, "dv": s.dv}


def _plain_cached(s):
    case, j = s.case, torch.arange(s.k.shape[1], device=DEV)
    begin, end = (s.spans[:, :, c].repeat_interleave(case["new"], 1)[:, :, None] for c in (0, 1))
    later = case["new"] - 1 - torch.arange(s.q.shape[1], device=DEV)[:, None] % case["new"]       # new tokens behind this one
    _, _, v, p, _ = _softmax(s, s.q, (j >= begin) & (j < end - later))
    return {"out": s.out.copy_(_rows(torch.matmul(p, v)))}


PLAIN = {"norm": _plain_norm, "norm_grad": _plain_norm_grad, "dropout": _plain_dropout, "attention": _plain_attention, "train": _plain_attention,
         "cached": _plain_cached}


def run(s):
    return _own(s) if own else PLAIN[s.case["op"]](s)


# ---- what a pass cannot do without ------------------------------------------

def work(case):
    op, N = case["op"], case["M"] ** case["d"]
    act = DTYPES[case["act"]][1]
    if op in ("norm", "norm_grad", "dropout"):
        T, W = case["T"], case["width"]
        arrays = {"norm": 2, "norm_grad": 3, "dropout": 2}[op] + ((2 if op == "norm" else 1) if case["residual"] else 0)
        a_row = arrays * W * act
        if case.get("saved"):
            a_row += 2 * (W + -(-W // GROUP)) + 2 * W                # written; read and restored in bfloat16
        state = DTYPES[case["state"]][1] if "state" in case else 0
        return {"bytes": N * (T * a_row + (2.0 if op == "norm_grad" else 1.0) * W * state), "flops": {"norm": 6.0, "norm_grad": 12.0, "dropout": 2.0}[op] * N * T * W}
    H, D = case["heads"], case["depth"]
    kv = H // case["group"]
    if op == "cached":
        keys = N * case["seqs"] * 0.75 * case["cap"] * (1.0 - 1.0 / case["seqs"] if case["seqs"] >= 8 else 1.0)
        return {"bytes": act * D * (2.0 * kv * keys + 2.0 * H * N * case["seqs"] * case["new"]), "flops": 4.0 * D * H * keys * case["new"]}
    T = case["T"]
    held = 0.94 * T if T >= 8 else T
    pairs = held * (held / (case["docs"] + 1.0) if case["docs"] > 1 else held / 2.0) + held / 2.0
    if case["window"]:
        pairs = min(pairs, held * case["window"])
    rows = N * T * D * act
    if op == "attention":
        return {"bytes": rows * (2.0 * H + 2.0 * kv) + 4.0 * N * T * H, "flops": 4.0 * D * N * H * pairs}
    return {"bytes": rows * (5.0 * H + 6.0 * kv), "flops": 14.0 * D * N * H * pairs}     # (out is written and read, q, k and v are read twice: two calls)


# ---- the same results in 64 bits --------------------------------------------

def _whole_power(e):
    """2^e in binary64 to the bit, which a power function need not give."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def exact(case, seed):
    s = prepare(case, seed)
    op, N = case["op"], case["M"] ** case["d"]
    f64 = torch.float64
    if op in ("norm", "norm_grad", "dropout"):
        T, W = case["T"], case["width"]
    if op == "dropout":
        cut = int(case["p"] * 65536 + 0.5)

        def mixed(x):                                              # (numpy's 64-bit integers without signs)
            x ^= x >> np.uint64(32)
            x *= np.uint64(0x9E3779B97F4A7C15)
            x ^= x >> np.uint64(29)
            x *= np.uint64(0x6A09E667F3BCC909)
            x ^= x >> np.uint64(32)
            return x
        base = mixed(np.array([(seed + 0xE7037ED1A0B428DB * 4) % 2 ** 64], dtype=np.uint64))
        key = mixed(base + np.uint64(0x8EBC6AF09C88C6E3) * np.arange(1, N * T + 1, dtype=np.uint64))
        word = mixed(key[:, None] ^ np.arange((W + 3) // 4, dtype=np.uint64))
        keep = torch.from_numpy(word.view(np.uint16).reshape(N, T, -1)[..., :W] >= cut).to(DEV)
        out = torch.where(keep, s.x.double() * (65536.0 / (65536 - cut)), 0.0)
        return {"out": out if s.residual is None else out + s.residual.double()}
    if op == "norm":
        y, total, saved = (torch.empty(s.x.shape, dtype=f64, device=DEV) for _ in range(3))
        for i in range(N):
            h = s.x[i].double() + (0.0 if s.residual is None else s.residual[i].double())
            total[i] = h
            y[i] = h / torch.sqrt((h * h).sum(1, keepdim=True) / W + EPS) * s.X[i, case["before"]:][:W].double()
            if case["saved"]:
                stored = y[i].to(s.x.dtype).double()
                for a in range(0, W, GROUP):
                    x = stored[:, a: a + GROUP]
                    most = x.abs().amax(1, keepdim=True)
                    e = torch.floor(torch.log2(most.clamp(min=2.0 ** -119))).long() - 7      # at or below the right one
                    for _ in range(3):
                        e = torch.where(torch.round(most / _whole_power(e)) > 127.0, e + 1, e)
                    saved[i][:, a: a + GROUP] = torch.round(x / _whole_power(e)) * _whole_power(e)
        got = {"y": y}
        if case["residual"]:
            got["total"] = total
        if case["saved"]:
            got["saved"] = saved
        return got
    if op == "norm_grad":
        dx = torch.empty(s.x.shape, dtype=f64, device=DEV)
        gain = torch.empty((N, W), dtype=f64, device=DEV)
        for i in range(N):
            h, dy, w = s.x[i].double(), s.dY[i].double(), s.X[i, case["before"]:][:W].double()
            size = torch.sqrt((h * h).sum(1, keepdim=True) / W + EPS)
            gain[i] = (dy * h / size).sum(0)
            u = dy * w / size
            dx[i] = u - h * ((u * h).sum(1, keepdim=True) / W) / size ** 2 + (0.0 if s.residual is None else s.residual[i].double())
        return {"dx": dx, "gain": gain}
    H, D, group = case["heads"], case["depth"], case["group"]
    out = torch.zeros(s.q.shape, dtype=f64, device=DEV)
    if op == "cached":
        spans, new = s.spans.tolist(), case["new"]
        for i in range(N):
            for a, (begin, end) in enumerate(spans[i]):
                k, v = (x[i, begin: end].double().view(-1, H // group, D) for x in (s.k, s.v))
                for b in range(new):
                    n = end - begin - (new - 1 - b)
                    if n <= 0:
                        continue
                    q = s.q[i, a * new + b].double().view(H // group, group, D)
                    p = torch.softmax(s.scale * torch.matmul(q, k[:n].permute(1, 2, 0).contiguous()), -1)
                    out[i, a * new + b] = torch.matmul(p, v[:n].permute(1, 0, 2).contiguous()).flatten()
        return {"out": out}
    T = case["T"]
    lse = torch.zeros((N, H, T), dtype=f64, device=DEV)
    dq, dk, dv = torch.zeros_like(out), torch.zeros(s.k.shape, dtype=f64, device=DEV), torch.zeros(s.k.shape, dtype=f64, device=DEV)
    t = torch.arange(T, device=DEV)
    for i in range(N):
        live = (s.first[i] >= 0).nonzero()[:, 0]
        hidden = (t[live] < s.first[i, live][:, None]) | (t[live] > live[:, None])
        for a in range(H):
            b = a // group
            q, k, v = s.q[i, live, a * D: a * D + D].double(), s.k[i, live, b * D: b * D + D].double(), s.v[i, live, b * D: b * D + D].double()
            z = (q @ k.t().contiguous() * s.scale).masked_fill(hidden, -math.inf)
            lse[i, a, live] = torch.logsumexp(z, 1)
            p = torch.exp(z - lse[i, a, live][:, None])
            out[i, live, a * D: a * D + D] = p @ v
            if op == "train":
                do = s.dout[i, live, a * D: a * D + D].double()
                dp = do @ v.t().contiguous()
                dz = p * (dp - (p * dp).sum(1, keepdim=True)) * s.scale
                dq[i, live, a * D: a * D + D] = dz @ k
                dk[i, live, b * D: b * D + D] += dz.t().contiguous() @ q
                dv[i, live, b * D: b * D + D] += p.t().contiguous() @ do
    return {"out": out, "lse": lse} if op == "attention" else {"out": out, "dq": dq, "dk": dk, "dv": dv}
