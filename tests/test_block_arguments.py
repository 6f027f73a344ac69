"""What the binding hands to the library for the operators of a transformer block, and what it refuses: on the CPU, with tensors that say they
are on the GPU and a library that writes down its calls."""
import contextlib

import pytest
import torch

from test_local_step_arguments import Lent, Stream, gpu, peers  # noqa: F401  (a fixture)

N, W, H, K, D = 4, 64, 4, 2, 16


@pytest.fixture(autouse=True)
def new_tensors_on_the_gpu(monkeypatch):
    empty = torch.empty
    monkeypatch.setattr(torch, "empty", lambda *a, **k: gpu(empty(*a, **k)))


def rows(T, width, dtype=torch.float32):
    return gpu(torch.zeros((N, T, width), dtype=dtype))


def operators(m, T):
    """name -> call with x in the place of the matrix that is named, and the width that matrix has."""
    G, first, lse = gpu(torch.zeros((N, m.P))), gpu(torch.zeros((N, T), dtype=torch.int32)), gpu(torch.zeros((N, H, T)))
    spans = gpu(torch.zeros((N, max(T, 1), 2), dtype=torch.int32)) if T else gpu(torch.zeros((N, 0, 2), dtype=torch.int32))
    r, q, k = rows(T, W), rows(T, H * D), rows(T, K * D)
    return {
        "norm x": (lambda x: m.norm(x, 0), W), "norm residual": (lambda x: m.norm(r, 0, residual=x), W), "norm out": (lambda x: m.norm(r, 0, out=x), W),
        "norm total": (lambda x: m.norm(r, 0, residual=r, total=x), W), "norm_grad dY": (lambda x: m.norm_grad(x, r, G, 0), W),
        "norm_grad x": (lambda x: m.norm_grad(r, x, G, 0), W), "norm_grad dtotal": (lambda x: m.norm_grad(r, r, G, 0, dtotal=x), W),
        "norm_grad out": (lambda x: m.norm_grad(r, r, G, 0, out=x), W), "dropout x": (lambda x: m.dropout(x, 0.1, 1), W),
        "dropout residual": (lambda x: m.dropout(r, 0.1, 1, residual=x), W), "dropout out": (lambda x: m.dropout(r, 0.1, 1, out=x), W),
        "attention q": (lambda x: m.attention(x, k, k, first, H, K), H * D), "attention k": (lambda x: m.attention(q, x, k, first, H, K), K * D),
        "attention v": (lambda x: m.attention(q, k, x, first, H, K), K * D), "attention out": (lambda x: m.attention(q, k, k, first, H, K, out=x), H * D),
        "attention_grad dout": (lambda x: m.attention_grad(x, q, k, k, q, lse, first, H, K), H * D),
        "attention_grad out": (lambda x: m.attention_grad(q, q, k, k, x, lse, first, H, K), H * D),
        "attention_grad dq": (lambda x: m.attention_grad(q, q, k, k, q, lse, first, H, K, dq=x), H * D),
        "attention_grad dk": (lambda x: m.attention_grad(q, q, k, k, q, lse, first, H, K, dk=x), K * D),
        "attention_grad dv": (lambda x: m.attention_grad(q, q, k, k, q, lse, first, H, K, dv=x), K * D),
        "attention_cached q": (lambda x: m.attention_cached(x, k, k, spans, H, K), H * D),
        "attention_cached k": (lambda x: m.attention_cached(q, x, k, spans, H, K), K * D),
        "attention_cached out": (lambda x: m.attention_cached(q, k, k, spans, H, K, out=x), H * D),
    }


NAMES = ["norm x", "norm residual", "norm out", "norm total", "norm_grad dY", "norm_grad x", "norm_grad dtotal", "norm_grad out", "dropout x",
         "dropout residual", "dropout out", "attention q", "attention k", "attention v", "attention out", "attention_grad dout", "attention_grad out",
         "attention_grad dq", "attention_grad dk", "attention_grad dv", "attention_cached q", "attention_cached k", "attention_cached out"]


@pytest.mark.parametrize("name", NAMES)
def test_rows_of_single_tokens_that_share_memory_are_refused(peers, name):  # noqa: F811
    call, width = operators(peers, 1)[name]
    for x in (torch.zeros((1, 1, width)).expand(N, 1, width), torch.zeros(N * width).as_strided((N, 1, width), (width - 1, width, 1))):
        with pytest.raises(ValueError, match="constant distance"):
            call(gpu(x))
    assert not peers._lib.made


@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("T", [0, 1, 3])
def test_row_strides_reach_the_library(peers, name, T):  # noqa: F811
    call, width = operators(peers, T)[name]
    for x, stride in ((rows(T, width), width), (gpu(torch.zeros((N, T, width + 5)))[..., :width], width + 5)):
        peers._lib.made.clear()
        call(x)
        (_, args), = peers._lib.made
        if T:
            at = max(i for i, a in enumerate(args) if isinstance(a, int) and a == x.data_ptr())
            assert stride in args[at: at + 3], args


@pytest.mark.parametrize("name", NAMES)
def test_other_types_and_shapes_are_refused(peers, name):  # noqa: F811
    call, width = operators(peers, 3)[name]
    alone = name.split()[1] in ("x", "q") and not name.startswith("norm_grad")      # what the others are measured by
    for x in ([] if alone else [rows(3, width, torch.bfloat16), rows(2, width)]) + [rows(3, width).half(), torch.zeros((N, 3, width)), rows(3, width)[:2],
                                                                                rows(3, width)[0], rows(3, 2 * width)[..., ::2]]:
        if name == "attention_cached k" and x.shape[1:2] == (2,):
            continue                                                   # (a cache has rows of its own number, but v must have as many)
        with pytest.raises((ValueError, IndexError)):
            call(x)
    assert not peers._lib.made


def test_arguments_besides_matrices(peers):  # noqa: F811
    m, T = peers, 6
    q, k, first, r = rows(T, H * D), rows(T, K * D), gpu(torch.zeros((N, T), dtype=torch.int32)), rows(T, W)
    spans = gpu(torch.zeros((N, 3, 2), dtype=torch.int32))
    for call in (lambda: m.norm(r, 0, total=r), lambda: m.norm_grad(r, r, gpu(torch.zeros((N, 5))), 0), lambda: m.dropout(r, 0.1, -1), lambda: m.dropout(r, 0.1, 1 << 64),
                 lambda: m.dropout(r, 0.1, 1, step=gpu(torch.zeros(2, dtype=torch.int64))), lambda: m.dropout(r, 0.1, 1, step=gpu(torch.zeros(1))),
                 lambda: m.dropout(r, 0.1, 1, step=torch.zeros(1, dtype=torch.int64)), lambda: m.attention(q, k, k, first.long(), H, K),
                 lambda: m.attention(q, k, k, first[:, :5], H, K), lambda: m.attention(q, k, k, torch.zeros((N, T), dtype=torch.int32), H, K),
                 lambda: m.attention(q, k, k, first, 5, K), lambda: m.attention(q, k, k, first, 0, K), lambda: m.attention(q, k, k, first, H, 0), lambda: m.attention(q, k, k, first, H, H),
                 lambda: m.attention_grad(q, q, k, k, q, gpu(torch.zeros((N, H, 5))), first, H, K), lambda: m.attention_cached(q, k, k, spans[..., 0], H, K),
                 lambda: m.attention_cached(rows(5, H * D), k, k, spans, H, K), lambda: m.attention_cached(rows(0, H * D), k, k, spans, H, K),
                 lambda: m.attention_cached(q, k, k, spans.long(), H, K)):
        with pytest.raises(ValueError):
            call()
    assert not m._lib.made
    m.attention_cached(q, rows(11, K * D), rows(11, K * D), spans, H, K)
    (name, args), = m._lib.made
    assert name == "moshpit_attention_cached" and (3, 2, 11, H, K, D) == tuple(args[9:15])      # sequences, new tokens, keys, heads
    m._lib.made.clear()
    m.norm(r, 7, residual=r, saved=True)
    m.dropout(r, 0.25, (1 << 64) - 1, step=gpu(torch.zeros((), dtype=torch.int64)))
    (_, norm), (_, drop) = m._lib.made
    assert norm[6:9] == (T, 7, W) and all(norm[-2:]) and drop[6:10] == (T, W, 0.25, (1 << 64) - 1) and drop[10]


@pytest.mark.parametrize("away", [False, True])
def test_the_allocator_hears_of_the_stream_that_uses_a_tensor(peers, away, monkeypatch):  # noqa: F811
    """Every tensor of a call is lent to the bound stream where another one is current, and the new ones, which are the bound stream's, to the
    current one."""
    from paper_2103_03239_amd import binding
    bound, current, empty = Stream(7), Stream(5 if away else 7), torch.empty
    monkeypatch.setattr(binding, "_current_stream", lambda index: current.cuda_stream)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: current)
    monkeypatch.setattr(torch.cuda, "stream", lambda stream: contextlib.nullcontext())
    monkeypatch.setattr(torch, "empty", lambda *a, **k: empty(*a, **k).as_subclass(Lent))
    m, T = peers, 3
    m._state, m._bound = (m._state[0], bound), (0, bound.cuda_stream)

    def new(*shape, dtype=torch.float32):
        return torch.zeros(shape, dtype=dtype).as_subclass(Lent)

    def q():
        return new(N, T, H * D)

    def k():
        return new(N, T, K * D)

    def r():
        return new(N, T, W)

    def first():
        return new(N, T, dtype=torch.int32)
    for call, given in (
            (lambda x: m.norm(x, 0)[0], [r()]), (lambda x, y: m.norm(x, 0, residual=y, saved=True), [r(), r()]),
            (lambda x, y, o, t: (m.norm(x, 0, residual=y, out=o, total=t), ())[1], [r(), r(), r(), r()]),
            (lambda y, x, G, d: m.norm_grad(y, x, G, 0, dtotal=d), [r(), r(), new(N, m.P), r()]), (lambda y, x, G, o: (m.norm_grad(y, x, G, 0, out=o), ())[1], [r(), r(), new(N, m.P), r()]),
            (lambda x, s, y: m.dropout(x, 0.1, 1, step=s, residual=y), [r(), new(1, dtype=torch.int64), r()]), (lambda x, o: (m.dropout(x, 0.1, 1, out=o), ())[1], [r(), r()]),
            (lambda a, b, c, f: m.attention(a, b, c, f, H, K), [q(), k(), k(), first()]),
            (lambda a, b, c, f, o: m.attention(a, b, c, f, H, K, out=o)[1], [q(), k(), k(), first(), q()]),
            (lambda y, a, b, c, o, s, f: m.attention_grad(y, a, b, c, o, s, f, H, K), [q(), q(), k(), k(), q(), new(N, H, T), first()]),
            (lambda y, a, b, c, o, s, f, d: m.attention_grad(y, a, b, c, o, s, f, H, K, dk=d)[::2], [q(), q(), k(), k(), q(), new(N, H, T), first(), k()]),
            (lambda a, b, c, s: m.attention_cached(a, b, c, s, H, K), [q(), k(), k(), new(N, T, 2, dtype=torch.int32)])):
        made = call(*given)
        flat = [x for y in (made if isinstance(made, tuple) else [made]) for x in (y if isinstance(y, tuple) else [y])]
        made = [x for x in flat if isinstance(x, Lent) and not any(x is g for g in given)]
        for x in given:
            assert (bound in x.__dict__.get("lent", [])) == away
        for x in made:
            assert (current in x.__dict__.get("lent", [])) == away
