"""What the binding hands to the library for the local step's operators, and what it refuses: on the CPU, with tensors that
say they are on the GPU and a library that writes down its calls."""
import contextlib
import ctypes

import pytest
import torch

from paper_2103_03239_amd import binding


class OnGpu(torch.Tensor):
    is_cuda = True


def gpu(x):
    return x.as_subclass(OnGpu)


class Calls:
    """Every entry point succeeds; `made` holds their names and arguments."""

    def __init__(self):
        self.made = []

    def __getattr__(self, name):
        def call(*args):
            self.made.append((name, args))
            return 0
        return call


N, W, V = 4, 64, 10


@pytest.fixture
def peers():
    m = object.__new__(binding.Moshpit)
    m._lib, m._h, m._state = Calls(), ctypes.c_void_p(1), None
    m.N, m.P, m.M, m.d, m.dtype = N, 1_000, 2, 2, binding.F32
    m._state = (gpu(torch.zeros((N, m.P))), None)
    return m


def operators(m, T):
    """name -> call with x [N, T, W] in the place of the matrix that is named."""
    tokens = gpu(torch.zeros((N, T), dtype=torch.int32))
    v = gpu(torch.zeros((N, T)))
    G = gpu(torch.zeros((N, m.P)))
    codes, scales = gpu(torch.zeros((N, T, W), dtype=torch.int8)), gpu(torch.zeros((N, T, W // 32), dtype=torch.uint8))
    z = gpu(torch.zeros((N, T, W)))
    return {
        "embed out": lambda x: m.embed(tokens, 0, V, W, out=x),
        "embed_grad dY": lambda x: m.embed_grad(x, tokens, G, 0, V),
        "checkpoint x": lambda x: m.checkpoint(x),
        "checkpoint_restore out": lambda x: m.checkpoint_restore(codes, scales, out=x),
        "weight_grad dY": lambda x: m.weight_grad(x, codes, scales, G, 0),
        "token_logp logits": lambda x: m.token_logp(x, tokens),
        "policy_loss logits": lambda x: m.policy_loss(x, tokens, v, v, v),
        "policy_loss grad": lambda x: m.policy_loss(z, tokens, v, v, v, grad=x),
    }


NAMES = ["embed out", "embed_grad dY", "checkpoint x", "checkpoint_restore out", "weight_grad dY", "token_logp logits", "policy_loss logits",
         "policy_loss grad"]


@pytest.mark.parametrize("name", NAMES)
def test_rows_of_single_tokens_that_share_memory_are_refused(peers, name):
    """One row for all peers (stride 0), or rows closer than they are long, is no matrix [N][row stride]."""
    call = operators(peers, 1)[name]
    one = torch.zeros((1, 1, W))
    for x in (one.expand(N, 1, W), torch.zeros(N * W).as_strided((N, 1, W), (W - 1, W, 1)), torch.zeros(N * W).as_strided((N, 1, W), (1, W, 1))):
        with pytest.raises(ValueError, match="constant distance"):
            call(gpu(x))
    assert not peers._lib.made


@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("T", [0, 1, 3])
def test_row_strides_reach_the_library(peers, name, T):
    """Contiguous rows, and rows with others' elements between them, whatever the stride of a token dimension of one."""
    call = operators(peers, T)[name]
    wide = gpu(torch.zeros((N, T, W + 5)))[..., :W]
    odd = gpu(torch.zeros(N * (W + 5)).as_strided((N, 1, W), (W + 5, 1, 1))) if T == 1 else wide
    for x, stride in ((gpu(torch.zeros((N, T, W))), W), (wide, W + 5), (odd, W + 5)):
        peers._lib.made.clear()
        call(x)
        (_, args), = peers._lib.made
        at = max(i for i, a in enumerate(args) if a == x.data_ptr()) if T else None
        if T:
            assert stride in args[at: at + 6], args


class Stream:
    def __init__(self, handle):
        self.cuda_stream = handle


class Lent(OnGpu):
    """Writes down the streams that the allocator is told of."""

    def record_stream(self, stream):
        self.__dict__.setdefault("lent", []).append(stream)


@pytest.mark.parametrize("away", [False, True])
def test_the_allocator_hears_of_the_stream_that_uses_a_tensor(peers, away, monkeypatch):
    """Every tensor of a call is lent to the bound stream where another one is current, and the new ones, which are the bound stream's, to the
    current one.  (A temporary's memory could be given out again while the bound stream still reads it, else.)"""
    bound, current, empty = Stream(7), Stream(5 if away else 7), torch.empty
    monkeypatch.setattr(binding, "_current_stream", lambda index: current.cuda_stream)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: current)
    monkeypatch.setattr(torch.cuda, "stream", lambda stream: contextlib.nullcontext())
    monkeypatch.setattr(torch, "empty", lambda *a, **k: empty(*a, **k).as_subclass(Lent))
    m, T = peers, 3
    m._state, m._bound = (m._state[0], bound), (0, bound.cuda_stream)

    def new(shape, dtype=torch.float32):
        return torch.zeros(shape, dtype=dtype).as_subclass(Lent)

    def tokens():
        return new((N, T), torch.int32)

    def v():
        return new((N, T))

    def saved():
        return new((N, T, W), torch.int8), new((N, T, W // 32), torch.uint8)
    # of each call: the tensors given to it, and the ones it makes
    for call, given in (
            (lambda t, out: (m.embed(t, 0, V, W, out=out), ())[1], [tokens(), new((N, T, W))]),
            (lambda t: m.embed(t, 0, V, W), [tokens()]),
            (lambda y, t, G: m.embed_grad(y, t, G, 0, V), [new((N, T, W)), tokens(), new((N, m.P))]),
            (lambda x: m.checkpoint(x), [new((N, T, W))]),
            (lambda c, s: m.checkpoint_restore(c, s), [*saved()]),
            (lambda c, s, out: (m.checkpoint_restore(c, s, out=out), ())[1], [*saved(), new((N, T, W))]),
            (lambda y, c, s, G: m.weight_grad(y, c, s, G, 0), [new((N, T, V)), *saved(), new((N, m.P))]),
            (lambda z, t: m.token_logp(z, t), [new((N, T, W)), tokens()]),
            (lambda z, t, o, a, w: m.policy_loss(z, t, o, a, w), [new((N, T, W)), tokens(), v(), v(), v()]),
            (lambda z, t, o, a, w, r, g: m.policy_loss(z, t, o, a, w, ref_logp=r, grad=g), [new((N, T, W)), tokens(), v(), v(), v(), v(), new((N, T, W))]),
            (lambda G: m.local_step(G, 0.1), [new((N, m.P))]),
            (lambda G: m.sgd_round(0, G, 0.1), [new((N, m.P))]),
            (lambda G: m.sgd_run(0, 1, G, 0.1), [new((N, m.P))])):
        made = call(*given)
        made = [x for x in (made if isinstance(made, tuple) else [made]) if isinstance(x, Lent)]
        for x in given:
            assert (bound in x.__dict__.get("lent", [])) == away
        for x in made:
            assert (current in x.__dict__.get("lent", [])) == away


@pytest.mark.parametrize("bound_before", [False, True])
@pytest.mark.parametrize("handle", [0, 9])
def test_a_raw_binding_takes_the_place_of_the_one_before(peers, bound_before, handle, monkeypatch):
    """After bind_raw the operators' tensors are lent to its stream, not to an earlier binding's, and gradients are taken."""
    streams = []
    monkeypatch.setattr(binding, "_current_stream", lambda index: 5)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: Stream(5))
    monkeypatch.setattr(torch.cuda, "stream", lambda stream: streams.append(stream) or contextlib.nullcontext())
    monkeypatch.setattr(torch.cuda, "ExternalStream", Stream)
    monkeypatch.setattr(torch.cuda, "default_stream", lambda device=None: Stream(0))
    empty = torch.empty
    monkeypatch.setattr(torch, "empty", lambda *a, **k: empty(*a, **k).as_subclass(Lent))
    m = peers
    m._state, m._bound = ((m._state[0], Stream(7)), (0, 7)) if bound_before else (None, None)
    m.bind_raw(4096, m.P, handle)
    x, tokens = torch.zeros((N, 3, W)).as_subclass(Lent), torch.zeros((N, 3), dtype=torch.int32).as_subclass(Lent)
    G = torch.zeros((N, m.P)).as_subclass(Lent)
    made = m.checkpoint(x)
    m.embed_grad(x, tokens, G, 0, V)
    for t in (x, tokens, G):
        assert {s.cuda_stream for s in t.__dict__.get("lent", [])} == {handle}
    assert [s.cuda_stream for s in streams] == [handle]
    for t in made:
        assert [s.cuda_stream for s in t.__dict__["lent"]] == [5]
    with pytest.raises(ValueError, match="gradient tensor"):
        m.embed_grad(x, tokens, G.bfloat16(), 0, V)
