"""What the binding hands to the library for the local step's operators, and what it refuses: on the CPU, with tensors that
say they are on the GPU and a library that writes down its calls."""
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
