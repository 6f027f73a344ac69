"""The local step's operators as programs use them: captured graphs replayed after other calls."""
import pytest
import torch

from paper_2103_03239_amd import binding
from test_gpu_local_ops import DEV, normal, rng, some_tokens

pytestmark = pytest.mark.gpu


def test_a_graph_replays_after_calls_that_need_more_workspace():
    """Every operator that has a workspace is captured at a small size, then called eagerly at growing ones, whose workspace does not fit the
    captured block; memory of that block's size is taken and filled; the replays still give what eager calls give."""
    g = rng(21)
    N, V, D, I = 4, 500, 64, 96
    X, G = normal((N, 4_000_000), torch.float32, g), torch.zeros((N, 4_000_000), device=DEV)

    def inputs(T, vocab):
        tokens = some_tokens("any", N, T, V, g)
        return dict(tokens=tokens, x=normal((N, T, I), torch.float32, g), y=normal((N, T, D), torch.float32, g), z=normal((N, T, vocab), torch.float32, g),
                    v=torch.rand((N, T), generator=g, device=DEV), grad=torch.empty((N, T, vocab), device=DEV))

    def step(m, c):
        logp = m.token_logp(c["z"], c["tokens"])
        stats, lp = m.policy_loss(c["z"], c["tokens"], c["v"], c["v"], c["v"], grad=c["grad"])
        codes, scales = m.checkpoint(c["x"])
        m.weight_grad(c["y"], codes, scales, G, V * D)
        m.embed_grad(c["y"], c["tokens"], G, 0, V)
        return logp, stats, lp

    side = torch.cuda.Stream()
    small, larger = inputs(300, 70_000), [inputs(T, 600) for T in (2_000, 9_000, 30_000)]
    torch.cuda.synchronize()
    with binding.Moshpit(N, X.shape[1], 2, 2, binding.F32) as m, torch.cuda.stream(side):
        m.bind_state(X, side)
        step(m, small)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            held = step(m, small)
        for k, c in enumerate(larger):
            step(m, c)
            side.synchronize()
            filled = [torch.full((1 << e,), 0x7fc00000, dtype=torch.int32, device=DEV) for e in range(10, 26)]
            small["z"].normal_(generator=g)
            small["y"].normal_(generator=g)
            G.fill_(9.0)
            graph.replay()
            side.synchronize()
            replayed = [t.clone() for t in (G, small["grad"], *held)]
            G.fill_(9.0)
            eager = step(m, small)
            side.synchronize()
            for a, b in zip(replayed, (G, small["grad"], *eager)):
                assert torch.equal(a, b), k
            assert all(bool((t == 0x7fc00000).all()) for t in filled)
            del filled


def test_memory_waits_for_the_stream_that_still_uses_it():
    """With another stream current than the bound one: a temporary input's memory is not given out again while the bound stream has yet to
    read it, nor a result's while the current stream has yet to."""
    g = rng(22)
    N, T, W = 4, 250, 1_000
    X, x = torch.zeros((N, 16), device=DEV), normal((N, T, W), torch.float32, g)
    big = normal((8_192, 8_192), torch.float32, g)
    side, here = torch.cuda.Stream(), torch.cuda.current_stream()

    def busy(stream):
        """Work of some hundred milliseconds, and an event behind it."""
        with torch.cuda.stream(stream):
            for _ in range(30):
                torch.mm(big, big)
            return stream.record_event()

    torch.mm(big, big)
    torch.cuda.synchronize()
    with binding.Moshpit(N, 16, 2, 2, binding.F32) as m:
        m.bind_state(X, side)
        codes, scales = m.checkpoint(x * 2.0)
        torch.cuda.synchronize()
        want, want_scales = codes.clone(), scales.clone()
        value = m.checkpoint_restore(codes, scales)
        torch.cuda.synchronize()
        value = value.clone()

        temporary = x * 2.0
        side.wait_stream(here)
        end = busy(side)
        at = temporary.data_ptr()
        got = m.checkpoint(temporary)
        del temporary
        other = [torch.empty_like(x) for _ in range(3)]
        assert not end.query(), "the queue was too short to tell"
        assert at not in [t.data_ptr() for t in other]
        torch.cuda.synchronize()
        assert torch.equal(got[0], want) and torch.equal(got[1], want_scales)

        result = m.checkpoint_restore(codes, scales)
        here.wait_stream(side)
        end = busy(here)
        total = result.double().sum()
        at = result.data_ptr()
        del result
        other = [m.checkpoint_restore(codes, scales) for _ in range(3)]
        assert not end.query(), "the queue was too short to tell"
        assert at not in [t.data_ptr() for t in other]
        torch.cuda.synchronize()
        assert float(total) == float(value.double().sum())


def test_a_state_bound_by_address():
    """bind_raw with a stream's handle, after bind_state with another stream: results as with the tensor."""
    g = rng(23)
    N, T, V, D = 4, 90, 70, 32
    X, G = normal((N, V * D), torch.float32, g), torch.zeros((N, V * D), device=DEV)
    tokens, y = some_tokens("any", N, T, V, g), normal((N, T, D), torch.float32, g)
    side, third = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with binding.Moshpit(N, V * D, 2, 2, binding.F32) as m:
        m.bind_state(X, third)
        want = m.embed(tokens, 0, V, D)
        m.embed_grad(y, tokens, G, 0, V)
        m.sync()
        want, want_grad = want.clone(), G.clone()
        torch.cuda.synchronize()
        for stream in (side, torch.cuda.default_stream()):
            m.bind_raw(X.data_ptr(), V * D, stream.cuda_stream)
            G.zero_()
            torch.cuda.synchronize()
            out = m.embed(tokens, 0, V, D)
            codes, scales = m.checkpoint(out)
            m.embed_grad(y, tokens, G, 0, V)
            m.sync()
            assert torch.equal(out, want) and torch.equal(G, want_grad)
            del out, codes, scales
