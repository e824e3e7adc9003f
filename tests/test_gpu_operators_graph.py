"""Graphs of operators hold the context's second buffer: it stays where a later call needs a larger one, and does not grow under a recording."""
import pytest
import torch

from paper_2602_03067_amd import binding
from tests._gpu_common import say

pytestmark = pytest.mark.gpu


def normal(seed, dtype, *shape):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_buffer_of_a_graph_stays(dtype):
    say("operators graph, buffer grown later %s" % dtype)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        ctx = binding.Context(0)
        q, k = normal(1, dtype, 2, 3, 4, 64), normal(2, dtype, 2, 4000, 4, 64)

        def step():
            o, st = ctx.fs_attention(q, k, k)
            return (o, st, *ctx.fs_attention_grad(q, k, k, o, st, q))

        step()
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            out = step()
        for rep in range(3):
            big = normal(3, dtype, 2 + rep, 700 + 500 * rep, 8, 128)   # (needs more, and more again)
            o, st = ctx.fs_attention(big, big, big)
            ctx.fs_attention_grad(big, big, big, o, st, big)
            other = [torch.full((1 << 20,), float(rep), device="cuda") for _ in range(40)]   # (whoever takes memory that was given back)
            q.copy_(normal(10 + rep, dtype, 2, 3, 4, 64))
            graph.replay()
            stream.synchronize()
            got = [t.clone() for t in out]
            assert all(torch.equal(a, b) for a, b in zip(got, step()))
            assert all((t == rep).all() for t in other)
        stream.synchronize()
        del graph
        ctx.close()


def test_no_growth_under_a_recording():
    say("operators graph, no growth")
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        ctx = binding.Context(0)
        q, k = normal(1, torch.float32, 2, 3, 4, 64), normal(2, torch.float32, 2, 4000, 4, 64)
        small = normal(3, torch.float32, 50, 64)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            y, _ = ctx.fs_layer_norm(small)
            with pytest.raises(binding.FlashSinkError):
                ctx.fs_attention(q, k, k)
        for rep in range(2):   # (the recording is none the worse)
            small.copy_(normal(4 + rep, torch.float32, 50, 64))
            graph.replay()
            stream.synchronize()
            assert torch.equal(y, ctx.fs_layer_norm(small)[0])
        ctx.fs_attention(q, k, k)
        stream.synchronize()
        ctx.close()
