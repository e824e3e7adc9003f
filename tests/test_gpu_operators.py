"""What the operators share with the rest of the library: streams, graphs, the workspace beside kept clouds."""
import pytest
import torch

from paper_2602_03067_amd import binding
from tests._gpu_common import say

pytestmark = pytest.mark.gpu


def normal(seed, dtype, *shape):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()


@pytest.mark.parametrize("dtype,n", [(torch.bfloat16, 300), (torch.float32, 300), (torch.float32, 1100)])
def test_recorded_into_a_graph(dtype, n):
    """A step of all operators, recorded once (its buffers grown before) and replayed with other inputs and eager work in between."""
    say("operators graph %s %d" % (dtype, n))
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        ctx = binding.Context(0)
        x = normal(1, dtype, 2 * n, 64)
        gamma, beta = normal(2, torch.float32, 64), normal(3, torch.float32, 64)
        w = [normal(4, torch.float32, 5000), normal(5, torch.float32, 37)]
        start = [t.clone() for t in w]
        opt = binding.AdamW(ctx, w, lr=1e-2)
        grads = [normal(6, torch.float32, 5000), normal(7, torch.float32, 37)]

        def step():
            y, st = ctx.fs_layer_norm(x, gamma, beta)
            q = y.view(2, n, 1, 64)
            o, stat = ctx.fs_attention(q, q, q, causal=True)
            dq, dk, dv = ctx.fs_attention_grad(q, q, q, o, stat, q, causal=True)
            return (y, o, dq, dk, dv, *ctx.fs_layer_norm_grad(x, gamma, st, dq.reshape(2 * n, 64)))

        step()
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            out = step()
            opt.step(grads)
        stream.synchronize()
        for t, s in zip(w, start):   # (recording does nothing)
            assert torch.equal(t, s)
        for k in range(4):
            x.copy_(normal(10 + k, dtype, 2 * n, 64))
            graph.replay()
            stream.synchronize()
            got = [t.clone() for t in out]
            for a, b in zip(got, step()):
                assert torch.equal(a, b)
            stream.synchronize()
        again = [t.clone() for t in start]
        other = binding.AdamW(ctx, again, lr=1e-2)
        for _ in range(4):
            other.step(grads)
            other.step_count = 0   # (the graph holds the step that it was recorded with)
        assert all(torch.equal(a, b) for a, b in zip(w, again))
        ctx.close()


def test_beside_kept_clouds():
    """The operators use the second buffer: copies of clouds declared unchanged stay, and results with them."""
    say("operators beside kept clouds")
    ctx, alone = binding.Context(0), binding.Context(0)
    x, y = normal(1, torch.float32, 3000, 3), normal(2, torch.float32, 2500, 3)
    prob = binding.Problem(x, y)
    res = []
    for c, busy in ((alone, False), (ctx, True)):
        f, g = torch.zeros(3000).cuda(), torch.zeros(2500).cuda()
        c.fs_points_keep(prob)
        for _ in range(3):
            c.fs_solve(prob, 0.1, 0.1, 1, 5, f, g)
            if busy:
                q = normal(3, torch.float32, 1, 700, 4, 64)
                o, st = c.fs_attention(q, q, q)
                c.fs_attention_grad(q, q, q, o, st, q)
                _, st = c.fs_layer_norm(q.view(700, 256))
                c.fs_layer_norm_grad(q.view(700, 256), None, st, q.view(700, 256))
        res.append((f, g, c.fs_grad_x(prob, 0.1, f, g)))
        c.fs_points_release()
    assert all(torch.equal(a, b) for a, b in zip(*res))
    ctx.close()
    alone.close()


def test_one_context_many_sizes():
    """The buffer grows and is laid out anew by every call: a large call after small ones and small ones after it."""
    say("operators many sizes")
    ctx = binding.Context(0)
    want = {}
    for rep in range(2):
        for n, m, dt in ((1, 3000, torch.bfloat16), (900, 40, torch.float32), (64, 64, torch.bfloat16), (1500, 1500, torch.float32), (3, 5, torch.float32)):
            q, k = normal(n, dt, 2, n, 2, 64), normal(m, dt, 2, m, 2, 64)
            o, st = ctx.fs_attention(q, k, k)
            got = (o, st, *ctx.fs_attention_grad(q, k, k, o, st, q))
            for a, b in zip(got, want.setdefault((n, m), got)):
                assert torch.equal(a, b)
    ctx.close()
