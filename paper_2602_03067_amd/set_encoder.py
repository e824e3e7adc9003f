"""A small encoder of point sets, trained on the debiased Sinkhorn divergence.

    python -m paper_2602_03067_amd.set_encoder [--steps 60] [--dtype float32|bfloat16] [--state-bits 32|8]

It moves the points of a cloud onto a target: layers of pre-norm attention and of a two-matrix map, residual connections, and a last
map whose output is added to the points.  Attention, layer norm, their gradients, the loss with its gradient and the optimiser step
are the library's; the projections are torch products.  There is no autograd: every step's backward pass is written out, and
``SetEncoder.backward`` may be read as the order in which the operators' gradients are called.
"""
from __future__ import annotations

import argparse

import torch

from . import binding


class SetEncoder:
    """Weights are in ``params`` (one type); with bfloat16 ``masters`` holds them as floats for the optimiser."""

    def __init__(self, ctx: binding.Context, coords: int = 3, width: int = 64, heads: int = 4, layers: int = 2, dtype=torch.float32, seed: int = 0):
        if width % heads:
            raise ValueError("heads must divide width")
        self.ctx, self.coords, self.width, self.heads, self.layers, self.dtype = ctx, coords, width, heads, layers, dtype
        gen = torch.Generator().manual_seed(seed)

        def dense(rows, cols, gain=1.0):
            return torch.randn(rows, cols, generator=gen) * (gain / cols ** 0.5)

        one, zero = torch.ones(width), torch.zeros(width)
        w = [dense(width, coords), zero]
        for _ in range(layers):
            w += [one, zero, dense(3 * width, width), dense(width, width, 0.5), one, zero, dense(4 * width, width), dense(width, 4 * width, 0.5)]
        w += [one, zero, dense(coords, width, 0.1)]
        floats = [t.clone().to("cuda:%d" % ctx.device) for t in w]
        self.params = [t.to(dtype) for t in floats]
        self.masters = floats if dtype != torch.float32 else None

    def forward(self, x: torch.Tensor, k_len=None) -> torch.Tensor:
        """x (sets, points, coordinates) float32 -> the moved points; ``k_len``: points of each set, the others are padding."""
        p, ctx = self.params, self.ctx
        b, n, _ = x.shape
        xt = x.reshape(b * n, self.coords).to(self.dtype)
        h = torch.addmm(p[1], xt, p[0].t())
        self._saved = [x.shape, xt, k_len]
        for i in range(self.layers):
            g1, b1, wqkv, wo, g2, b2, wu, wd = p[2 + 8 * i:10 + 8 * i]
            a, st1 = ctx.fs_layer_norm(h, g1, b1)
            q, k, v = (a @ wqkv.t()).view(b, n, 3, self.heads, -1).unbind(2)
            o, st = ctx.fs_attention(q, k, v, q_len=k_len, k_len=k_len)
            mid = torch.addmm(h, o.reshape(b * n, -1), wo.t())
            c, st2 = ctx.fs_layer_norm(mid, g2, b2)
            u = torch.relu(c @ wu.t())
            self._saved.append((h, st1, a, q, k, v, o, st, mid, st2, c, u))
            h = torch.addmm(mid, u, wd.t())
        g, bb, w = p[-3:]
        a, st1 = ctx.fs_layer_norm(h, g, bb)
        self._saved.append((h, st1, a))
        return x + (a @ w.t()).view(x.shape).float()

    def backward(self, dy: torch.Tensor):
        """Gradients of all weights, in their order and type, for the gradient of the moved points."""
        p, ctx = self.params, self.ctx
        shape, xt, k_len = self._saved[:3]
        b, n = shape[:2]
        h, st1, a = self._saved[-1]
        d = dy.reshape(b * n, self.coords).to(self.dtype)
        tail = [d.t() @ a]
        dh, dg, db = ctx.fs_layer_norm_grad(h, p[-3], st1, d @ p[-1])
        tail = [dg, db] + tail
        for i in reversed(range(self.layers)):
            g1, b1, wqkv, wo, g2, b2, wu, wd = p[2 + 8 * i:10 + 8 * i]
            h, st1, a, q, k, v, o, st, mid, st2, c, u = self._saved[3 + i]
            dwd = dh.t() @ u
            du = (dh @ wd) * (u > 0)
            dc, dg2, db2 = ctx.fs_layer_norm_grad(mid, g2, st2, du @ wu)
            dwu, dm = du.t() @ c, dh + dc
            do = (dm @ wo).view(b, n, self.heads, -1)
            dwo = dm.t() @ o.reshape(b * n, -1)
            dqkv = torch.stack(ctx.fs_attention_grad(q, k, v, o, st, do, q_len=k_len, k_len=k_len), 2).view(b * n, -1)
            da, dg1, db1 = ctx.fs_layer_norm_grad(h, g1, st1, dqkv @ wqkv)
            tail = [dg1, db1, dqkv.t() @ a, dwo, dg2, db2, dwu, dwd] + tail
            dh = dm + da
        grads = [dh.t() @ xt, dh.float().sum(0)] + tail
        return [t.to(self.dtype).contiguous() for t in grads]


def divergence(ctx: binding.Context, x: torch.Tensor, y: torch.Tensor, eps: float, iters: int):
    """Debiased Sinkhorn divergence of two clouds and its gradient with respect to x (the self term counts both of its sides)."""
    value, _, f, g = ctx.fs_divergence(binding.Problem(x, y), eps, iters)
    grad = ctx.fs_grad_x(binding.Problem(x, y), eps, f, g, 0)
    own = binding.Problem(x, x)
    f, g = torch.zeros_like(f), torch.zeros(x.shape[0], device=x.device)
    ctx.fs_solve(own, eps, eps, 1, iters, f, g)
    return value, grad - 0.5 * (ctx.fs_grad_x(own, eps, f, g, 0) + ctx.fs_grad_y(own, eps, f, g, 0))


def train(steps: int = 60, points: int = 1024, dtype=torch.float32, state_bits: int = 32, eps: float = 0.05, iters: int = 20, lr: float = 2e-3,
          device: int = 0, seed: int = 0, say=None):
    """Trains an encoder to move a normal cloud onto a ring; returns the loss of every step."""
    dev = "cuda:%d" % device
    gen = torch.Generator().manual_seed(seed + 1)
    x = torch.randn(1, points, 3, generator=gen).to(dev)
    angle = torch.rand(points, generator=gen) * 6.2831853
    y = (torch.stack([angle.cos(), angle.sin(), 0.0 * angle], 1) + 0.05 * torch.randn(points, 3, generator=gen)).to(dev)
    ctx = binding.Context(device)
    net = SetEncoder(ctx, dtype=dtype, seed=seed)
    opt = binding.AdamW(ctx, net.params, lr=lr, weight_decay=0.01, state_bits=state_bits, master=net.masters)
    losses = []
    for step in range(steps):
        moved = net.forward(x)
        loss, grad = divergence(ctx, moved[0].contiguous(), y, eps, iters)
        # (the gradient of a mean over points: of the order of the points' distances, not of 1 / points)
        opt.step(net.backward(points * grad[None]))
        losses.append(loss)
        if say and (step % 10 == 0 or step == steps - 1):
            say("step %3d  divergence %.5f" % (step, loss))
    ctx.close()
    return losses


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--points", type=int, default=1024)
    ap.add_argument("--dtype", choices=("float32", "bfloat16"), default="float32")
    ap.add_argument("--state-bits", type=int, choices=(32, 8), default=32)
    a = ap.parse_args()
    train(a.steps, a.points, getattr(torch, a.dtype), a.state_bits, say=lambda s: print(s, flush=True))
