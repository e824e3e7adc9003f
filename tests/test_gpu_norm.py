"""Layer norm, forward and backward, against the formulas in 64 bits.

Tolerances (relative, 2-norm): float32 outputs 2e-6 (mean and deviation in fp32 sums, a few roundings of 2^-24 each, the
deviations' own cancellation against a mean of a quarter of the spread), bfloat16 outputs 2.5e-3 (their own rounding is
1.1e-3 rms); sums over rows 5e-6 of the norm of the terms."""
import math

import pytest
import torch

from paper_2602_03067_amd import binding
from tests._gpu_common import say

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
TOL = {F32: 2e-6, BF16: 2.5e-3}


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(0)
    yield c
    c.close()


def normal(seed, dtype, *shape):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()


def formulas(x, gamma, beta, eps, dy):
    x, dy = x.double(), dy.double()
    g = torch.ones(x.shape[1], dtype=torch.float64, device=x.device) if gamma is None else gamma.double()
    b = torch.zeros_like(g) if beta is None else beta.double()
    mean = x.mean(1, keepdim=True)
    rstd = ((x - mean).square().mean(1, keepdim=True) + eps).rsqrt()
    xh = (x - mean) * rstd
    w = dy * g
    dx = rstd * (w - w.mean(1, keepdim=True) - xh * (w * xh).mean(1, keepdim=True))
    return dict(y=xh * g + b, stat=torch.cat([mean, rstd], 1), dx=dx, dgamma=(dy * xh).sum(0), dbeta=dy.sum(0),
                terms=(dy * xh).norm().item(), plain=dy.norm().item(), dxn=(rstd * w).norm().item())


def close(name, got, want, tol, size=None):
    off = (got.double() - want).norm().item()
    size = want.norm().item() if size is None else size
    assert off <= tol * size, "%s: off by %.3g of %.3g" % (name, off, size)


def check(ctx, x, gamma, beta, dy, eps=1e-5):
    want = formulas(x, gamma, beta, eps, dy)
    y, stat = ctx.fs_layer_norm(x, gamma, beta, eps)
    dx, dg, db = ctx.fs_layer_norm_grad(x, gamma, stat, dy)
    tol = TOL[x.dtype]
    close("y", y, want["y"], tol)
    close("stat", stat, want["stat"], 2e-6)
    close("dx", dx, want["dx"], tol, max(want["dx"].norm().item(), 0.1 * want["dxn"]))   # (short rows: what is left of the terms)
    close("dgamma", dg, want["dgamma"], 5e-6, want["terms"])
    close("dbeta", db, want["dbeta"], 5e-6, want["plain"])
    return y, stat, dx, dg, db


COLS = [2, 3, 7, 8, 31, 64, 65, 127, 256, 333, 512, 784, 1000, 1024, 2047, 2048, 2056, 4096, 5001, 8192, 8200, 16384, 16400, 20001, 40000]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("cols", COLS)
def test_columns(ctx, cols, dtype):
    for rows in (1, 5, 37) if cols > 4096 else (1, 5, 1100):
        say("norm %d x %d %s" % (rows, cols, dtype))
        check(ctx, normal(1, dtype, rows, cols) * 2 + 0.5, 1 + 0.1 * normal(2, F32, cols), 0.1 * normal(3, F32, cols), normal(4, dtype, rows, cols))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows", [2, 255, 1024, 9001])
def test_rows(ctx, rows, dtype):
    say("norm rows %d %s" % (rows, dtype))
    check(ctx, normal(5, dtype, rows, 96), normal(6, BF16, 96), normal(7, BF16, 96), normal(8, dtype, rows, 96))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_without_weights(ctx, dtype):
    say("norm without weights %s" % dtype)
    x, dy = normal(9, dtype, 50, 200), normal(10, dtype, 50, 200)
    check(ctx, x, None, None, dy)
    check(ctx, x, normal(11, F32, 200), None, dy)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("how", ["spaced", "shifted", "unaligned weights"])
def test_strides(ctx, how, dtype):
    say("norm strides %s %s" % (how, dtype))
    x, dy = normal(12, dtype, 70, 170), normal(13, dtype, 70, 170)
    gamma, beta = normal(14, F32, 129), normal(15, F32, 129)
    if how == "spaced":
        check(ctx, x[:, 8:136], gamma[:128], beta[:128], dy[:, 16:144])
    elif how == "shifted":
        check(ctx, x[:, 3:131], gamma[:128], beta[:128], dy[:, 1:129])
    else:
        check(ctx, x[:, :128].contiguous(), gamma[1:], beta[1:], dy[:, :128].contiguous())


def test_constant_rows_and_offsets(ctx):
    """A row of one value has deviation 0: rstd = 1 / sqrt(eps).  A mean far from zero costs the deviations its ulp and no more."""
    say("norm constant rows")
    x = torch.full((4, 300), 3.0).cuda()
    y, stat = ctx.fs_layer_norm(x, eps=1e-4)
    assert (y == 0).all() and torch.allclose(stat[:, 1], torch.full((4,), 100.0).cuda(), rtol=1e-6)
    x = normal(16, F32, 20, 300) + 1000.0
    y, stat = ctx.fs_layer_norm(x)
    want = formulas(x, None, None, 1e-5, x)
    # the mean is rounded to 2^-14, against deviations of 1
    assert (y.double() - want["y"]).abs().max() < 3e-4


def test_values_that_are_not_finite_stay_in_their_row(ctx):
    say("norm not finite")
    x, dy = normal(17, F32, 9, 130), normal(18, F32, 9, 130)
    clean, _ = ctx.fs_layer_norm(x)
    x[4, 7] = math.inf
    y, stat = ctx.fs_layer_norm(x)
    assert torch.isnan(y[4]).any() and torch.equal(y[:4], clean[:4]) and torch.equal(y[5:], clean[5:])


def test_no_rows(ctx):
    x = torch.empty(0, 40).cuda()
    y, stat = ctx.fs_layer_norm(x)
    dx, dg, db = ctx.fs_layer_norm_grad(x, None, stat, x)
    assert y.shape == (0, 40) and (dg == 0).all() and (db == 0).all()


@pytest.mark.parametrize("cols", [100, 30000, 40000])
def test_gradient_in_place_of_dy(ctx, cols):
    say("norm in place %d" % cols)
    x, dy = normal(19, F32, 12, cols), normal(20, F32, 12, cols)
    y, stat = ctx.fs_layer_norm(x)
    want = ctx.fs_layer_norm_grad(x, None, stat, dy)
    dw = torch.empty(2, cols).cuda()
    st = ctx.lib.fs_layer_norm_grad(ctx.h, x.data_ptr(), 0, 12, cols, cols, None, 0, stat.data_ptr(), dy.data_ptr(), cols, dy.data_ptr(), cols,
                                    dw.data_ptr(), dw.data_ptr() + 4 * cols)
    assert st == 0 and torch.equal(dy, want[0]) and torch.equal(dw[0], want[1]) and torch.equal(dw[1], want[2])


def test_same_call_same_bits(ctx):
    x, dy = normal(21, BF16, 3000, 784), normal(22, BF16, 3000, 784)
    y, stat = ctx.fs_layer_norm(x)
    a, b = ctx.fs_layer_norm_grad(x, None, stat, dy), ctx.fs_layer_norm_grad(x, None, stat, dy)
    for s, t in zip(a, b):
        assert torch.equal(s, t)


def test_differences(ctx):
    """<w, y> along random directions: truncation h^2 = 1e-4, fp32 noise 1e-6 / h, of the product of the norms; 1e-3."""
    say("norm differences")
    x, gamma, beta, w = normal(23, F32, 6, 50), normal(24, F32, 50), normal(25, F32, 50), normal(26, F32, 6, 50)
    y, stat = ctx.fs_layer_norm(x, gamma, beta)
    grads = ctx.fs_layer_norm_grad(x, gamma, stat, w)
    h = 1e-2
    for i in range(3):
        args = [x, gamma, beta]
        e = normal(30 + i, F32, *args[i].shape)
        vals = []
        for sign in (1, -1):
            a = list(args)
            a[i] = args[i] + sign * h * e
            vals.append((ctx.fs_layer_norm(*a)[0].double() * w.double()).sum().item())
        want = (grads[i].double() * e.double()).sum().item()
        assert abs((vals[0] - vals[1]) / (2 * h) - want) <= 1e-3 * grads[i].double().norm().item() * e.double().norm().item()


def test_refusals(ctx):
    x = normal(40, F32, 4, 8)
    y, stat = ctx.fs_layer_norm(x)
    for bad in (lambda: ctx.fs_layer_norm(x.half()), lambda: ctx.fs_layer_norm(x.t()), lambda: ctx.fs_layer_norm(x, gamma=x[0, :5]),
                lambda: ctx.fs_layer_norm(x.cpu()), lambda: ctx.fs_layer_norm(x, x[0].clone(), x[0].to(BF16))):
        with pytest.raises(TypeError):
            bad()
    with pytest.raises(ValueError):
        ctx.fs_layer_norm_grad(x, None, stat, x[:, :4])
    for eps in (-1.0, math.nan, math.inf):
        with pytest.raises(binding.FlashSinkError):
            ctx.fs_layer_norm(x, eps=eps)
