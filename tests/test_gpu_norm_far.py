"""Layer norm of rows whose mean is far from zero beside their spread: the mean, a float, is off by up to half an ulp, and what that leaves in
the deviations is taken off in the gradients as well, at every length of a row.  Formulas and tolerances are those of test_gpu_norm.py."""
import pytest
import torch

from paper_2602_03067_amd import binding
from tests._gpu_common import say
from tests.test_gpu_norm import BF16, F32, TOL, close, formulas, normal

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(0)
    yield c
    c.close()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("mean", [100.0, 1000.0])
@pytest.mark.parametrize("rows,cols", [(50, 300), (33, 2056), (9, 16384), (9, 16385), (12, 20001), (7, 40000), (300, 16400)])
def test_gradients_of_rows_far_from_zero(ctx, rows, cols, mean, dtype):
    say("norm far %d x %d at %g %s" % (rows, cols, mean, dtype))
    x = (normal(1, F32, rows, cols) + mean * (1 + 0.3 * normal(2, F32, rows, 1))).to(dtype)
    gamma, beta, dy = 1 + 0.1 * normal(3, F32, cols), 0.1 * normal(4, F32, cols), normal(5, dtype, rows, cols) + 0.5
    # (the gradients from the statistics in 64 bits, rounded, as a forward pass gives them at best)
    want = formulas(x, gamma, beta, 1e-5, dy)
    y, _ = ctx.fs_layer_norm(x, gamma, beta)
    close("y", y, want["y"], TOL[dtype])
    dx, dg, db = ctx.fs_layer_norm_grad(x, gamma, want["stat"].float(), dy)
    close("dx", dx, want["dx"], TOL[dtype])
    close("dgamma", dg, want["dgamma"], 5e-6, want["terms"])
    close("dbeta", db, want["dbeta"], 5e-6, want["plain"])


@pytest.mark.parametrize("cols", [300, 16384, 20001])
def test_weights_alone_and_in_place_are_the_same(ctx, cols):
    """The weights' gradients do not depend on whether dx is wanted, or takes dy's place."""
    say("norm far, weights alone %d" % cols)
    x, dy = normal(1, F32, 11, cols) + 1000.0, normal(2, F32, 11, cols)
    _, stat = ctx.fs_layer_norm(x)
    dx, dg, db = ctx.fs_layer_norm_grad(x, None, stat, dy)
    for at in (None, dy.clone()):
        given = dy if at is None else at
        dw = torch.empty(2, cols, device="cuda")
        assert ctx.lib.fs_layer_norm_grad(ctx.h, x.data_ptr(), 0, 11, cols, cols, None, 0, stat.data_ptr(), given.data_ptr(), cols,
                                          None if at is None else at.data_ptr(), cols, dw.data_ptr(), dw.data_ptr() + 4 * cols) == 0
        assert torch.equal(dw[0], dg) and torch.equal(dw[1], db) and (at is None or torch.equal(at, dx))
