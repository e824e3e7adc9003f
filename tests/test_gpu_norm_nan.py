"""Layer norm of rows with NaN and infinities: all that such a row gives is NaN, its statistics too, and the other rows are as without it."""
import math

import pytest
import torch

from paper_2602_03067_amd import binding
from tests._gpu_common import say
from tests.test_gpu_norm import BF16, F32, normal

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("cols", [5, 64, 130, 784, 4096, 20001])
def test_row(cols, value, dtype):
    say("norm %g in a row of %d %s" % (value, cols, dtype))
    ctx = binding.Context(0)
    x, dy = normal(1, dtype, 9, cols), normal(2, dtype, 9, cols)
    y0, st0 = ctx.fs_layer_norm(x)
    dx0 = ctx.fs_layer_norm_grad(x, None, st0, dy)[0]
    x[4, cols // 2] = value
    y, st = ctx.fs_layer_norm(x)
    dx, dg, db = ctx.fs_layer_norm_grad(x, None, st, dy)
    keep = torch.arange(9, device="cuda") != 4
    for t, clean in ((y, y0), (st, st0), (dx, dx0)):
        assert torch.equal(t[keep], clean[keep])
    assert torch.isnan(y[4]).all() and torch.isnan(dx[4]).all() and torch.isnan(dg).all() and torch.isfinite(db).all()
    assert torch.isnan(st[4, 1]) and not torch.isfinite(st[4, 0])
    ctx.close()
