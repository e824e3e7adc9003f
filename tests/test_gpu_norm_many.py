"""Layer norm of more rows than one launch has threads for."""
import pytest
import torch

from paper_2602_03067_amd import binding
from tests._gpu_common import say
from tests.test_gpu_norm import BF16, normal

pytestmark = pytest.mark.gpu


def test_half_a_billion_short_rows():
    """2^29 rows and some of two columns, eight threads each: 2 GB in, 2 out, 4 of statistics.  A row (a, b) with h = (a - b) / 2 gives
    +-h / sqrt(h^2 + eps), in bf16 (2^-8 of it with the two roundings of fp32 before)."""
    rows = (1 << 29) + 4099
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("less than 24 GB of GPU memory")
    say("norm 2^29 rows")
    ctx = binding.Context(0)
    some = normal(1, BF16, 1 << 20, 2)
    x = torch.empty(rows, 2, dtype=BF16, device="cuda")
    x[:1 << 29].view(512, 1 << 20, 2).copy_(some.expand(512, 1 << 20, 2))
    x[1 << 29:] = normal(2, BF16, 4099, 2)
    y, stat = ctx.fs_layer_norm(x)

    def check(y, stat, x):
        h = (x[:, 0].double() - x[:, 1].double()) / 2
        want = h / (h * h + 1e-5).sqrt()
        near = bool(((y[:, 0].double() - want).abs() <= 2.0 ** -8 * want.abs()).all() and ((y[:, 1].double() + want).abs() <= 2.0 ** -8 * want.abs()).all())
        mean = bool(((stat[:, 0].double() - x.double().mean(1)).abs() <= 1e-6 * x.double().abs().amax(1)).all())
        assert near and mean

    check(y[:1 << 20], stat[:1 << 20], some)
    for k in range(1, 512):
        at = slice(k << 20, (k + 1) << 20)
        same = torch.equal(y[at], y[:1 << 20]) and torch.equal(stat[at], stat[:1 << 20])
        assert same, k
    check(y[1 << 29:], stat[1 << 29:], x[1 << 29:])
    ctx.close()
    del x, y, stat
    torch.cuda.empty_cache()
