"""Keys and values whose rows lie far apart: offsets within one tile that come near 32 bits or pass them."""
import pytest
import torch

from paper_2602_03067_amd import binding
from tests._gpu_common import say
from tests.test_gpu_attention import BF16, case, check

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(0)
    yield c
    c.close()


@pytest.mark.parametrize("n,m,d", [(300, 300, 32), (300, 140, 96), (1, 300, 64)])
@pytest.mark.parametrize("megabytes", [15, 20, 40])
def test_far_rows(ctx, megabytes, n, m, d):
    say("attention rows %d MB apart n=%d m=%d d=%d" % (megabytes, n, m, d))
    q, k, v, do = case(3, BF16, 1, n, m, 1, 1, d)
    far = torch.empty(m, megabytes << 19, dtype=BF16, device="cuda")
    kk, vv = far[None, :, None, :d], far[None, :, None, 128:128 + d]
    kk.copy_(k)
    vv.copy_(v)
    check(ctx, q, kk, vv, do)
