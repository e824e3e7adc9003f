"""float32 attention through pairs of fp16 where q, k or their products leave a float's range: scores are as good as zero (or what they are),
and rows that see some keys only, or none, are as with any other scores.  Tolerance as in test_gpu_attention_pairs.py."""
import math

import pytest
import torch

from paper_2602_03067_amd import binding
from tests._gpu_common import say
from tests.test_gpu_attention import F32, case, check

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(0)
    c.fs_debug_set("attn_pairs", 1)
    yield c
    c.close()


@pytest.mark.parametrize("n,m", [(100, 130), (200, 77), (150, 2001)])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("sizes", [(1e-20, 1e-20), (1e-19, 1e-19), (1e-30, 1e-30), (1e-30, 1.0), (1e-12, 1e-28)])
def test_products_below_the_smallest_float(ctx, sizes, causal, n, m):
    say("pairs tiny scores %s causal=%s %d %d" % (sizes, causal, n, m))
    q, k, v, do = case(41, F32, 2, n, m, 2, 1, 64)
    q, k = q * sizes[0], k * sizes[1]
    q_len = torch.tensor([n, n - 40], dtype=torch.int32).cuda()
    k_len = torch.tensor([m, m - 33], dtype=torch.int32).cuda()
    check(ctx, q, k, v, do, causal, q_len, k_len)


def test_removed_keys_beside_scores_of_zero(ctx):
    say("pairs tiny scores, removed keys")
    q, k, v, do = case(42, F32, 2, 70, 130, 2, 2, 40)
    bias = torch.zeros(2, 130)
    bias[0, ::3] = -math.inf
    bias[1] = -math.inf
    check(ctx, q * 1e-25, k * 1e-25, v, do, False, None, None, bias.cuda())


@pytest.mark.parametrize("sizes", [(1e30, 1e-30), (1e-25, 1e25), (1e18, 1e-18)])
def test_sizes_that_cancel(ctx, sizes):
    say("pairs sizes that cancel %s" % (sizes,))
    q, k, v, do = case(43, F32, 2, 90, 150, 2, 1, 64)
    check(ctx, q * sizes[0], k * sizes[1], v, do, True)
