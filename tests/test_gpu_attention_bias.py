"""Removed keys (a bias of minus infinity) that hold NaN and infinities, in tiles of every kind: some keys of a tile, whole tiles, all of
them; few rows and many, one part of the keys and several.  The definition and the tolerances are those of test_gpu_attention.py.
"""
import math

import pytest
import torch

from paper_2602_03067_amd import binding
from tests._gpu_common import say
from tests.test_gpu_attention import BF16, F32, case, check

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(0)
    yield c
    c.close()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,m,heads,kv_heads,d", [
    (300, 700, 4, 4, 32), (300, 700, 4, 2, 64), (130, 1100, 4, 4, 96), (300, 700, 2, 2, 128), (3, 2000, 4, 1, 64), (700, 65, 2, 2, 64),
    (64, 257, 3, 3, 63), (2000, 300, 8, 8, 64)])
def test_removed_keys_of_any_tile(ctx, n, m, heads, kv_heads, d, dtype):
    say("attention removed keys n=%d m=%d heads=%d/%d d=%d %s" % (n, m, heads, kv_heads, d, dtype))
    q, k, v, do = case(7, dtype, 4, n, m, heads, kv_heads, d)
    g = torch.Generator().manual_seed(n + m)
    bias = torch.log(torch.rand(4, m, generator=g) + 0.25)
    bias[0, torch.rand(m, generator=g) < 0.5] = -math.inf
    bias[1, m // 3:] = -math.inf             # whole tiles at the end
    bias[2, :m - m // 3 - 1] = -math.inf     # and at the beginning
    bias[3, 1:] = -math.inf                  # one is left
    bias = bias.cuda()
    gone = bias == -math.inf
    k[gone] = math.nan
    v[gone] = math.inf
    _, _, grads = check(ctx, q, k, v, do, False, None, None, bias)
    assert (grads[3][gone] == 0).all()


def test_lengths_inside_removed_keys(ctx):
    """Lengths that end within a run of removed keys, whose bias past them is not a number."""
    say("attention lengths inside removed keys")
    q, k, v, do = case(8, BF16, 3, 200, 600, 4, 4, 64)
    bias = torch.zeros(3, 600)
    bias[:, 250:400] = -math.inf
    k_len = torch.tensor([300, 450, 251], dtype=torch.int32)
    for b in range(3):
        k[b, 250:400] = v[b, 250:400] = math.nan
        k[b, k_len[b]:] = v[b, k_len[b]:] = math.inf
        bias[b, k_len[b]:] = math.nan
    check(ctx, q, k, v, do, False, None, k_len.cuda(), bias.cuda())
