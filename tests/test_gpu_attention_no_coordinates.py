"""Heads of no coordinates, or no heads, are refused by the library as any other shape that it does not take."""
import pytest
import torch

from paper_2602_03067_amd import binding
from tests._gpu_common import say

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shape", [(2, 3, 4, 0), (2, 3, 0, 16)])
def test_refused(shape):
    say("attention of shape %s" % (shape,))
    ctx = binding.Context(0)
    q = torch.zeros(shape, device="cuda")
    with pytest.raises(binding.FlashSinkError):
        ctx.fs_attention(q, q, q)
    with pytest.raises(binding.FlashSinkError):
        ctx.fs_attention_grad(q, q, q, q, torch.zeros(shape[0], shape[2], shape[1], 2, device="cuda"), q)
    ctx.close()
