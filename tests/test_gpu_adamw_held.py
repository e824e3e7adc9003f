"""AdamW and weights whose memory changes hands: what a weight had is not given to anyone before the next step, so another tensor, of
another size, cannot be taken for it by its address."""
import pytest
import torch

from paper_2602_03067_amd import binding
from tests._gpu_common import say

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [32, 8])
def test_memory_is_kept_until_the_next_step(bits):
    say("adamw held %d" % bits)
    ctx = binding.Context(0)
    p = torch.nn.Parameter(torch.zeros(1000, device="cuda"))
    opt = binding.AdamW(ctx, [p], lr=0.1, state_bits=bits)
    g = torch.ones(1000, device="cuda")
    opt.step([g])
    first = p.data_ptr()
    p.data = torch.zeros(1000, device="cuda")
    taken = [torch.zeros(900, device="cuda") for _ in range(50)]   # (of the same 4 KB)
    assert all(t.data_ptr() != first for t in taken)
    p.data = taken[-1]
    with pytest.raises(ValueError):
        opt.step([g])
    p.data = torch.zeros(1000, device="cuda")
    opt.step([g])
    assert (p.data < 0).all() and all((t == 0).all() for t in taken)
    ctx.close()


def test_state_is_kept():
    say("adamw held state")
    ctx = binding.Context(0)
    p = torch.nn.Parameter(torch.zeros(1000, device="cuda"))
    opt = binding.AdamW(ctx, [p], lr=0.1)
    at = opt.m[0].data_ptr(), opt.v[0].data_ptr()
    opt.m[0].data = torch.zeros(1000, device="cuda")
    opt.v[0].data = torch.zeros(1000, device="cuda")
    taken = [torch.zeros(1000, device="cuda") for _ in range(50)]
    assert not {t.data_ptr() for t in taken} & set(at)
    opt.step([torch.ones(1000, device="cuda")])
    torch.cuda.synchronize()
    assert all((t == 0).all() for t in taken)
    ctx.close()
