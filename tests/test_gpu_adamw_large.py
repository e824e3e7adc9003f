"""AdamW over more weights than one launch has threads for: a tensor goes on in the next launch."""
import pytest
import torch

from paper_2602_03067_amd import binding
from tests._gpu_common import say

pytestmark = pytest.mark.gpu


def test_seventeen_billion_weights():
    """2^34 bf16 weights and some with 8-bit state, 103 GB, and a small tensor behind them.  All gradients are one: m = 0.1, v = 0.001, an update
    is lr (rounded to bf16, from a weight of zero); codes are one of the two neighbours of 0.1 and of the root of 0.001, each in every place."""
    n, few = (1 << 34) + 1301, 700
    if torch.cuda.mem_get_info()[0] < 140 << 30:
        pytest.skip("less than 140 GB of GPU memory")
    say("adamw 2^34 weights")
    torch.cuda.empty_cache()
    ctx = binding.Context(0)
    f8 = torch.float8_e4m3fn
    p = [torch.zeros(k, dtype=torch.bfloat16, device="cuda") for k in (n, few)]
    m, v = ([torch.zeros(k, dtype=torch.uint8, device="cuda").view(f8) for k in (n, few)] for _ in range(2))
    sm, sv = ([torch.ones((k + 255) // 256, device="cuda") for k in (n, few)] for _ in range(2))
    g = [torch.ones(k, dtype=torch.bfloat16, device="cuda") for k in (n, few)]
    opt = binding.AdamW(ctx, p, lr=0.25, state_bits=8, m=m, v=v, m_scale=sm, v_scale=sv)
    opt.step(g)
    torch.cuda.synchronize()
    part = 1 << 30
    for i, k in enumerate((n, few)):
        for a in range(0, k, part):
            moved = bool((p[i][a:a + part] == -0.25).all())
            assert moved, (i, a)
            for code, scale, value in ((m, sm, 0.1), (v, sv, 0.001 ** 0.5)):
                sc = scale[i][0].item()   # (of every block: its weights are equal)
                got = code[i][a:a + part].view(torch.uint8)
                low = int(got.min().item())
                lo, hi = (torch.tensor([c], dtype=torch.uint8).view(f8).float().item() * sc for c in (low, low + 1))
                assert lo <= value * (1 + 1e-6) and hi >= value * (1 - 1e-6) and int(got.max().item()) <= low + 1, (i, a)
        alike = bool((sm[i] == sm[i][0]).all() and (sv[i] == sv[i][0]).all())
        assert alike
    # numbered on through the tensor: the same stretch in another place is rounded up in other places
    at = [m[0][a:a + part].view(torch.uint8) for a in (0, (1 << 34) - part)]
    same = torch.equal(*at)
    assert not same
    ctx.close()
    del p, m, v, sm, sv, g, opt, at, got
    torch.cuda.empty_cache()
