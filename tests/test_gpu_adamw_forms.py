"""AdamW with 8-bit state and bf16 weights without float masters, for every type of gradient.  Formulas and tolerances are those of
test_gpu_adamw.py; a weight is rounded to bf16, 2^-8 of it."""
import pytest
import torch

from paper_2602_03067_amd import binding
from tests._gpu_common import say
from tests.test_gpu_adamw import BF16, F32, SIZES, decoded, exact, normal

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("ptype,gtype", [(BF16, BF16), (BF16, F32), (F32, BF16)])
def test_step_8bit_without_masters(ptype, gtype):
    say("adamw 8 without masters %s %s" % (ptype, gtype))
    ctx = binding.Context(0)
    p = [normal(i, ptype, n) for i, n in enumerate(SIZES)]
    opt = binding.AdamW(ctx, p, lr=1e-2, weight_decay=0.01, state_bits=8)
    for t in range(1, 6):
        g = [normal(200 * t + i, gtype, n) * torch.exp(3 * normal(300 + i, F32, n)).to(gtype) for i, n in enumerate(SIZES)]
        before = [x.clone() for x in p]
        m = [decoded(c, s) for c, s in zip(opt.m, opt.m_scale)]
        r = [decoded(c, s) for c, s in zip(opt.v, opt.v_scale)]
        opt.step(g)
        for i, n in enumerate(SIZES):
            if not n:
                continue
            wp, wm, wv, step = exact(before[i], g[i], m[i], r[i].double().square(), t)
            ulp = 2.0 ** -8 if ptype == BF16 else 2.0 ** -23
            assert ((p[i].double() - wp).abs() <= step + ulp * wp.abs() + 1e-30).all(), (t, i)
            for code, scale, val in ((opt.m[i], opt.m_scale[i], wm), (opt.v[i], opt.v_scale[i], wv.sqrt())):
                sc = scale.repeat_interleave(256)[:n].double()
                width = torch.maximum(val.abs() / sc / 8, torch.full_like(val, 2.0 ** -9)) * sc
                assert ((decoded(code, scale).double() - val).abs() <= width * (1 + 1e-5)).all(), (t, i)
    ctx.close()
