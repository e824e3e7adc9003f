"""AdamW over many tensors against the formulas in 64 bits.

Tolerances: m and v are two roundings of 2^-24 from exact: 3e-7 relative per element of the sum's terms; the update of a weight is
off by some ulps of fp32 (root, reciprocal, products: 1e-6 of it) and by what m is off by, which where m's two terms cancel is not
a share of m, and the weight by its own rounding.  Codes of 8-bit states
are one of the two neighbours of the value: up to a step of 2^-3 of it (2^-9 of the scale below 2^-6)."""
import math

import pytest
import torch

from paper_2602_03067_amd import binding
from tests._gpu_common import say

pytestmark = pytest.mark.gpu
F32, BF16, F8 = torch.float32, torch.bfloat16, torch.float8_e4m3fn


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(0)
    yield c
    c.close()


def normal(seed, dtype, n):
    return torch.randn(n, generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()


def exact(p, g, m, v, t, lr=1e-2, b1=0.9, b2=0.999, eps=1e-8, wd=0.01):
    p, g, m, v = (x.double() for x in (p, g, m, v))
    terms = m.abs() + g.abs()
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g * g
    rate = lr / (1 - b1 ** t) / ((v / (1 - b2 ** t)).sqrt() + eps)
    # (and how far an update may be off)
    return p * (1 - lr * wd) - rate * m, m, v, rate * (2e-6 * m.abs() + 3e-7 * terms)


def decoded(code, scale):
    n = code.numel()
    return code.float() * scale.repeat_interleave(256)[:n]


SIZES = [1, 3, 4, 5, 255, 256, 257, 1000, 4095, 4096, 4097, 12345, 0, 70001]


@pytest.mark.parametrize("master", [False, True])
@pytest.mark.parametrize("ptype,gtype", [(F32, F32), (F32, BF16), (BF16, BF16), (BF16, F32)])
def test_steps_32bit(ctx, ptype, gtype, master):
    if master and ptype == F32:
        return
    say("adamw 32 %s %s master=%s" % (ptype, gtype, master))
    p = [normal(i, ptype, n) for i, n in enumerate(SIZES)]
    ms = [x.float() for x in p] if master else None
    opt = binding.AdamW(ctx, p, lr=1e-2, weight_decay=0.01, master=ms)
    for t in (1, 2, 3):
        g = [normal(100 * t + i, gtype, n) for i, n in enumerate(SIZES)]
        before = [(x.clone(), m.clone(), v.clone()) for x, m, v in zip(ms or p, opt.m, opt.v)]
        opt.step(g)
        for i, (w, m, v) in enumerate(before):
            wp, wm, wv, step = exact(w, g[i], m, v, t)
            got = (ms or p)[i].double()
            ulp = 2.0 ** -8 if (ptype == BF16 and not master) else 2.0 ** -23
            assert ((got - wp).abs() <= step + ulp * wp.abs() + 1e-30).all(), (t, i)
            if master:
                assert torch.equal(p[i], ms[i].to(BF16))
            assert ((opt.m[i].double() - wm).abs() <= 3e-7 * (m.double().abs() + g[i].double().abs())).all()
            assert ((opt.v[i].double() - wv).abs() <= 3e-7 * wv).all()


@pytest.mark.parametrize("shift", [1, 2, 4])
@pytest.mark.parametrize("bits", [32, 8])
def test_alignment(ctx, shift, bits):
    """Tensors that begin anywhere give what aligned ones give, and nothing beside them is touched."""
    say("adamw alignment %d %d" % (shift, bits))
    n = 1300
    outs = []
    for s in (0, shift):
        kind = F32 if bits == 32 else F8
        room = [normal(7, F32, n + 16), normal(8, F32, n + 16) * 0.1, torch.zeros(n + 16).cuda().to(kind), torch.zeros(n + 16).cuda().to(kind)]
        p, m, v = (torch.zeros(n + 16).cuda().to(x.dtype) for x in (room[0], room[2], room[3]))
        p[s:s + n] = room[0][:n]
        g = torch.zeros(n + 16).cuda()
        g[s:s + n] = room[1][:n]
        sc = dict(m_scale=[torch.ones(6).cuda()], v_scale=[torch.ones(6).cuda()]) if bits == 8 else {}
        opt = binding.AdamW(ctx, [p[s:s + n]], lr=1e-2, state_bits=bits, m=[m[s:s + n]], v=[v[s:s + n]], **sc)
        opt.step([g[s:s + n]])
        opt.step([g[s:s + n]])
        for x in (p, m, v):
            x = x.float()
            assert (x[:s] == 0).all() and (x[s + n:] == 0).all()
        outs.append([x[s:s + n].float().clone() for x in (p, m, v)])
    for a, b in zip(*outs):
        assert torch.equal(a, b)


@pytest.mark.parametrize("ptype", [F32, BF16])
def test_step_8bit(ctx, ptype):
    say("adamw 8 %s" % ptype)
    p = [normal(i, ptype, n) for i, n in enumerate(SIZES)]
    opt = binding.AdamW(ctx, p, lr=1e-2, weight_decay=0.01, state_bits=8, master=[x.float() for x in p] if ptype == BF16 else None)
    for t in range(1, 6):
        # gradients over many sizes: blocks with large and small weights
        g = [normal(200 * t + i, ptype, n) * torch.exp(3 * normal(300 + i, F32, n)).to(ptype) for i, n in enumerate(SIZES)]
        w = [x.clone() for x in (opt.master or p)]
        m = [decoded(c, s) for c, s in zip(opt.m, opt.m_scale)]
        r = [decoded(c, s) for c, s in zip(opt.v, opt.v_scale)]
        opt.step(g)
        for i in range(len(SIZES)):
            if not SIZES[i]:
                continue
            wp, wm, wv, step = exact(w[i], g[i], m[i], r[i].double().square(), t)
            assert (((opt.master or p)[i].double() - wp).abs() <= step + 2.0 ** -23 * wp.abs()).all(), (t, i)
            for code, scale, val in ((opt.m[i], opt.m_scale[i], wm), (opt.v[i], opt.v_scale[i], wv.sqrt())):
                sc = scale.repeat_interleave(256)[:len(val)].double()
                step8 = torch.maximum(val.abs() / sc / 8, torch.full_like(val, 2.0 ** -9)) * sc
                assert ((decoded(code, scale).double() - val).abs() <= step8 * (1 + 1e-5)).all(), (t, i)
                assert torch.equal(torch.frexp(scale)[0], torch.full_like(scale, 0.5))   # powers of two
                pad = torch.zeros(len(scale) * 256, dtype=torch.float64, device="cuda")
                pad[:len(val)] = val.abs()
                top = pad.view(-1, 256).amax(1) / scale.double()
                assert ((top <= 448 * (1 + 1e-6)) & (top > 224 * (1 - 1e-6))).all()
            assert ((opt.v[i].view(torch.uint8) == 0) == (wv == 0)).all()


def test_codes_are_unbiased(ctx):
    """Over many seeds the mean of the decoded momentum is the value: with N = 64 x 256 roundings of up to an eighth each (rms
    at most 1/16 of a value), the mean relative deviation is below 5 / 16 / sqrt(N) = 2.5e-3 with all but certainty."""
    say("adamw dither")
    n = 256
    g = (torch.rand(n, generator=torch.Generator().manual_seed(1)) + 0.5).cuda()
    total = torch.zeros(n, dtype=torch.float64, device="cuda")
    roots = torch.zeros(n, dtype=torch.float64, device="cuda")
    for seed in range(64):
        p = torch.zeros(n).cuda()
        opt = binding.AdamW(ctx, [p], state_bits=8, seed=1000 * seed)
        opt.step([g])
        total += decoded(opt.m[0], opt.m_scale[0]).double() / (0.1 * g.double())
        roots += decoded(opt.v[0], opt.v_scale[0]).double() / (math.sqrt(0.001) * g.double())
    assert abs(total.mean().item() / 64 - 1) < 2.5e-3 and abs(roots.mean().item() / 64 - 1) < 2.5e-3


def test_small_decay_moves_an_8bit_state(ctx):
    """A second moment that is to grow by 0.1 % a step does grow: after 400 steps of a gradient of one, from a root of 1/4, v is
    1 - (15/16) 0.999^400 = 0.372 on average."""
    say("adamw growth")
    n = 4096
    p, g = torch.zeros(n).cuda(), torch.ones(n).cuda()
    ones = torch.ones(16).cuda() * 2.0 ** -10
    opt = binding.AdamW(ctx, [p], state_bits=8, m=[torch.zeros(n).cuda().to(F8)], v=[torch.full((n,), 256.0).cuda().to(F8)],
                        m_scale=[torch.ones(16).cuda()], v_scale=[ones])
    for _ in range(400):
        opt.step([g])
    v = decoded(opt.v[0], opt.v_scale[0]).double().square().mean().item()
    assert abs(v - 0.372) < 0.05


def test_same_step_same_bits_and_seeds(ctx):
    say("adamw seeds")
    outs = []
    for seed in (5, 5, 6):
        p = [normal(1, F32, 5000), normal(2, F32, 300)]
        opt = binding.AdamW(ctx, p, state_bits=8, seed=seed)
        opt.step([normal(3, F32, 5000), normal(4, F32, 300)])
        outs.append([x.float() for x in (*p, *opt.m, *opt.v)])
    assert all(torch.equal(a, b) for a, b in zip(outs[0], outs[1]))
    assert not torch.equal(outs[0][2], outs[2][2])


def test_many_tensors(ctx):
    """More tensors than a launch has room for addresses: the same as one by one, numbering of the codes apart."""
    say("adamw many")
    sizes = [(37 * i) % 1000 + 1 for i in range(300)]
    p = [normal(i, F32, n) for i, n in enumerate(sizes)]
    q = [x.clone() for x in p]
    g = [normal(1000 + i, F32, n) for i, n in enumerate(sizes)]
    binding.AdamW(ctx, p, lr=1e-2).step(g)
    for x, y in zip(q, g):
        binding.AdamW(ctx, [x], lr=1e-2).step([y])
    assert all(torch.equal(a, b) for a, b in zip(p, q))


def test_grad_scale(ctx):
    say("adamw grad scale")
    p, q, g = normal(1, F32, 777), normal(1, F32, 777), normal(2, F32, 777)
    binding.AdamW(ctx, [p]).step([g], grad_scale=torch.tensor(0.25).cuda())
    binding.AdamW(ctx, [q]).step([g * 0.25])
    assert torch.equal(p, q)


def test_not_finite(ctx):
    """A gradient that is not finite shows: in its weight with float states, in its block's states with 8 bits; others are as without."""
    say("adamw not finite")
    for bits in (32, 8):
        g = normal(1, F32, 600)
        ps = [normal(2, F32, 600), normal(2, F32, 600)]
        opts = [binding.AdamW(ctx, [x], state_bits=bits) for x in ps]
        opts[0].step([g])
        g = g.clone()
        g[300] = math.nan
        opts[1].step([g])
        keep = torch.arange(600) != 300
        assert torch.equal(ps[0][keep], ps[1][keep]) and torch.isnan(ps[1][300])
        if bits == 8:
            assert torch.isnan(opts[1].m_scale[0][1]) and torch.isfinite(opts[1].m_scale[0][[0, 2]]).all()


def test_refusals(ctx):
    p = normal(1, F32, 10)
    for bad in (lambda: binding.AdamW(ctx, []), lambda: binding.AdamW(ctx, [p], state_bits=16), lambda: binding.AdamW(ctx, [p], m=[]),
                lambda: binding.AdamW(ctx, [p]).step([])):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: binding.AdamW(ctx, [p.half()]), lambda: binding.AdamW(ctx, [p, p.to(BF16)]), lambda: binding.AdamW(ctx, [p[::2]]),
                lambda: binding.AdamW(ctx, [p], m=[p[:5]]), lambda: binding.AdamW(ctx, [p]).step([p[:5]]),
                lambda: binding.AdamW(ctx, [p]).step([p.clone()], grad_scale=torch.ones(2).cuda())):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: binding.AdamW(ctx, [p], lr=-1.0).step([p.clone()]), lambda: binding.AdamW(ctx, [p], betas=(1.0, 0.9)).step([p.clone()]),
                lambda: binding.AdamW(ctx, [p]).step([p]), lambda: binding.AdamW(ctx, [p], master=[p.clone()]).step([p.clone()])):
        with pytest.raises(binding.FlashSinkError):
            bad()
