"""float32 gradients through pairs of fp16, row by row: do whose rows differ in size by up to 2^28, probabilities of one and of 1 / keys.

Tolerance, of every row of dq on its own: the operands and the gradients of scores have 22 bits (2^-22 of each, in quadrature), the
scores |s| <= 6 are off by 6 2^-22, and a row dot is a sum of fp32; some 3e-6 of the norm of the row's terms, so 1e-5 of that norm, which
where nothing cancels is the row's own.  dk and dv are sums over rows, of which the largest decide: 1e-5 of a head's."""
import math

import pytest
import torch

from paper_2602_03067_amd import binding
from tests._gpu_common import say
from tests.test_gpu_attention import F32, case, check, close, normal, reference

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(0)
    c.fs_debug_set("attn_pairs", 1)
    yield c
    c.close()


def terms(q, k, v, do, scale, causal):
    """For one set: dq, and for every row the root of the sum of squares of what it is a sum of, in float64 on the GPU."""
    n, H, _ = q.shape
    m, hk, _ = k.shape
    dq, size = torch.zeros_like(q, dtype=torch.float64), torch.zeros(n, H, dtype=torch.float64, device=q.device)
    for h in range(H):
        Q, G, K, V = q[:, h].double(), do[:, h].double(), k[:, h // (H // hk)].double(), v[:, h // (H // hk)].double()
        S = torch.mm(Q, K.t().contiguous()) * scale
        if causal:
            seen = torch.arange(m, device=q.device)[None, :] <= torch.arange(n, device=q.device)[:, None] + m - n
            S = torch.where(seen, S, torch.full_like(S, -math.inf))
        P = torch.nan_to_num(torch.softmax(S, 1), nan=0.0)   # (a row that sees no key)
        dP = torch.mm(G, V.t().contiguous())
        D = (P * dP).sum(1, keepdim=True)
        dq[:, h] = torch.mm(P * (dP - D), K) * scale
        size[:, h] = torch.mm((P * (dP.abs() + D.abs())) ** 2, (K ** 2).sum(1, keepdim=True)).sqrt()[:, 0] * scale
    return dq, size


def rows_close(got, want, size):
    off = (got.double() - want).norm(dim=-1)
    worst = (off / size.clamp_min(1e-300)).max().item()
    assert torch.isfinite(got).all() and (off <= 1e-5 * size).all(), "worst row off by %.3g of its terms" % worst


@pytest.mark.parametrize("spread", [0, 12, 20, 28])
@pytest.mark.parametrize("n,m,H,hk,d", [(256, 160, 2, 2, 64), (1024, 4096, 2, 1, 64), (300, 1000, 4, 4, 40), (512, 9000, 1, 1, 128), (333, 2047, 2, 2, 96)])
@pytest.mark.parametrize("causal", [False, True])
def test_every_row_of_dq(ctx, causal, n, m, H, hk, d, spread):
    say("pairs rows n=%d m=%d heads=%d/%d d=%d causal=%s 2^-%d" % (n, m, H, hk, d, causal, spread))
    q, k, v, do = case(201, F32, 1, n, m, H, hk, d)
    order = torch.randperm(n, generator=torch.Generator().manual_seed(1)).cuda()
    do = do * torch.exp2(-spread * torch.linspace(0, 1, n, device="cuda"))[order].view(1, n, 1, 1)
    o, stat = ctx.fs_attention(q, k, v, causal=causal)
    dq, dk, dv = ctx.fs_attention_grad(q, k, v, o, stat, do, causal=causal)
    want, size = terms(q[0], k[0], v[0], do[0], d ** -0.5, causal)
    rows_close(dq[0], want, size)


@pytest.mark.parametrize("spread", [12, 28])
def test_one_large_row(ctx, spread):
    """All rows but one are small: they and the keys' gradients, which the large row decides."""
    say("pairs one large row 2^-%d" % spread)
    q, k, v, do = case(211, F32, 1, 300, 700, 2, 2, 64)
    do[:, torch.arange(300) != 77] *= 2.0 ** -spread
    o, stat = ctx.fs_attention(q, k, v)
    dq, dk, dv = ctx.fs_attention_grad(q, k, v, o, stat, do)
    rows_close(dq[0], *terms(q[0], k[0], v[0], do[0], 0.125, False))
    want = reference(q, k, v, 0.125, do=do)
    for h in range(2):
        close("dk", dk[:, :, h], want["dk"][:, :, h], 1e-5)
        close("dv", dv[:, :, h], want["dv"][:, :, h], 1e-5)


def test_rows_of_zeros_and_sets_of_zeros(ctx):
    say("pairs rows of zeros")
    q, k, v, do = case(221, F32, 3, 200, 300, 2, 1, 64)
    do[0, ::2] = 0.0
    do[1] = 0.0
    v[2] = 0.0
    _, _, (dq, dk, dv) = check(ctx, q, k, v, do)
    assert (dq[0, ::2] == 0).all() and (dq[1:] == 0).all() and (dk[1:] == 0).all() and (dv[1] == 0).all()


def test_bias_gradient_of_spread_rows(ctx):
    say("pairs bias gradient of spread rows")
    q, k, v, do = case(231, F32, 2, 260, 500, 2, 2, 64)
    do = do * torch.exp2(-20 * torch.linspace(0, 1, 260, device="cuda")).view(1, -1, 1, 1)
    bias = torch.log(torch.rand(2, 500, generator=torch.Generator().manual_seed(3)) + 0.25).cuda()
    check(ctx, q, k, v, do, False, None, torch.tensor([500, 333], dtype=torch.int32).cuda(), bias)


@pytest.mark.parametrize("sizes", [(1e-10, 1e10, 1e-15, 1e-15), (1e-5, 1e20, 1e-25, 1e-18), (1e5, 1e-20, 1e15, 1e20), (1.0, 1.0, 1e20, 1e17)])
def test_products_of_norms_beyond_a_float(ctx, sizes):
    """|do| |v| and what dq is made of leave a float's normal range on the way, or come near; dq does not."""
    say("pairs sizes of v and do %s" % (sizes,))
    q, k, v, do = (t * s for t, s in zip(case(241, F32, 1, 200, 300, 1, 1, 64), sizes))
    scale = 0.125 / (sizes[0] * sizes[1])
    o, stat = ctx.fs_attention(q, k, v, scale)
    dq, _, dv = ctx.fs_attention_grad(q, k, v, o, stat, do, scale)
    want, size = terms(q[0], k[0], v[0], do[0], scale, False)
    rows_close(dq[0], want, size)
    close("dv", dv, reference(q, k, v, scale, do=do)["dv"], 1e-5)


def test_the_way_by_size_is_as_exact(ctx):
    """What a call of some size does by itself, beside the fp32 matrix cores."""
    say("pairs rows by size")
    c = binding.Context(0)
    q, k, v = (normal(251 + i, F32, 1, 2048, 4, 64) for i in range(3))
    do = normal(254, F32, 1, 2048, 4, 64) * torch.exp2(-20 * torch.rand(2048, generator=torch.Generator().manual_seed(5)).cuda()).view(1, -1, 1, 1)
    o, stat = c.fs_attention(q, k, v)
    rows_close(c.fs_attention_grad(q, k, v, o, stat, do)[0][0], *terms(q[0], k[0], v[0], do[0], 0.125, False))
    c.close()
