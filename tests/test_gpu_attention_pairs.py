"""float32 attention through pairs of fp16, forced at small sizes, against the definition in 64 bits.

Tolerance: 1e-5 (relative, 2-norm), that of the fp32 matrix cores: operands carry 22 bits, so a product is off by 2^-21 of itself, a score
|s| <= 12 by 12 2^-21 / sqrt(d) = 7e-7 at d = 64 (and 5.7e-6 if all errors of a score had one sign), a probability relatively as much."""
import math

import pytest
import torch

from paper_2602_03067_amd import binding
from tests._gpu_common import say
from tests.test_gpu_attention import F32, ODD, SHAPES, case, check, close, normal, reference

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(0)
    c.fs_debug_set("attn_pairs", 1)
    yield c
    c.close()


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("shape", SHAPES + ODD)
def test_shapes(ctx, shape, causal):
    say("pairs %s causal=%s" % (shape, causal))
    q, k, v, do = case(1, F32, *shape)
    check(ctx, q, k, v, do, causal, floor=0.05 * math.sqrt(q.numel()) if causal or shape[2] <= 2 else 0.0)


@pytest.mark.parametrize("causal", [False, True])
def test_lengths_and_what_lies_beyond(ctx, causal):
    say("pairs lengths causal=%s" % causal)
    q, k, v, do = case(11, F32, 6, 75, 140, 4, 2, 64)
    q_len = torch.tensor([75, 0, 1, 70, 64, 500], dtype=torch.int32).cuda()
    k_len = torch.tensor([140, 30, 128, 1, 0, 65], dtype=torch.int32).cuda()
    for b in range(6):
        q[b, q_len[b]:] = math.nan
        do[b, q_len[b]:] = math.inf
        k[b, k_len[b]:] = 1e30   # (and it does not set a scale)
        v[b, k_len[b]:] = math.inf
    o, stat, grads = check(ctx, q, k, v, do, causal, q_len, k_len)
    assert (o[1] == 0).all() and (o[4] == 0).all() and (grads[0][4] == 0).all() and (grads[2][3, 1:] == 0).all()


@pytest.mark.parametrize("n,m", [(70, 130), (1, 3000), (300, 45)])
def test_bias(ctx, n, m):
    say("pairs bias n=%d m=%d" % (n, m))
    q, k, v, do = case(21, F32, 3, n, m, 4, 2, 40)
    g = torch.Generator().manual_seed(3)
    bias = torch.log(torch.rand(3, m, generator=g) + 0.25)
    bias[torch.rand(3, m, generator=g) < 0.3] = -math.inf
    bias[2] = -math.inf
    bias = bias.cuda()
    gone = bias == -math.inf
    k[gone], v[gone] = math.nan, math.inf
    o, stat, grads = check(ctx, q, k, v, do, False, None, None, bias)
    assert (o[2] == 0).all() and (grads[3][gone] == 0).all()


@pytest.mark.parametrize("layout", ["packed", "heads first", "shifted"])
def test_strides(ctx, layout):
    say("pairs strides %s" % layout)
    B, n, H, d = 2, 75, 3, 48
    if layout == "packed":
        q, k, v = normal(51, F32, B, n, 3, H, d).unbind(2)
        do = normal(52, F32, B, n, H, d)
    elif layout == "heads first":
        q, k, v, do = (normal(53 + i, F32, B, H, n, d).transpose(1, 2) for i in range(4))
    else:
        q, k, v, do = (normal(61 + i, F32, B * n * H * d + 1)[1:].view(B, n, H, d) for i in range(4))
    check(ctx, q, k, v, do, True)


@pytest.mark.parametrize("B,n,m,H,hk,d", [(2, 1, 5003, 8, 2, 128), (1, 2500, 37, 2, 1, 64), (1, 200, 7001, 4, 4, 32)])
def test_long_sides(ctx, B, n, m, H, hk, d):
    say("pairs long %s" % ((B, n, m, H, hk, d),))
    q, k, v, do = case(81, F32, B, n, m, H, hk, d)
    check(ctx, q, k, v, do, n < m)


@pytest.mark.parametrize("sizes", [(1e-20, 1e-15, 1e25, 1e-25), (3e4, 1e-6, 1e-30, 1e30), (1e18, 1e-18, 7.0, 1e-3)])
def test_any_size_of_values(ctx, sizes):
    say("pairs sizes %s" % (sizes,))
    q, k, v, do = (t * s for t, s in zip(case(91, F32, 2, 90, 150, 2, 1, 64), sizes))
    check(ctx, q, k, v, do, scale=0.125 / (sizes[0] * sizes[1]))


def test_heads_and_rows_of_unequal_size(ctx):
    """A scale belongs to a head; inside a head the rows' sizes are spread over 2^20."""
    say("pairs unequal rows")
    q, k, v, do = case(95, F32, 2, 100, 160, 4, 4, 64)
    v = v * torch.exp2(torch.linspace(-20, 0, 160)).cuda().view(1, -1, 1, 1) * torch.tensor([1.0, 1e-8, 1e8, 1.0]).cuda().view(1, 1, 4, 1)
    do = do * torch.exp2(torch.linspace(0, -12, 100)).cuda().view(1, -1, 1, 1)
    o, stat = ctx.fs_attention(q, k, v)
    want = reference(q, k, v, 0.125, do=do)
    grads = ctx.fs_attention_grad(q, k, v, o, stat, do)
    for h in range(4):
        close("o", o[:, :, h], want["o"][:, :, h], 1e-5)
        for name, t in zip(("dq", "dk", "dv"), grads):
            close(name, t[:, :, h], want[name][:, :, h], 1e-5)


def test_large_scores(ctx):
    say("pairs large scores")
    q, k, v, do = case(101, F32, 1, 60, 500, 1, 1, 32)
    k = k * torch.linspace(0.1, 30.0, 500, device="cuda").view(1, -1, 1, 1)
    o, stat = ctx.fs_attention(q, k, v)
    close("o", o, reference(q, k, v, 32 ** -0.5)["o"], 5e-4)   # (scores up to some 500: off by 500 2^-21)


def test_both_ways_agree_and_are_chosen_by_size(ctx):
    say("pairs by size")
    plain, free = binding.Context(0), binding.Context(0)
    plain.fs_debug_set("attn_pairs", 2)
    q, k, v, do = case(111, F32, 1, 1024, 2048, 8, 8, 64)
    a, b, c = (x.fs_attention(q, k, v)[0] for x in (plain, ctx, free))
    assert torch.equal(b, c) and not torch.equal(a, b)
    assert ((a - b).norm() <= 1e-5 * a.norm()).item()
    q, k, v, do = case(112, F32, 1, 64, 64, 1, 1, 64)
    a, c = (x.fs_attention(q, k, v)[0] for x in (plain, free))
    assert torch.equal(a, c)
    plain.close()
    free.close()


def test_same_call_same_bits(ctx):
    say("pairs twice")
    q, k, v, do = case(121, F32, 1, 300, 2000, 4, 1, 64)
    a = ctx.fs_attention(q, k, v)
    ga = ctx.fs_attention_grad(q, k, v, *a, do)
    b = ctx.fs_attention(q, k, v)
    gb = ctx.fs_attention_grad(q, k, v, *b, do)
    assert all(torch.equal(x, y) for x, y in zip((*a, *ga), (*b, *gb)))
