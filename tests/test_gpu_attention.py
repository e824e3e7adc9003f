"""Attention, forward and backward, against the definition in 64 bits.

Tolerances (relative, 2-norm over a tensor).  float32: a score of size S is off by some 2^-23 S (its sum, its scaling, the
argument of exp2), with |s| <= 12 here by 1.5e-6, a probability relatively as much, and sums average it: 1e-5.  bfloat16: the
output's own rounding is 2^-9 / sqrt(3) = 1.1e-3 (uniform, rms), the rounding of the probabilities and of their gradients as
much again each, and as much from the rounded output that the row dots take up: 2.3e-3 where nothing cancels; 6e-3.
Statistics and float32 row dots: 1e-5 in both, of values of bf16 inputs, whose products are exact.
"""
import math

import pytest
import torch

from paper_2602_03067_amd import binding
from tests._gpu_common import say

pytestmark = pytest.mark.gpu

TOL = {torch.float32: 1e-5, torch.bfloat16: 6e-3}
F32, BF16 = torch.float32, torch.bfloat16
LOWEST = torch.finfo(torch.float32).min


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(0)
    yield c
    c.close()


def reference(q, k, v, scale, causal=False, q_len=None, k_len=None, bias=None, do=None):
    """The definition, set by set and head by head, in float64 on the host; only admitted keys are looked at."""
    q, k, v = (t.detach().cpu().double() for t in (q, k, v))
    do = None if do is None else do.detach().cpu().double()
    (B, n, H, d), (m, hk) = q.shape, k.shape[1:3]
    out = dict(o=torch.zeros_like(q), stat=torch.zeros(B, H, n, 2, dtype=torch.float64), dq=torch.zeros_like(q), dk=torch.zeros_like(k),
               dv=torch.zeros_like(v), dbias=torch.zeros(B, m, dtype=torch.float64))
    out["stat"][..., 0] = -math.inf
    for b in range(B):
        nq = n if q_len is None else min(max(int(q_len[b]), 0), n)
        nk = m if k_len is None else min(max(int(k_len[b]), 0), m)
        w = torch.zeros(nk, dtype=torch.float64) if bias is None else bias[b, :nk].detach().cpu().double()
        there = (w > -math.inf).nonzero().flatten()
        if nq == 0 or len(there) == 0:
            continue
        for h in range(H):
            Q, K, V = q[b, :nq, h], k[b, there, h // (H // hk)], v[b, there, h // (H // hk)]
            S = Q @ K.T * scale + w[there]
            if causal:
                S = torch.where(there[None, :] <= torch.arange(nq)[:, None] + nk - nq, S, torch.full_like(S, -math.inf))
            top = S.amax(1)
            seen = top > -math.inf
            P = torch.exp(S - torch.where(seen, top, torch.zeros_like(top))[:, None])
            total = P.sum(1)
            P = P / torch.where(seen, total, torch.ones_like(total))[:, None]
            O = P @ V
            out["o"][b, :nq, h] = O
            out["stat"][b, h, :nq, 0], out["stat"][b, h, :nq, 1] = top, total
            if do is not None:
                G = do[b, :nq, h]
                dS = P * (G @ V.T - (G * O).sum(1, keepdim=True))
                out["dq"][b, :nq, h] = dS @ K * scale
                out["dk"][b, there, h // (H // hk)] += dS.T @ Q * scale
                out["dv"][b, there, h // (H // hk)] += P.T @ G
                out["dbias"][b, there] += dS.sum(0)
    return out


def close(name, got, want, tol, floor=0.0):
    got, want = got.detach().cpu().double(), want.double()
    assert got.shape == want.shape, name
    inf = torch.isinf(want)
    assert torch.equal(torch.isinf(got) & (got < 0), inf), name
    got, want = got[~inf], want[~inf]
    assert torch.isfinite(got).all(), name
    off, size = (got - want).norm().item(), want.norm().item()
    assert off <= tol * max(size, floor), "%s: off by %.3g of %.3g" % (name, off, size)


def check(ctx, q, k, v, do, causal=False, q_len=None, k_len=None, bias=None, scale=None, floor=0.0):
    sc = q.shape[-1] ** -0.5 if scale is None else scale
    tol = TOL[q.dtype]
    o, stat = ctx.fs_attention(q, k, v, scale, causal, q_len, k_len, bias)
    want = reference(q, k, v, sc, causal, q_len, k_len, bias, do)
    close("o", o, want["o"], tol)
    close("stat", stat, want["stat"], 1e-5)
    got = ctx.fs_attention_grad(q, k, v, o, stat, do, scale, causal, q_len, k_len, bias, want_bias=bias is not None)
    for name, t in zip(("dq", "dk", "dv", "dbias"), got):
        close(name, t, want[name], tol, floor)
    return o, stat, got


def normal(seed, dtype, *shape):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(*shape, generator=g).to(dtype).cuda()


def case(seed, dtype, B, n, m, H, hk, d):
    return (normal(seed, dtype, B, n, H, d), normal(seed + 1, dtype, B, m, hk, d), normal(seed + 2, dtype, B, m, hk, d),
            normal(seed + 3, dtype, B, n, H, d))


SHAPES = [
    # B, n, m, H, kv, d
    (1, 1, 2, 1, 1, 64), (2, 31, 33, 2, 1, 32), (1, 64, 64, 1, 1, 64), (2, 65, 63, 4, 2, 40), (1, 129, 128, 2, 2, 128),
    (3, 100, 257, 3, 3, 96), (1, 200, 90, 8, 1, 72), (2, 33, 300, 6, 2, 8), (1, 333, 511, 1, 1, 128), (1, 257, 129, 2, 1, 80),
]
ODD = [(1, 50, 70, 2, 1, 1), (2, 40, 65, 2, 2, 13), (1, 130, 131, 3, 1, 33), (1, 70, 40, 2, 2, 100), (1, 33, 200, 1, 1, 127)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("shape", SHAPES + ODD)
def test_shapes(ctx, shape, causal, dtype):
    say("attention %s causal=%s %s" % (shape, causal, dtype))
    q, k, v, do = case(1, dtype, *shape)
    # (few coordinates: rows that see one key have no gradient of their scores, the rounding of o stands beside it)
    check(ctx, q, k, v, do, causal, floor=0.05 * math.sqrt(q.numel()) if causal or shape[2] <= 2 else 0.0)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_one_key_gives_its_value(ctx, dtype):
    say("attention one key %s" % dtype)
    q, k, v, do = case(5, dtype, 2, 37, 1, 2, 2, 64)
    o, stat = ctx.fs_attention(q, k, v)
    assert torch.equal(o, v.expand_as(o))
    # (bfloat16: the maximum is taken off the score in one fma, after it was rounded: 2^-24 |s| log2 e)
    assert (stat[..., 1] - 1).abs().max() <= (0.0 if dtype == F32 else 2e-6)
    dq, dk, dv = ctx.fs_attention_grad(q, k, v, o, stat, do)
    # p = 1, <do, v> - <do, o> = 0 up to fp32 sums of 64 terms
    assert dq.float().abs().max() < 1e-4 and dk.float().abs().max() < 1e-3
    close("dv", dv, do.cpu().double().sum(1, keepdim=True), TOL[dtype])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("causal", [False, True])
def test_lengths(ctx, causal, dtype):
    say("attention lengths causal=%s %s" % (causal, dtype))
    q, k, v, do = case(11, dtype, 6, 75, 140, 4, 2, 64)
    q_len = torch.tensor([75, 0, 1, 70, 64, 500], dtype=torch.int32).cuda()
    k_len = torch.tensor([140, 30, 128, 1, 0, 65], dtype=torch.int32).cuda()   # (one is empty, one longer queries than keys)
    # what lies beyond the lengths is not looked at
    for b in range(6):
        q[b, q_len[b]:] = math.nan
        do[b, q_len[b]:] = math.inf
        k[b, k_len[b]:] = math.nan
        v[b, k_len[b]:] = math.inf
    o, stat, grads = check(ctx, q, k, v, do, causal, q_len, k_len)
    assert (o[1] == 0).all() and (o[4] == 0).all() and (stat[4, :, :, 1] == 0).all() and (o[3, 70:] == 0).all()
    assert (grads[0][4] == 0).all() and (grads[1][0, 140:] == 0).all() and (grads[2][3, 1:] == 0).all() and (grads[1][1] == 0).all()
    if causal:   # more queries than keys: the first of them see nothing
        assert (o[3, :69] == 0).all() and (o[3, 69] != 0).any()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,m", [(70, 130), (1, 3000), (300, 45)])
def test_bias_removes_keys_and_rows(ctx, n, m, dtype):
    say("attention bias n=%d m=%d %s" % (n, m, dtype))
    q, k, v, do = case(21, dtype, 3, n, m, 4, 2, 40)
    g = torch.Generator().manual_seed(3)
    bias = torch.log(torch.rand(3, m, generator=g) + 0.25)
    bias[torch.rand(3, m, generator=g) < 0.3] = -math.inf
    bias[2] = -math.inf   # nothing left
    bias = bias.cuda()
    gone = (bias == -math.inf)
    k[gone] = math.nan
    v[gone] = math.inf
    o, stat, grads = check(ctx, q, k, v, do, False, None, None, bias)
    assert (o[2] == 0).all() and (stat[2, ..., 0] == -math.inf).all() and (stat[2, ..., 1] == 0).all()
    for t in grads[:3]:
        assert (t[2] == 0).all()
    assert (grads[3][gone] == 0).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_lowest_bias_is_a_number(ctx, dtype):
    """Masks of the type's lowest value: beside other keys they leave nothing, alone they are a uniform average, whose backward pass
    needs the number of keys that the maximum alone cannot carry."""
    say("attention lowest bias %s" % dtype)
    q, k, v, do = case(31, dtype, 2, 40, 100, 2, 2, 64)
    bias = torch.zeros(2, 100).cuda()
    bias[0, 50:] = LOWEST
    bias[1] = LOWEST
    o, stat = ctx.fs_attention(q, k, v, bias=bias)
    cut = reference(q[:1], k[:1, :50], v[:1, :50], 0.125, do=do[:1])
    close("o", o[:1], cut["o"], TOL[dtype])
    close("o", o[1:], v[1:].cpu().double().mean(1, keepdim=True).expand(1, 40, 2, 64), TOL[dtype])
    dq, dk, dv, db = ctx.fs_attention_grad(q, k, v, o, stat, do, bias=bias, want_bias=True)
    close("dv", dv[1:], (do[1:].cpu().double().sum(1, keepdim=True) / 100).expand(1, 100, 2, 64), TOL[dtype])
    close("dk", dk[:1, :50], cut["dk"], TOL[dtype])
    assert (dk[:1, 50:] == 0).all() and torch.isfinite(dq.float()).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_infinite_scores_of_removed_keys(ctx, dtype):
    """Keys beyond the causal line hold infinities: rows that do not see them are as without them."""
    say("attention infinities beyond the line %s" % dtype)
    q, k, v, do = case(41, dtype, 1, 64, 64, 1, 1, 32)
    want = reference(q, k, v, 32 ** -0.5, True)
    k[0, 40:] = math.inf
    o, _ = ctx.fs_attention(q, k, v, causal=True)
    close("o", o[:, :40], want["o"][:, :40], TOL[dtype])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("layout", ["packed", "heads first", "spaced", "shifted"])
def test_strides(ctx, layout, dtype):
    say("attention strides %s %s" % (layout, dtype))
    B, n, H, d = 2, 75, 3, 48
    if layout == "packed":
        q, k, v = normal(51, dtype, B, n, 3, H, d).unbind(2)
        do = normal(52, dtype, B, n, H, d)
    elif layout == "heads first":
        q, k, v, do = (normal(53 + i, dtype, B, H, n, d).transpose(1, 2) for i in range(4))
    elif layout == "spaced":
        q, k, v, do = (normal(57 + i, dtype, B, n + 2, H + 1, d + 5)[:, 1:n + 1, :H, 2:d + 2] for i in range(4))
    else:   # contiguous, but not aligned to more than an element
        q, k, v, do = (normal(61 + i, dtype, B * n * H * d + 1)[1:].view(B, n, H, d) for i in range(4))
    check(ctx, q, k, v, do, True)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_broadcast_inputs(ctx, dtype):
    say("attention broadcast %s" % dtype)
    q, do = normal(71, dtype, 3, 50, 2, 32), normal(72, dtype, 3, 50, 2, 32)
    k, v = normal(73, dtype, 1, 70, 2, 32).expand(3, 70, 2, 32), normal(74, dtype, 1, 70, 2, 32).expand(3, 70, 2, 32)
    check(ctx, q, k, v, do)
    bias = torch.randn(1, 70, generator=torch.Generator().manual_seed(1)).cuda().expand(3, 70)
    o, _ = ctx.fs_attention(q, k, v, bias=bias)
    close("o", o, reference(q, k, v, 32 ** -0.5, bias=bias)["o"], TOL[dtype])
    with pytest.raises(binding.FlashSinkError):
        ctx.fs_attention_grad(q, k, v, o, _, do, bias=bias, want_bias=True)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,n,m,H,hk,d", [(2, 1, 5003, 8, 2, 128), (1, 3, 2000, 4, 4, 64), (1, 2500, 37, 2, 1, 64), (1, 1, 70001, 1, 1, 32),
                                          (2, 7, 1111, 12, 4, 56)])
def test_long_sides(ctx, B, n, m, H, hk, d, dtype):
    """Few rows over many keys and the other way round: the long side is split and merged."""
    say("attention long %s" % ((B, n, m, H, hk, d, dtype),))
    q, k, v, do = case(81, dtype, B, n, m, H, hk, d)
    k_len = torch.tensor([m - 100 * b - 1 for b in range(B)], dtype=torch.int32).clamp(min=1).cuda()
    check(ctx, q, k, v, do, False, None, k_len)
    check(ctx, q, k, v, do, n < m)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_no_rows_and_no_keys(ctx, dtype):
    say("attention empty %s" % dtype)
    q, k, v, do = case(91, dtype, 2, 5, 0, 2, 2, 16)
    o, stat, grads = check(ctx, q, k, v, do)
    assert (o == 0).all() and (grads[0] == 0).all()
    q, k, v, do = case(92, dtype, 2, 0, 5, 2, 2, 16)
    o, stat, grads = check(ctx, q, k, v, do)
    assert (grads[1] == 0).all() and (grads[2] == 0).all()
    q, k, v, do = case(93, dtype, 0, 4, 5, 2, 2, 16)
    check(ctx, q, k, v, do)


def test_large_scores(ctx):
    """Scores far apart: the running reference moves many times, and the largest must not overflow."""
    say("attention large scores")
    q, k, v, do = case(101, F32, 1, 60, 500, 1, 1, 32)
    k = k * torch.linspace(0.1, 30.0, 500, device="cuda").view(1, -1, 1, 1)
    # (scores up to some 500: off by 500 2^-22)
    o, stat = ctx.fs_attention(q, k, v)
    want = reference(q, k, v, 32 ** -0.5)
    close("o", o, want["o"], 5e-4)
    assert (stat[..., 1].cpu().double() >= 1.0 - 1e-6).all()


def test_offsets_beyond_32_bits(ctx):
    say("attention offsets")
    row = 1 << 20
    room = torch.empty(row * 2100 + 64, dtype=BF16, device="cuda")   # 4.4 GB, of which the rows alone are written
    k = room.as_strided((1, 2100, 1, 64), (0, row, 64, 1))
    k.copy_(normal(111, BF16, 1, 2100, 1, 64))
    q, v, do = normal(112, BF16, 1, 3, 1, 64), normal(113, BF16, 1, 2100, 1, 64), normal(114, BF16, 1, 3, 1, 64)
    check(ctx, q, k, v, do)
    check(ctx, q, v, k, do)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_same_call_same_bits(ctx, dtype):
    say("attention twice %s" % dtype)
    q, k, v, do = case(121, dtype, 1, 300, 2000, 4, 1, 64)
    a = ctx.fs_attention(q, k, v)
    ga = ctx.fs_attention_grad(q, k, v, *a, do)
    other = case(131, dtype, 3, 40, 700, 2, 2, 32)   # (the workspace is used for something else in between)
    b = ctx.fs_attention(*other[:3])
    ctx.fs_attention_grad(*other[:3], *b, other[3])
    c = ctx.fs_attention(q, k, v)
    gc = ctx.fs_attention_grad(q, k, v, *c, do)
    for x, y in zip((*a, *ga), (*c, *gc)):
        assert torch.equal(x, y)


def test_other_stream():
    say("attention on a stream of its own")
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        c = binding.Context(0)
        q, k, v, do = case(141, BF16, 2, 100, 3000, 2, 2, 64)
        check(c, q, k, v, do)
    s.synchronize()
    c.close()


def test_differences(ctx):
    """Directional derivatives of <w, o> against central differences of the forward pass: truncation and fp32 noise are both some 1e-4 of the
    product of the norms at h = 1e-2; 2e-3."""
    say("attention differences")
    q, k, v, w = case(151, F32, 2, 20, 50, 2, 1, 24)
    bias = torch.randn(2, 50, generator=torch.Generator().manual_seed(2)).cuda()
    lens = torch.tensor([50, 33], dtype=torch.int32).cuda()
    o, stat = ctx.fs_attention(q, k, v, k_len=lens, bias=bias, causal=True)
    grads = ctx.fs_attention_grad(q, k, v, o, stat, w, k_len=lens, bias=bias, causal=True, want_bias=True)
    h = 1e-2
    for i in range(4):
        args = [q, k, v, bias]
        e = torch.randn(args[i].shape, generator=torch.Generator().manual_seed(160 + i)).cuda()
        vals = []
        for sign in (1, -1):
            a = list(args)
            a[i] = args[i] + sign * h * e
            vals.append((ctx.fs_attention(a[0], a[1], a[2], k_len=lens, bias=a[3], causal=True)[0].double() * w.double()).sum().item())
        slope, want = (vals[0] - vals[1]) / (2 * h), (grads[i].double() * e.double()).sum().item()
        assert abs(slope - want) <= 2e-3 * grads[i].double().norm().item() * e.double().norm().item(), i


def test_refusals(ctx):
    q, k, v, do = case(171, F32, 1, 4, 6, 2, 1, 16)
    o, stat = ctx.fs_attention(q, k, v)
    for bad in (lambda: ctx.fs_attention(q.cpu(), k, v), lambda: ctx.fs_attention(q, k.to(BF16), v),
                lambda: ctx.fs_attention(q, k, v, bias=torch.zeros(6).cuda()), lambda: ctx.fs_attention(q.half(), k.half(), v.half()),
                lambda: ctx.fs_attention(q, k, v, k_len=torch.tensor([3]).cuda())):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: ctx.fs_attention(q, k, v[:, :5]), lambda: ctx.fs_attention(q[..., ::2], k[..., ::2], v[..., ::2]),
                lambda: ctx.fs_attention_grad(q, k, v, o, stat, do, want_bias=True),
                lambda: ctx.fs_attention_grad(q, k, v, o, stat[:, :1].contiguous(), do)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: ctx.fs_attention(q, k, v, scale=0.0), lambda: ctx.fs_attention(q, k, v, scale=math.nan),
                lambda: ctx.fs_attention(*case(1, F32, 1, 4, 6, 3, 2, 16)[:3]), lambda: ctx.fs_attention(*case(1, F32, 1, 4, 6, 2, 1, 136)[:3])):
        with pytest.raises(binding.FlashSinkError):
            bad()
