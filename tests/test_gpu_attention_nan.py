"""NaN in what a row sees shows in that row, however the keys are cut: in one piece, over the waves of a workgroup, over splits."""
import math

import pytest
import torch

from paper_2602_03067_amd import binding
from tests._gpu_common import say
from tests.test_gpu_attention import BF16, F32, TOL, case, close, reference

pytestmark = pytest.mark.gpu

# B, n, m, H, kv, d: one query (32 rows, split), a few, 64-row workgroups whose waves share the keys, 128 rows in splits, one piece
SHAPES = [(2, 1, 5000, 4, 4, 64), (1, 1, 257, 8, 2, 128), (1, 5, 3000, 4, 1, 40), (2, 300, 2000, 2, 2, 64), (1, 1000, 1000, 4, 4, 64),
          (8, 300, 60, 8, 8, 32), (1, 40, 9000, 1, 1, 96)]


@pytest.fixture(scope="module", params=[0, 1], ids=["by size", "pairs"])
def ctx(request):
    c = binding.Context(0)
    c.fs_debug_set("attn_pairs", request.param)
    yield c
    c.close()


def same_but(rows, got, clean, tol):
    """`rows`: which (set, query, head) are NaN; the others are what they are without them."""
    assert torch.isnan(got[rows]).all()
    close("others", got[~rows], clean[~rows].cpu(), tol)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shape", SHAPES)
def test_query(ctx, shape, dtype):
    say("attention NaN query %s %s" % (shape, dtype))
    q, k, v, do = case(5, dtype, *shape)
    clean, clean_stat = ctx.fs_attention(q, k, v)
    b, i, h = shape[0] - 1, shape[1] // 2, shape[3] - 1
    q[b, i, h, shape[5] // 2] = math.nan
    o, stat = ctx.fs_attention(q, k, v)
    rows = torch.zeros(o.shape[:3], dtype=torch.bool, device="cuda")
    rows[b, i, h] = True
    same_but(rows, o, clean, TOL[dtype])
    same_but(rows.transpose(1, 2), stat, clean_stat, 1e-5)
    dq, dk, dv = ctx.fs_attention_grad(q, k, v, o, stat, do)
    assert torch.isnan(dq[b, i, h]).all() and torch.isfinite(dq[~rows].float()).all()
    own = h // (shape[3] // shape[4])
    assert torch.isnan(dk[b, :, own]).all() and torch.isnan(dv[b, :, own]).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("where", ["first", "last", "one"])
def test_run_of_keys(ctx, where, shape, dtype):
    """A stretch of NaN keys that is a whole part of the cut, or one key of it: every row of that head sees it."""
    say("attention NaN keys %s %s %s" % (where, shape, dtype))
    q, k, v, do = case(6, dtype, *shape)
    clean, _ = ctx.fs_attention(q, k, v)
    m = shape[2]
    at = {"first": slice(0, m // 2), "last": slice(m - m // 3, m), "one": slice(m // 2, m // 2 + 1)}[where]
    k[0, at, 0] = math.nan
    o, stat = ctx.fs_attention(q, k, v)
    rows = torch.zeros(o.shape[:3], dtype=torch.bool, device="cuda")
    rows[0, :, :shape[3] // shape[4]] = True
    assert torch.isnan(o[rows]).all() and torch.isnan(stat.transpose(1, 2)[rows]).all()
    if not rows.all():
        close("others", o[~rows], clean[~rows].cpu(), TOL[dtype])


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_before_the_line_do_not_see_it(ctx, dtype):
    say("attention NaN key beyond the line %s" % dtype)
    q, k, v, _ = case(7, dtype, 1, 600, 600, 1, 1, 64)
    want = reference(q, k, v, 0.125, True)
    k[0, 350:] = math.nan
    o, stat = ctx.fs_attention(q, k, v, causal=True)
    close("o", o[:, :350], want["o"][:, :350], TOL[dtype])
    assert torch.isnan(o[:, 350:]).all() and torch.isnan(stat[:, :, 350:]).all()


def test_empty_rows_stay_empty(ctx):
    say("attention NaN and empty rows")
    q, k, v, _ = case(8, F32, 3, 4, 3000, 2, 2, 64)
    q[1] = math.nan
    lens = torch.tensor([3000, 0, 1], dtype=torch.int32).cuda()
    o, stat = ctx.fs_attention(q, k, v, k_len=lens)
    assert (o[1] == 0).all() and (stat[1, ..., 0] == -math.inf).all() and (stat[1, ..., 1] == 0).all()
    close("one key", o[2], v[2, :1].expand(4, 2, 64).cpu(), 1e-5)
