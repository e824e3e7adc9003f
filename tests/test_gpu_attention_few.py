"""Gradients of a few rows in bf16.  Their probabilities do not average out, and go on in two pieces: what is left is the rounding of the
gradients themselves, 2^-9 to 2^-8 of a number at its half, 1.7e-3 in the mean square over numbers of any size: 2.1e-3."""
import pytest

from paper_2602_03067_amd import binding
from tests._gpu_common import say
from tests.test_gpu_attention import BF16, case, close, reference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,m,heads,kv_heads,d", [(1, 153, 16, 4, 32), (1, 400, 8, 8, 64), (3, 700, 20, 2, 96), (8, 300, 8, 2, 128),
                                                  (32, 100, 4, 4, 128), (16, 90, 8, 4, 63), (2, 33, 12, 12, 100)])
@pytest.mark.parametrize("causal", [False, True])
def test_few_rows_round_once(causal, n, m, heads, kv_heads, d):
    say("attention few rows n=%d m=%d heads=%d/%d d=%d causal=%s" % (n, m, heads, kv_heads, d, causal))
    ctx = binding.Context(0)
    q, k, v, do = case(17, BF16, 4, n, m, heads, kv_heads, d)
    o, stat = ctx.fs_attention(q, k, v, causal=causal)
    want = reference(q, k, v, d ** -0.5, causal, do=do)
    for name, t in zip(("dk", "dv"), ctx.fs_attention_grad(q, k, v, o, stat, do, causal=causal)[1:3]):
        close(name, t, want[name], 2.1e-3)
    ctx.close()
