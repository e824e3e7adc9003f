"""AdamW refuses weights and states that share memory: two updates of one element would race."""
import pytest
import torch

from paper_2602_03067_amd import binding
from tests._gpu_common import say

pytestmark = pytest.mark.gpu
F8 = torch.float8_e4m3fn


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(0)
    yield c
    c.close()


def test_shared_memory_is_refused(ctx):
    say("adamw apart")
    room = torch.zeros(4000, device="cuda")
    p, q = room[:1000], room[1000:2000]
    state = lambda: [torch.zeros(1000, device="cuda") for _ in range(2)]
    one = torch.zeros(1000, device="cuda")
    for bad in (lambda: binding.AdamW(ctx, [p, p]), lambda: binding.AdamW(ctx, [p, room[999:1999]]),
                lambda: binding.AdamW(ctx, [p, q], m=[one, one]), lambda: binding.AdamW(ctx, [p, q], m=[one, state()[0]], v=[state()[0], one]),
                lambda: binding.AdamW(ctx, [p.bfloat16(), q.bfloat16()], master=[one, one]),
                lambda: binding.AdamW(ctx, [p, q], state_bits=8, m_scale=[one[:4], one[3:7]])):
        with pytest.raises(ValueError):
            bad()


def test_neighbours_and_empty_tensors_are_taken(ctx):
    say("adamw neighbours")
    room = torch.zeros(4000, device="cuda")
    for bits in (32, 8):
        p = [room[:1000], room[1000:1001], room[1001:1001], room[1001:4000]]
        opt = binding.AdamW(ctx, p, lr=0.5, state_bits=bits)
        opt.step([torch.ones(t.numel(), device="cuda") for t in p])
    assert (room < -0.9).all()


def test_memory_given_later(ctx):
    say("adamw apart, later")
    a, b = (torch.nn.Parameter(torch.zeros(500, device="cuda")) for _ in range(2))
    opt = binding.AdamW(ctx, [a, b], lr=0.5)
    g = [torch.ones(500, device="cuda") for _ in range(2)]
    own = b.data
    b.data = a.data
    for _ in range(2):
        with pytest.raises(ValueError):
            opt.step(g)
    b.data = own
    opt.step(g)
    torch.cuda.synchronize()
    assert torch.allclose(a.data, torch.full_like(a.data, -0.5)) and torch.equal(a.data, b.data)
