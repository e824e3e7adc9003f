"""Sizes that the operators' launches do not hold, and outputs that meet, are refused, through a host-only context."""
import ctypes

import pytest

from paper_2602_03067_amd import binding
from paper_2602_03067_amd.binding import FsAttn, FsHeads

OK_ON_HOST, INVALID, SHAPE = 7, 1, 2
TB = 1 << 40


@pytest.fixture(scope="module")
def lib():
    return binding.load_library()


@pytest.fixture()
def hctx(lib):
    h = ctypes.c_void_p()
    assert lib.fs_create(ctypes.byref(h), -1, None) == 0
    yield h
    lib.fs_destroy(h)


def call(batch, n, m, heads, kv_heads, d, dtype=1):
    """Tensors of a TB each, one behind the other."""
    q, kv = (n * heads * d, heads * d, d), (m * kv_heads * d, kv_heads * d, d)
    at = [FsHeads((1 + i) * TB, *(kv if i in (1, 2, 6, 7) else q)) for i in range(8)]
    q, k, v, o, do, dq, dk, dv = at
    kw = FsAttn(q, k, v, dtype, 0, batch, n, m, heads, kv_heads, d, 0.25, None, None, None, 0)
    return kw, [ctypes.byref(x) for x in (o, do, dq, dk, dv)]


@pytest.mark.parametrize("batch,n,m,heads,kv_heads,d,forward,backward", [
    (1 << 20, 1, 40, 16, 16, 8, OK_ON_HOST, SHAPE),          # 2^24 heads of keys: 64 threads each forward, 256 backward
    ((1 << 20) - 1, 1, 40, 16, 16, 8, OK_ON_HOST, OK_ON_HOST),
    (1 << 22, 1, 40, 16, 16, 8, SHAPE, SHAPE),               # 2^26
    ((1 << 22) - 1, 1, 40, 16, 16, 8, OK_ON_HOST, SHAPE),
    (1 << 22, 1, 40, 64, 16, 8, SHAPE, SHAPE),
    (1 << 20, 200, 40, 8, 8, 8, SHAPE, SHAPE),               # two workgroups of 256 threads a head
    (1 << 20, 200, 40, 4, 4, 8, OK_ON_HOST, OK_ON_HOST),
    (1 << 20, 1, 200, 8, 8, 8, OK_ON_HOST, SHAPE),
    (1, 1 << 24, 1 << 20, 64, 1, 8, OK_ON_HOST, OK_ON_HOST),
])
def test_attention(lib, hctx, batch, n, m, heads, kv_heads, d, forward, backward):
    a, (o, do, dq, dk, dv) = call(batch, n, m, heads, kv_heads, d)
    assert lib.fs_attention(hctx, ctypes.byref(a), o, 9 * TB) == forward
    assert lib.fs_attention_grad(hctx, ctypes.byref(a), o, 9 * TB, do, dq, dk, dv, None, 0) == backward


@pytest.mark.parametrize("strides,status", [
    ((4 * 8 * 16, 8 * 16, 16), OK_ON_HOST), ((8 * 4 * 16, 16, 4 * 16), OK_ON_HOST),      # rows first, heads first
    ((3 * 4 * 8 * 16, 3 * 8 * 16, 16), OK_ON_HOST), ((16, 2 * 8 * 16, 2 * 16), OK_ON_HOST),   # inside a projection's, sets innermost
    ((16, 16, 16), SHAPE), ((4 * 8 * 16, 16, 16), SHAPE), ((4 * 8 * 16, 8 * 16, 17), SHAPE), ((4 * 8 * 16, 8 * 16 - 1, 16), SHAPE),
    ((4 * 8 * 16 - 16, 8 * 16, 16), SHAPE), ((8 * 4 * 16, 16, 4 * 16 - 8), SHAPE), ((0, 8 * 16, 16), SHAPE), ((8 * 16, 4 * 8 * 16, 16), OK_ON_HOST), ((8 * 16, 2 * 8 * 16 - 16, 16), SHAPE),
])
def test_rows_of_an_output_do_not_meet(lib, hctx, strides, status):
    """Two sets of four rows, eight heads of 16."""
    a, (o, do, dq, dk, dv) = call(2, 4, 4, 8, 8, 16)
    out = ctypes.byref(FsHeads(10 * TB, *strides))
    assert lib.fs_attention(hctx, ctypes.byref(a), out, 9 * TB) == status
    assert lib.fs_attention_grad(hctx, ctypes.byref(a), o, 9 * TB, do, out, dk, dv, None, 0) == status
    assert lib.fs_attention_grad(hctx, ctypes.byref(a), o, 9 * TB, do, dq, dk, out, None, 0) == status


def test_outputs_of_attention_do_not_meet(lib, hctx):
    a, (o, do, dq, dk, dv) = call(2, 4, 4, 8, 8, 16)
    size = 2 * 4 * 8 * 16 * 2
    assert lib.fs_attention(hctx, ctypes.byref(a), o, 9 * TB) == OK_ON_HOST
    for stat in (4 * TB, 4 * TB + size - 8, 4 * TB - 8):
        assert lib.fs_attention(hctx, ctypes.byref(a), o, stat) == INVALID
    assert lib.fs_attention(hctx, ctypes.byref(a), o, 4 * TB + size) == OK_ON_HOST

    def backward(dq, dk, dv, db=None, a=a):
        return lib.fs_attention_grad(hctx, ctypes.byref(a), o, 9 * TB, do, dq, dk, dv, db, 4 if db else 0)

    assert backward(dq, dk, dv) == OK_ON_HOST
    assert backward(dq, dq, dv) == INVALID and backward(dq, dk, dk) == INVALID and backward(dv, dk, dv) == INVALID
    a.bias, a.bias_ld = 11 * TB, 4
    assert backward(dq, dk, dv, 12 * TB) == OK_ON_HOST
    for at in (6, 7, 8):
        assert backward(dq, dk, dv, at * TB) == INVALID


def test_outputs_of_attention_are_not_its_lengths(lib, hctx):
    a, (o, do, dq, dk, dv) = call(2, 4, 4, 8, 8, 16)
    for field in ("q_len", "k_len"):
        setattr(a, field, 9 * TB + 64)
        assert lib.fs_attention(hctx, ctypes.byref(a), o, 9 * TB) == INVALID
        setattr(a, field, 6 * TB + 64)
        assert lib.fs_attention_grad(hctx, ctypes.byref(a), o, 9 * TB, do, dq, dk, dv, None, 0) == INVALID
        setattr(a, field, 13 * TB)
        assert lib.fs_attention(hctx, ctypes.byref(a), o, 9 * TB) == OK_ON_HOST
        assert lib.fs_attention_grad(hctx, ctypes.byref(a), o, 9 * TB, do, dq, dk, dv, None, 0) == OK_ON_HOST


def test_outputs_of_layer_norm_do_not_meet(lib, hctx):
    def forward(y, stat):
        return lib.fs_layer_norm(hctx, TB, 0, 4, 8, 8, None, None, 0, 1e-5, y, 8, stat)

    assert forward(2 * TB, 2 * TB + 128) == OK_ON_HOST and forward(2 * TB, 2 * TB + 120) == INVALID and forward(2 * TB + 24, 2 * TB) == INVALID

    def backward(dx, dgamma, dbeta):
        return lib.fs_layer_norm_grad(hctx, TB, 0, 4, 8, 8, None, 0, 3 * TB, 4 * TB, 8, dx, 8, dgamma, dbeta)

    assert backward(5 * TB, 5 * TB + 128, 5 * TB + 160) == OK_ON_HOST
    assert backward(5 * TB, 5 * TB + 124, None) == INVALID and backward(5 * TB, None, 5 * TB + 64) == INVALID
    assert backward(None, 6 * TB, 6 * TB + 28) == INVALID and backward(4 * TB, 6 * TB, 4 * TB + 100) == INVALID
