"""CPU-only checks of the operators' arguments, through a host-only context: what is refused, and with which status."""
import ctypes
import math

import pytest

from paper_2602_03067_amd import binding
from paper_2602_03067_amd.binding import FsAdamwArgs, FsAdamwTensor, FsAttn, FsHeads

OK_ON_HOST, INVALID, SHAPE, EPS, UNSUPPORTED = 7, 1, 2, 3, 5
MB = 1 << 20


@pytest.fixture(scope="module")
def lib():
    return binding.load_library()


@pytest.fixture()
def hctx(lib):
    h = ctypes.c_void_p()
    assert lib.fs_create(ctypes.byref(h), -1, None) == 0
    yield h
    lib.fs_destroy(h)


def attn(**kw):
    b, n, m, h, hk, d = (kw.pop(k, v) for k, v in (("batch", 2), ("n", 5), ("m", 7), ("h", 4), ("hk", 2), ("d", 16)))
    a = FsAttn(FsHeads(64 * MB, n * h * d, h * d, d), FsHeads(65 * MB, m * hk * d, hk * d, d), FsHeads(66 * MB, m * hk * d, hk * d, d), 0, 0, b, n, m,
               h, hk, d, 0.25, None, None, None, 0)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def out(at, rows=5, h=4, d=16):
    return FsHeads(at * MB, rows * h * d, h * d, d)


ATTN = [
    (dict(), OK_ON_HOST), (dict(dtype=2), INVALID), (dict(causal=2), INVALID), (dict(batch=-1), SHAPE), (dict(q_rows=-1), SHAPE), (dict(k_rows=-1), SHAPE),
    (dict(q_heads=0), SHAPE), (dict(kv_heads=0), SHAPE), (dict(kv_heads=3), SHAPE), (dict(d=0), SHAPE), (dict(d=129), UNSUPPORTED),
    (dict(q_rows=(1 << 24) + 1), SHAPE), (dict(batch=1 << 23, q_heads=64, kv_heads=64), SHAPE), (dict(scale=0.0), INVALID), (dict(scale=-1.0), INVALID),
    (dict(scale=math.nan), INVALID), (dict(scale=math.inf), INVALID), (dict(q=FsHeads(None, 320, 64, 16)), INVALID), (dict(k=FsHeads(None, 1, 1, 1)), INVALID),
    (dict(v=FsHeads(66 * MB + 2, 224, 32, 16)), INVALID), (dict(q=FsHeads(64 * MB, -1, 64, 16)), SHAPE), (dict(k=FsHeads(65 * MB, 224, 1 << 41, 16)), SHAPE),
    (dict(k=FsHeads(65 * MB, 0, 0, 0)), OK_ON_HOST), (dict(bias=67 * MB, bias_ld=6), SHAPE), (dict(bias=67 * MB, bias_ld=7), OK_ON_HOST),
    (dict(k_rows=0, k=FsHeads(None, 0, 0, 0), v=FsHeads(None, 0, 0, 0)), OK_ON_HOST),
]


@pytest.mark.parametrize("kw,status", ATTN)
def test_attention_arguments(lib, hctx, kw, status):
    a = attn(**kw)
    o, do, dq, dk, dv = out(70), out(72), out(73), out(74, 7, 2), out(75, 7, 2)
    assert lib.fs_attention(hctx, ctypes.byref(a), ctypes.byref(o), 71 * MB) == status
    assert lib.fs_last_error(hctx) != b""
    assert lib.fs_attention_grad(hctx, ctypes.byref(a), ctypes.byref(o), 71 * MB, ctypes.byref(do), ctypes.byref(dq), ctypes.byref(dk), ctypes.byref(dv),
                                 None, 0) == status


def test_attention_outputs(lib, hctx):
    a, o = attn(), out(70)

    def forward(o, stat=71 * MB):
        return lib.fs_attention(hctx, ctypes.byref(a), None if o is None else ctypes.byref(o), stat)

    assert forward(None) == INVALID and forward(FsHeads(None, 320, 64, 16)) == INVALID
    assert forward(FsHeads(70 * MB, 320, 64, 15)) == SHAPE and forward(FsHeads(70 * MB, 320, 0, 16)) == SHAPE
    assert forward(FsHeads(64 * MB, 320, 64, 16)) == INVALID          # over q
    assert forward(FsHeads(66 * MB - 64, 320, 64, 16)) == INVALID     # into v
    assert forward(o, None) == INVALID and forward(o, 71 * MB + 4) == INVALID and forward(o, 65 * MB) == INVALID
    assert lib.fs_attention(None, ctypes.byref(a), ctypes.byref(o), 71 * MB) == INVALID
    assert lib.fs_attention(hctx, None, ctypes.byref(o), 71 * MB) == INVALID

    def backward(a=a, dq=out(73), dk=out(74, 7, 2), do=out(72), db=None, ld=0):
        args = [None if x is None else ctypes.byref(x) for x in (do, dq, dk, out(75, 7, 2))]
        return lib.fs_attention_grad(hctx, ctypes.byref(a), ctypes.byref(o), 71 * MB, *args, db, ld)

    assert backward() == OK_ON_HOST and backward(dq=None) == INVALID and backward(do=None) == INVALID
    assert backward(dk=out(65, 7, 2)) == INVALID and backward(dq=out(72)) == INVALID and backward(dq=out(71)) == INVALID
    assert backward(db=80 * MB, ld=7) == INVALID                      # no bias to have a gradient
    biased = attn(bias=67 * MB, bias_ld=7)
    assert backward(biased, db=80 * MB, ld=7) == OK_ON_HOST and backward(biased, db=80 * MB, ld=6) == SHAPE and backward(biased, db=67 * MB, ld=7) == INVALID
    assert backward(attn(bias=67 * MB, bias_ld=0), db=80 * MB, ld=7) == UNSUPPORTED


def test_packed_outputs_are_taken(lib, hctx):
    """dq, dk and dv inside one buffer, as a projection's gradient wants them."""
    a = attn(h=2, hk=2, n=7)
    o = out(70, 7, 2)
    d = [FsHeads(80 * MB + 4 * 32 * i, 7 * 96, 96, 16) for i in range(3)]
    assert lib.fs_attention_grad(hctx, ctypes.byref(a), ctypes.byref(o), 71 * MB, ctypes.byref(out(72, 7, 2)), *(ctypes.byref(x) for x in d), None, 0) == OK_ON_HOST


@pytest.mark.parametrize("kw,status", [
    (dict(), OK_ON_HOST), (dict(dtype=3), INVALID), (dict(wtype=3), INVALID), (dict(rows=-1), SHAPE), (dict(cols=0), SHAPE), (dict(ldx=7), SHAPE),
    (dict(ldy=7), SHAPE), (dict(cols=(1 << 24) + 1, ldx=1 << 25, ldy=1 << 25), SHAPE), (dict(x=None), INVALID), (dict(y=None), INVALID), (dict(x=8 * MB + 2), INVALID),
    (dict(gamma=9 * MB + 1), INVALID), (dict(y=8 * MB), INVALID), (dict(y=9 * MB), INVALID), (dict(stat=12 * MB + 4), INVALID), (dict(stat=8 * MB), INVALID),
    (dict(stat=None), OK_ON_HOST), (dict(gamma=None, beta=None), OK_ON_HOST), (dict(eps=-1e-5), EPS), (dict(eps=math.nan), EPS), (dict(eps=0.0), OK_ON_HOST),
    (dict(rows=0, x=None, y=None), OK_ON_HOST),
])
def test_layer_norm_arguments(lib, hctx, kw, status):
    p = dict(x=8 * MB, dtype=0, rows=4, cols=8, ldx=8, gamma=9 * MB, beta=10 * MB, wtype=0, eps=1e-5, y=11 * MB, ldy=8, stat=12 * MB)
    p.update(kw)
    assert lib.fs_layer_norm(hctx, p["x"], p["dtype"], p["rows"], p["cols"], p["ldx"], p["gamma"], p["beta"], p["wtype"], p["eps"], p["y"], p["ldy"],
                             p["stat"]) == status


@pytest.mark.parametrize("kw,status", [
    (dict(), OK_ON_HOST), (dict(dx=None), OK_ON_HOST), (dict(dx=11 * MB), OK_ON_HOST), (dict(dx=11 * MB, lddx=9), INVALID), (dict(dx=11 * MB + 32), INVALID),
    (dict(dx=8 * MB), INVALID), (dict(dgamma=9 * MB), INVALID), (dict(dbeta=12 * MB), INVALID), (dict(dy=None), INVALID), (dict(lddy=7), SHAPE), (dict(lddx=7), SHAPE),
    (dict(stat=None), INVALID), (dict(dgamma=None, dbeta=None), OK_ON_HOST),
])
def test_layer_norm_grad_arguments(lib, hctx, kw, status):
    p = dict(x=8 * MB, dtype=0, rows=4, cols=8, ldx=8, gamma=9 * MB, wtype=0, stat=12 * MB, dy=11 * MB, lddy=8, dx=13 * MB, lddx=8, dgamma=14 * MB,
             dbeta=15 * MB)
    p.update(kw)
    assert lib.fs_layer_norm_grad(hctx, *(p[k] for k in ("x", "dtype", "rows", "cols", "ldx", "gamma", "wtype", "stat", "dy", "lddy", "dx", "lddx", "dgamma",
                                                         "dbeta"))) == status


def tensor(i=0, **kw):
    p = dict(p=(8 + 8 * i) * MB, g=(9 + 8 * i) * MB, master=None, m=(10 + 8 * i) * MB, v=(11 + 8 * i) * MB, m_scale=(12 + 8 * i) * MB, v_scale=(13 + 8 * i) * MB, n=1000)
    p.update(kw)
    return FsAdamwTensor(*(p[k] for k in ("p", "g", "master", "m", "v", "m_scale", "v_scale", "n")))


@pytest.mark.parametrize("args,one,status", [
    (dict(), dict(), OK_ON_HOST), (dict(p_dtype=2), dict(), INVALID), (dict(g_dtype=-1), dict(), INVALID), (dict(state_bits=4), dict(), UNSUPPORTED),
    (dict(lr=-1.0), dict(), INVALID), (dict(lr=math.nan), dict(), INVALID), (dict(beta1=1.0), dict(), INVALID), (dict(beta2=-0.1), dict(), INVALID),
    (dict(eps=math.inf), dict(), INVALID), (dict(weight_decay=-1.0), dict(), INVALID), (dict(step=0), dict(), INVALID), (dict(), dict(n=-1), SHAPE),
    (dict(), dict(n=0, p=None), OK_ON_HOST), (dict(), dict(p=None), INVALID), (dict(), dict(g=None), INVALID), (dict(), dict(m=None), INVALID),
    (dict(), dict(v=None), INVALID), (dict(state_bits=8), dict(m_scale=None), INVALID), (dict(state_bits=8), dict(v_scale=None), INVALID),
    (dict(), dict(m_scale=None), OK_ON_HOST), (dict(), dict(master=14 * MB), UNSUPPORTED), (dict(), dict(g=8 * MB), INVALID), (dict(), dict(v=10 * MB + 4), INVALID),
    (dict(), dict(p=8 * MB + 2), INVALID), (dict(p_dtype=1), dict(p=8 * MB + 2), OK_ON_HOST), (dict(state_bits=8), dict(m=10 * MB + 3), OK_ON_HOST),
])
def test_adamw_arguments(lib, hctx, args, one, status):
    p = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0, step=1, p_dtype=0, g_dtype=0, state_bits=32)
    p.update(args)
    a = FsAdamwArgs(**p)
    t = (FsAdamwTensor * 2)(tensor(0, **one), tensor(1))
    assert lib.fs_adamw(hctx, ctypes.byref(a), t, 2) == status


def test_adamw_masters(lib, hctx):
    a = FsAdamwArgs(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=1, p_dtype=1, g_dtype=1, state_bits=8)
    both = (FsAdamwTensor * 2)(tensor(0, master=14 * MB), tensor(1, master=22 * MB))
    assert lib.fs_adamw(hctx, ctypes.byref(a), both, 2) == OK_ON_HOST
    one = (FsAdamwTensor * 2)(tensor(0, master=14 * MB), tensor(1))
    assert lib.fs_adamw(hctx, ctypes.byref(a), one, 2) == INVALID
    a.p_dtype = 0
    assert lib.fs_adamw(hctx, ctypes.byref(a), both, 2) == UNSUPPORTED
    assert lib.fs_adamw(hctx, ctypes.byref(a), None, 1) == INVALID and lib.fs_adamw(hctx, None, both, 2) == INVALID
    assert lib.fs_adamw(hctx, ctypes.byref(a), both, -1) == SHAPE and lib.fs_adamw(hctx, ctypes.byref(a), None, 0) == OK_ON_HOST
