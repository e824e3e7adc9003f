"""Thin ctypes binding of libflashsink (argument marshalling only).

Function names match the C ABI in ``include/flashsink.h``.  Tensors are PyTorch
CUDA(ROCm) tensors used purely as device memory; every step of the method runs
inside the library's HIP kernels.  There is no CPU fallback: if the library is
missing or a call fails, an exception is raised.
"""
from __future__ import annotations

import ctypes
import operator
import os
import struct
from typing import Optional, Tuple

import numpy as np
import torch  # loaded first so that the library binds to the same HIP runtime as torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libflashsink.so")

FS_F32, FS_BF16 = 0, 1
FS_COMPUTE_FP32, FS_COMPUTE_BF16_MFMA = 0, 1

EXPORTS = (
    "fs_create", "fs_destroy", "fs_status_str", "fs_last_error", "fs_version", "fs_row_norms",
    "fs_update_f", "fs_update_g", "fs_solve", "fs_solve_noalloc", "fs_solve_labeled", "fs_solve_symmetric", "fs_solve_tol", "fs_marginal_err", "fs_ot_value", "fs_check_weights", "fs_check_finite", "fs_divergence", "fs_apply_plan",
    "fs_apply_plan_T", "fs_apply_plan_hadamard", "fs_grad_x", "fs_grad_y", "fs_hvp", "fs_attention", "fs_attention_grad", "fs_layer_norm", "fs_layer_norm_grad", "fs_adamw", "fs_points_keep", "fs_points_release", "fs_debug_set", "fs_debug_get", "fs_profile_enable", "fs_profile_read",
)


class FsProblem(ctypes.Structure):
    _fields_ = [
        ("x", ctypes.c_void_p), ("y", ctypes.c_void_p),
        ("dtype", ctypes.c_int32), ("compute", ctypes.c_int32),
        ("n", ctypes.c_int64), ("m", ctypes.c_int64), ("d", ctypes.c_int64),
        ("ldx", ctypes.c_int64), ("ldy", ctypes.c_int64),
        ("a", ctypes.c_void_p), ("b", ctypes.c_void_p),
    ]


class FsHeads(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("batch", ctypes.c_int64), ("row", ctypes.c_int64), ("head", ctypes.c_int64)]


class FsAttn(ctypes.Structure):
    _fields_ = [
        ("q", FsHeads), ("k", FsHeads), ("v", FsHeads), ("dtype", ctypes.c_int32), ("causal", ctypes.c_int32),
        ("batch", ctypes.c_int64), ("q_rows", ctypes.c_int64), ("k_rows", ctypes.c_int64),
        ("q_heads", ctypes.c_int64), ("kv_heads", ctypes.c_int64), ("d", ctypes.c_int64), ("scale", ctypes.c_float),
        ("q_len", ctypes.c_void_p), ("k_len", ctypes.c_void_p), ("bias", ctypes.c_void_p), ("bias_ld", ctypes.c_int64),
    ]


class FsAdamwTensor(ctypes.Structure):
    _fields_ = [("p", ctypes.c_void_p), ("g", ctypes.c_void_p), ("master", ctypes.c_void_p), ("m", ctypes.c_void_p),
                ("v", ctypes.c_void_p), ("m_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p), ("n", ctypes.c_int64)]


class FsAdamwArgs(ctypes.Structure):
    _fields_ = [("lr", ctypes.c_double), ("beta1", ctypes.c_double), ("beta2", ctypes.c_double), ("eps", ctypes.c_double),
                ("weight_decay", ctypes.c_double), ("step", ctypes.c_int64), ("p_dtype", ctypes.c_int32), ("g_dtype", ctypes.c_int32),
                ("state_bits", ctypes.c_int32), ("seed", ctypes.c_uint32), ("grad_scale", ctypes.c_void_p)]


class FlashSinkError(RuntimeError):
    def __init__(self, status: int, what: str, detail: str):
        super().__init__("%s: status %d (%s)" % (what, status, detail))
        self.status = status


_lib = None


def load_library(path: Optional[str] = None) -> ctypes.CDLL:
    """Load libflashsink.so (built in-tree by ``python -m paper_2602_03067_amd.build``)."""
    global _lib
    if _lib is not None and path is None:
        return _lib
    path = path or LIB_PATH
    if not os.path.exists(path):
        raise FileNotFoundError(
            "%s not found: build it with `python -m paper_2602_03067_amd.build` "
            "(there is no fallback path)" % path)
    lib = ctypes.CDLL(path)
    vp, i32, i64, f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float
    PP = ctypes.POINTER(FsProblem)
    lib.fs_create.argtypes = [ctypes.POINTER(vp), ctypes.c_int, vp]
    lib.fs_destroy.argtypes = [vp]
    lib.fs_status_str.argtypes = [ctypes.c_int]
    lib.fs_status_str.restype = ctypes.c_char_p
    lib.fs_last_error.argtypes = [vp]
    lib.fs_last_error.restype = ctypes.c_char_p
    lib.fs_version.argtypes = []
    lib.fs_version.restype = ctypes.c_char_p
    lib.fs_row_norms.argtypes = [vp, vp, i32, i64, i64, i64, vp]
    lib.fs_update_f.argtypes = [vp, PP, f32, vp, vp]
    lib.fs_update_g.argtypes = [vp, PP, f32, vp, vp]
    lib.fs_solve.argtypes = [vp, PP, f32, f32, i32, i32, vp, vp]
    lib.fs_solve_noalloc.argtypes = [vp, PP, f32, f32, i32, i32, vp, vp]
    lib.fs_solve_labeled.argtypes = [vp, PP, vp, vp, vp, i32, f32, f32, f32, i32, vp, vp]
    lib.fs_solve_symmetric.argtypes = [vp, PP, f32, i32, vp, vp]
    lib.fs_solve_tol.argtypes = [vp, PP, f32, i32, i32, f32, vp, vp, ctypes.POINTER(i32), ctypes.POINTER(f32)]
    lib.fs_marginal_err.argtypes = [vp, PP, f32, vp, vp, ctypes.POINTER(f32), ctypes.POINTER(f32)]
    lib.fs_ot_value.argtypes = [vp, PP, f32, vp, vp, ctypes.POINTER(ctypes.c_double)]
    lib.fs_check_finite.argtypes = [vp, vp, i64, ctypes.POINTER(ctypes.c_int64)]
    lib.fs_check_weights.argtypes = [vp, PP, f32, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_double)]
    lib.fs_divergence.argtypes = [vp, PP, f32, i32, vp, vp, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_double)]
    lib.fs_apply_plan.argtypes = [vp, PP, f32, vp, vp, vp, i64, i64, vp, i64, vp]
    lib.fs_apply_plan_T.argtypes = [vp, PP, f32, vp, vp, vp, i64, i64, vp, i64, vp]
    lib.fs_apply_plan_hadamard.argtypes = [vp, PP, f32, vp, vp, vp, i64, vp, i64, i64, vp, i64]
    lib.fs_grad_x.argtypes = [vp, PP, f32, vp, vp, i32, vp, i64]
    lib.fs_grad_y.argtypes = [vp, PP, f32, vp, vp, i32, vp, i64]
    lib.fs_hvp.argtypes = [vp, PP, f32, vp, vp, vp, i64, f32, f32, i32, vp, i64, ctypes.POINTER(i32)]
    # (fs_attn and fs_heads as bytes or by reference)
    lib.fs_attention.argtypes = [vp, vp, vp, vp]
    lib.fs_attention_grad.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, i64]
    lib.fs_layer_norm.argtypes = [vp, vp, i32, i64, i64, i64, vp, vp, i32, f32, vp, i64, vp]
    lib.fs_layer_norm_grad.argtypes = [vp, vp, i32, i64, i64, i64, vp, i32, vp, vp, i64, vp, i64, vp, vp]
    lib.fs_adamw.argtypes = [vp, ctypes.POINTER(FsAdamwArgs), ctypes.POINTER(FsAdamwTensor), i32]
    lib.fs_debug_set.argtypes = [vp, ctypes.c_char_p, i64]
    lib.fs_debug_get.argtypes = [vp, ctypes.c_char_p, ctypes.POINTER(i64)]
    lib.fs_points_keep.argtypes = [vp, PP]
    lib.fs_points_release.argtypes = [vp]
    lib.fs_profile_enable.argtypes = [vp, i32]
    lib.fs_profile_read.argtypes = [vp, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(i64),
                                    ctypes.POINTER(ctypes.c_double)]
    for name in EXPORTS:
        if name not in ("fs_status_str", "fs_last_error", "fs_version"):
            getattr(lib, name).restype = ctypes.c_int
    if path == LIB_PATH:
        _lib = lib
    return lib


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _dev_f32(t: torch.Tensor, name: str, shape=None):
    if not isinstance(t, torch.Tensor) or not t.is_cuda or t.dtype != torch.float32 \
            or not t.is_contiguous():
        raise TypeError("%s must be a contiguous float32 tensor on the GPU" % name)
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError("%s has shape %s, expected %s" % (name, tuple(t.shape), tuple(shape)))
    return t


_get_dtype, _get_is_cuda = operator.attrgetter("dtype"), operator.attrgetter("is_cuda")
_DTYPES = {torch.float32: FS_F32, torch.bfloat16: FS_BF16}


def _heads(t: torch.Tensor, name: str, shape, dtype):
    """Address and strides of a (sets, rows, heads, coordinates) tensor, as fs_heads has them."""
    if t.dtype is not dtype or not t.is_cuda:
        raise TypeError("%s must be a %s tensor on the GPU" % (name, dtype))
    if t.shape != shape:
        raise ValueError("%s has shape %s, expected %s" % (name, tuple(t.shape), tuple(shape)))
    b, r, h, e = t.stride()
    if e != 1 and shape[3] != 1:
        raise ValueError("%s must have unit stride within a head" % name)
    return t.data_ptr(), b, r, h


# (the structures' bytes: made faster than ctypes fills their fields)
_HEADS, _ATTN = struct.Struct("Qqqq"), struct.Struct("QqqqQqqqQqqqiiqqqqqqf4xQQQq")
assert _HEADS.size == ctypes.sizeof(FsHeads) and _ATTN.size == ctypes.sizeof(FsAttn)


def _lengths(t: Optional[torch.Tensor], name: str, batch: int):
    if t is None:
        return 0
    if not t.is_cuda or t.dtype != torch.int32 or not t.is_contiguous() or t.shape != (batch,):
        raise TypeError("%s must be a contiguous int32 GPU tensor of %d lengths" % (name, batch))
    return t.data_ptr()


def _attn(q, k, v, scale, causal, q_len, k_len, bias):
    dtype = q.dtype
    if q.dim() != 4 or k.dim() != 4 or dtype not in _DTYPES:
        raise TypeError("q, k, v must be float32 or bfloat16 tensors of (sets, rows, heads, coordinates)")
    (batch, n, heads, d), (_, m, kv_heads, _) = q.shape, k.shape
    kv, at, ld = (batch, m, kv_heads, d), 0, 0
    if bias is not None:
        if not bias.is_cuda or bias.dtype != torch.float32 or bias.shape != (batch, m) or (m > 1 and bias.stride(1) != 1):
            raise TypeError("bias must be a float32 GPU tensor of (sets, keys) with unit inner stride")
        at, ld = bias.data_ptr(), bias.stride(0) if batch > 1 else m
    return _ATTN.pack(*_heads(q, "q", q.shape, dtype), *_heads(k, "k", kv, dtype), *_heads(v, "v", kv, dtype), _DTYPES[dtype], 1 if causal else 0,
                      batch, n, m, heads, kv_heads, d, max(d, 1) ** -0.5 if scale is None else scale, _lengths(q_len, "q_len", batch),
                      _lengths(k_len, "k_len", batch), at, ld)


def _matrix(t: torch.Tensor, name: str):
    if not t.is_cuda or t.dim() != 2 or t.dtype not in _DTYPES or (t.shape[1] > 1 and t.stride(1) != 1):
        raise TypeError("%s must be a 2-d float32 or bfloat16 GPU tensor with unit inner stride" % name)


def _ld(t: torch.Tensor) -> int:
    return t.stride(0) if t.shape[0] > 1 else t.shape[1]


def _weights(t: Optional[torch.Tensor], name: str, cols: int):
    if t is None:
        return None
    if not t.is_cuda or t.dtype not in _DTYPES or t.shape != (cols,) or not t.is_contiguous():
        raise TypeError("%s must be a contiguous float32 or bfloat16 GPU tensor of %d values" % (name, cols))
    return t.data_ptr()


class Problem:
    """Holds the tensors of one OT problem and the matching C struct."""

    def __init__(self, x: torch.Tensor, y: torch.Tensor, a: Optional[torch.Tensor] = None,
                 b: Optional[torch.Tensor] = None, compute: int = FS_COMPUTE_FP32):
        for t, nm in ((x, "x"), (y, "y")):
            if not t.is_cuda or t.dim() != 2 or t.stride(1) != 1:
                raise TypeError("%s must be a 2-d GPU tensor with unit inner stride" % nm)
        if x.dtype != y.dtype or x.dtype not in (torch.float32, torch.bfloat16):
            raise TypeError("x and y must both be float32 or both bfloat16")
        if x.shape[1] != y.shape[1]:
            raise ValueError("x and y differ in feature dimension")
        self.x, self.y, self.a, self.b = x, y, a, b
        if a is not None:
            _dev_f32(a, "a", (x.shape[0],))
        if b is not None:
            _dev_f32(b, "b", (y.shape[0],))
        self.n, self.m, self.d = x.shape[0], y.shape[0], x.shape[1]
        self.c = FsProblem(
            x.data_ptr(), y.data_ptr(), FS_BF16 if x.dtype == torch.bfloat16 else FS_F32,
            int(compute), self.n, self.m, self.d, x.stride(0), y.stride(0),
            None if a is None else a.data_ptr(), None if b is None else b.data_ptr())


class Context:
    """fs_ctx bound to a device and to the torch stream current at creation."""

    def __init__(self, device: int = 0, stream: Optional[torch.cuda.Stream] = None):
        self.lib = load_library()
        if not torch.cuda.is_available():
            raise RuntimeError("flashsink needs a GPU: torch.cuda.is_available() is False")
        self.device = int(device)
        with torch.cuda.device(self.device):
            self.stream = stream if stream is not None else torch.cuda.current_stream()
        h = ctypes.c_void_p()
        st = self.lib.fs_create(ctypes.byref(h), self.device, ctypes.c_void_p(self.stream.cuda_stream))
        if st != 0:
            raise FlashSinkError(st, "fs_create", self.lib.fs_status_str(st).decode())
        self.h = h

    def close(self):
        if getattr(self, "h", None):
            self.lib.fs_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check(self, st: int, what: str):
        if st != 0:
            detail = self.lib.fs_last_error(self.h).decode() or self.lib.fs_status_str(st).decode()
            raise FlashSinkError(st, what, detail)

    # ---- entry points (same names as the C ABI) --------------------------------------
    def fs_row_norms(self, pts: torch.Tensor) -> torch.Tensor:
        out = torch.empty(pts.shape[0], dtype=torch.float32, device=pts.device)
        dt = FS_BF16 if pts.dtype == torch.bfloat16 else FS_F32
        self._check(self.lib.fs_row_norms(self.h, _ptr(pts), dt, pts.shape[0], pts.shape[1],
                                          pts.stride(0), _ptr(out)), "fs_row_norms")
        return out

    def fs_update_f(self, prob: Problem, eps: float, g: torch.Tensor) -> torch.Tensor:
        _dev_f32(g, "g", (prob.m,))
        f = torch.empty(prob.n, dtype=torch.float32, device=g.device)
        self._check(self.lib.fs_update_f(self.h, ctypes.byref(prob.c), eps, _ptr(g), _ptr(f)),
                    "fs_update_f")
        return f

    def fs_update_g(self, prob: Problem, eps: float, f: torch.Tensor) -> torch.Tensor:
        _dev_f32(f, "f", (prob.n,))
        g = torch.empty(prob.m, dtype=torch.float32, device=f.device)
        self._check(self.lib.fs_update_g(self.h, ctypes.byref(prob.c), eps, _ptr(f), _ptr(g)),
                    "fs_update_g")
        return g

    def fs_solve(self, prob: Problem, eps_start: float, eps_end: float, n_stages: int,
                 iters_per_stage: int, f: torch.Tensor, g: torch.Tensor) -> None:
        """In place: f, g are the starting potentials and receive the result."""
        _dev_f32(f, "f", (prob.n,))
        _dev_f32(g, "g", (prob.m,))
        self._check(self.lib.fs_solve(self.h, ctypes.byref(prob.c), eps_start, eps_end,
                                      int(n_stages), int(iters_per_stage), _ptr(f), _ptr(g)),
                    "fs_solve")

    def fs_solve_noalloc(self, prob: Problem, eps_start: float, eps_end: float, n_stages: int,
                         iters_per_stage: int, f: torch.Tensor, g: torch.Tensor) -> None:
        """fs_solve in the library's static scratch array (no device allocation); in place like fs_solve."""
        _dev_f32(f, "f", (prob.n,))
        _dev_f32(g, "g", (prob.m,))
        self._check(self.lib.fs_solve_noalloc(self.h, ctypes.byref(prob.c), eps_start, eps_end,
                                              int(n_stages), int(iters_per_stage), _ptr(f), _ptr(g)),
                    "fs_solve_noalloc")

    def fs_solve_labeled(self, prob: Problem, lx: torch.Tensor, ly: torch.Tensor, W: torch.Tensor, lambda1: float,
                         lambda2: float, eps: float, iters: int, f: torch.Tensor, g: torch.Tensor) -> None:
        """Alternating Sinkhorn for lambda1 |x - y|^2 + lambda2 W[lx, ly]; in place like fs_solve."""
        _dev_f32(f, "f", (prob.n,))
        _dev_f32(g, "g", (prob.m,))
        _dev_f32(W, "W")
        if W.dim() != 2 or W.shape[0] != W.shape[1]:
            raise ValueError("W must be square")
        for t, nm, cnt in ((lx, "lx", prob.n), (ly, "ly", prob.m)):
            if not t.is_cuda or t.dtype != torch.int32 or not t.is_contiguous() or tuple(t.shape) != (cnt,):
                raise TypeError("%s must be a contiguous int32 GPU tensor of %d labels" % (nm, cnt))
        self._check(self.lib.fs_solve_labeled(self.h, ctypes.byref(prob.c), _ptr(lx), _ptr(ly), _ptr(W), W.shape[0],
                                              float(lambda1), float(lambda2), float(eps), int(iters), _ptr(f), _ptr(g)),
                    "fs_solve_labeled")

    def fs_solve_tol(self, prob: Problem, eps: float, max_iters: int, check_every: int, tol: float,
                     f: torch.Tensor, g: torch.Tensor) -> Tuple[int, float]:
        """In place like fs_solve; returns (iterations done, measured L1 row marginal error)."""
        _dev_f32(f, "f", (prob.n,))
        _dev_f32(g, "g", (prob.m,))
        done, err = ctypes.c_int32(), ctypes.c_float()
        self._check(self.lib.fs_solve_tol(self.h, ctypes.byref(prob.c), eps, int(max_iters), int(check_every),
                                          float(tol), _ptr(f), _ptr(g), ctypes.byref(done), ctypes.byref(err)),
                    "fs_solve_tol")
        return done.value, err.value

    def fs_ot_value(self, prob: Problem, eps: float, f: torch.Tensor, g: torch.Tensor) -> float:
        _dev_f32(f, "f", (prob.n,))
        _dev_f32(g, "g", (prob.m,))
        v = ctypes.c_double()
        self._check(self.lib.fs_ot_value(self.h, ctypes.byref(prob.c), eps, _ptr(f), _ptr(g), ctypes.byref(v)),
                    "fs_ot_value")
        return v.value

    def fs_check_finite(self, v: torch.Tensor) -> int:
        """Raises (status 8) if an entry of the float tensor is NaN or infinite; returns 0 otherwise."""
        assert v.dtype == torch.float32 and v.is_contiguous()
        bad = ctypes.c_int64()
        self._check(self.lib.fs_check_finite(self.h, _ptr(v), v.numel(), ctypes.byref(bad)), "fs_check_finite")
        return bad.value

    def fs_check_weights(self, prob: Problem, tol: float = 1e-5):
        """Raises if a weight is not positive and finite or a sum is off by more than tol; returns the two sums."""
        sa, sb = ctypes.c_double(), ctypes.c_double()
        self._check(self.lib.fs_check_weights(self.h, ctypes.byref(prob.c), tol, ctypes.byref(sa), ctypes.byref(sb)),
                    "fs_check_weights")
        return sa.value, sb.value

    def fs_divergence(self, prob: Problem, eps: float, iters: int):
        """Debiased Sinkhorn divergence; returns (value, (OT(a,b), OT(a,a), OT(b,b)), f, g)."""
        f = torch.empty(prob.n, dtype=torch.float32, device=prob.x.device)
        g = torch.empty(prob.m, dtype=torch.float32, device=prob.x.device)
        v = ctypes.c_double()
        t = (ctypes.c_double * 3)()
        self._check(self.lib.fs_divergence(self.h, ctypes.byref(prob.c), eps, int(iters), _ptr(f), _ptr(g), ctypes.byref(v), t),
                    "fs_divergence")
        return v.value, (t[0], t[1], t[2]), f, g

    def fs_solve_symmetric(self, prob: Problem, eps: float, iters: int, f: torch.Tensor,
                           g: torch.Tensor) -> None:
        """In place: f, g are the starting potentials and receive the result."""
        _dev_f32(f, "f", (prob.n,))
        _dev_f32(g, "g", (prob.m,))
        self._check(self.lib.fs_solve_symmetric(self.h, ctypes.byref(prob.c), eps, int(iters), _ptr(f), _ptr(g)),
                    "fs_solve_symmetric")

    def fs_marginal_err(self, prob: Problem, eps: float, f: torch.Tensor,
                        g: torch.Tensor) -> Tuple[float, float]:
        _dev_f32(f, "f", (prob.n,))
        _dev_f32(g, "g", (prob.m,))
        er, ec = ctypes.c_float(), ctypes.c_float()
        self._check(self.lib.fs_marginal_err(self.h, ctypes.byref(prob.c), eps, _ptr(f), _ptr(g),
                                             ctypes.byref(er), ctypes.byref(ec)), "fs_marginal_err")
        return er.value, ec.value

    def _apply(self, fn, what, prob, eps, f, g, M, rows_out, rows_in, want_mass):
        _dev_f32(f, "f", (prob.n,))
        _dev_f32(g, "g", (prob.m,))
        if M.dim() != 2 or M.shape[0] != rows_in or M.dtype != torch.float32 or M.stride(1) != 1:
            raise TypeError("matrix to apply must be float32 (rows=%d, p), unit inner stride" % rows_in)
        p = M.shape[1]
        out = torch.empty((rows_out, p), dtype=torch.float32, device=M.device)
        mass = torch.empty(rows_out, dtype=torch.float32, device=M.device) if want_mass else None
        self._check(fn(self.h, ctypes.byref(prob.c), eps, _ptr(f), _ptr(g), _ptr(M), p, M.stride(0),
                       _ptr(out), out.stride(0), _ptr(mass)), what)
        return (out, mass) if want_mass else out

    def fs_apply_plan(self, prob: Problem, eps: float, f, g, V, want_mass: bool = False):
        return self._apply(self.lib.fs_apply_plan, "fs_apply_plan", prob, eps, f, g, V, prob.n,
                           prob.m, want_mass)

    def fs_apply_plan_T(self, prob: Problem, eps: float, f, g, U, want_mass: bool = False):
        return self._apply(self.lib.fs_apply_plan_T, "fs_apply_plan_T", prob, eps, f, g, U, prob.m,
                           prob.n, want_mass)

    def fs_apply_plan_hadamard(self, prob: Problem, eps: float, f, g, A: torch.Tensor, V: torch.Tensor) -> torch.Tensor:
        """(P o (A y^T)) V (Alg. 5); A is n x d, V is m x p; returns n x p."""
        _dev_f32(f, "f", (prob.n,))
        _dev_f32(g, "g", (prob.m,))
        _dev_f32(A, "A", (prob.n, prob.d))
        if V.dim() != 2 or V.shape[0] != prob.m or V.dtype != torch.float32 or V.stride(1) != 1:
            raise TypeError("V must be float32 (m, p) with unit inner stride")
        p = V.shape[1]
        out = torch.empty((prob.n, p), dtype=torch.float32, device=V.device)
        self._check(self.lib.fs_apply_plan_hadamard(self.h, ctypes.byref(prob.c), eps, _ptr(f), _ptr(g), _ptr(A), A.stride(0),
                                                    _ptr(V), p, V.stride(0), _ptr(out), out.stride(0)),
                    "fs_apply_plan_hadamard")
        return out

    def _grad(self, fn, name, prob: Problem, eps: float, f, g, mode: int, rows: int) -> torch.Tensor:
        _dev_f32(f, "f", (prob.n,))
        _dev_f32(g, "g", (prob.m,))
        out = torch.empty(rows, prob.d, dtype=torch.float32, device=f.device)
        self._check(fn(self.h, ctypes.byref(prob.c), eps, _ptr(f), _ptr(g), int(mode), _ptr(out), prob.d), name)
        return out

    def fs_grad_x(self, prob: Problem, eps: float, f, g, mode: int = 0) -> torch.Tensor:
        """Gradient with respect to x (n x d); mode 0: 2(diag(a)x - Py), 1: with r = P1, 2: x - (Py)/a."""
        return self._grad(self.lib.fs_grad_x, "fs_grad_x", prob, eps, f, g, mode, prob.n)

    def fs_grad_y(self, prob: Problem, eps: float, f, g, mode: int = 0) -> torch.Tensor:
        return self._grad(self.lib.fs_grad_y, "fs_grad_y", prob, eps, f, g, mode, prob.m)

    def fs_hvp(self, prob: Problem, eps: float, f: torch.Tensor, g: torch.Tensor, A: torch.Tensor,
               tau: float, eta: float, max_cg: int) -> Tuple[torch.Tensor, int]:
        """Hessian-vector product T A (Thm. 5); returns (G [n x d], CG iterations)."""
        _dev_f32(f, "f", (prob.n,))
        _dev_f32(g, "g", (prob.m,))
        _dev_f32(A, "A", (prob.n, prob.d))
        out = torch.empty(prob.n, prob.d, dtype=torch.float32, device=f.device)
        it = ctypes.c_int32()
        self._check(self.lib.fs_hvp(self.h, ctypes.byref(prob.c), eps, _ptr(f), _ptr(g), _ptr(A), prob.d,
                                    float(tau), float(eta), int(max_cg), _ptr(out), prob.d, ctypes.byref(it)),
                    "fs_hvp")
        return out, it.value

    # ---- operators of a network trained on the losses --------------------------------
    def fs_attention(self, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, scale: Optional[float] = None, causal: bool = False,
                     q_len: Optional[torch.Tensor] = None, k_len: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None):
        """Softmax attention of q (sets, rows, heads, d) over k, v (sets, keys, kv heads, d); returns (o, stat).

        ``scale`` defaults to d^-1/2, ``bias`` (sets, keys) is added to the scores (log-weights; -inf removes a key), ``q_len``,
        ``k_len`` are the lengths of padded sets.  ``stat`` is what ``fs_attention_grad`` takes up."""
        a = _attn(q, k, v, scale, causal, q_len, k_len, bias)
        b, n, h, _ = shape = q.shape
        o, stat = q.new_empty(shape), q.new_empty((b, h, n, 2), dtype=torch.float32)
        self._check(self.lib.fs_attention(self.h, a, _HEADS.pack(*_heads(o, "o", shape, q.dtype)), stat.data_ptr()), "fs_attention")
        return o, stat

    def fs_attention_grad(self, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, o: torch.Tensor, stat: torch.Tensor, do: torch.Tensor,
                          scale: Optional[float] = None, causal: bool = False, q_len: Optional[torch.Tensor] = None,
                          k_len: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None, want_bias: bool = False):
        """Gradients of ``fs_attention`` (same mask arguments) for the gradient ``do`` of its output: (dq, dk, dv), with ``want_bias``
        (dq, dk, dv, dbias)."""
        a = _attn(q, k, v, scale, causal, q_len, k_len, bias)
        shape, dtype = q.shape, q.dtype
        _dev_f32(stat, "stat", (shape[0], shape[2], shape[1], 2))
        if want_bias and bias is None:
            raise ValueError("want_bias without a bias")
        g = [q.new_empty(t.shape) for t in (q, k, v)]
        db = q.new_empty(bias.shape) if want_bias else None
        h = [_HEADS.pack(*_heads(t, nm, sh, dtype)) for t, nm, sh in
             ((o, "o", shape), (do, "do", shape), (g[0], "dq", shape), (g[1], "dk", k.shape), (g[2], "dv", k.shape))]
        self._check(self.lib.fs_attention_grad(self.h, a, h[0], stat.data_ptr(), h[1], h[2], h[3], h[4],
                                               None if db is None else db.data_ptr(), k.shape[1]), "fs_attention_grad")
        return (*g, db) if want_bias else tuple(g)

    def fs_layer_norm(self, x: torch.Tensor, gamma: Optional[torch.Tensor] = None, beta: Optional[torch.Tensor] = None, eps: float = 1e-5):
        """Layer norm over the last dimension of x (rows, cols); returns (y, stat) with stat (rows, 2) = (mean, rstd)."""
        _matrix(x, "x")
        rows, cols = x.shape
        w = [_weights(gamma, "gamma", cols), _weights(beta, "beta", cols)]
        if gamma is not None and beta is not None and gamma.dtype != beta.dtype:
            raise TypeError("gamma and beta must have one type")
        wt = _DTYPES[gamma.dtype if gamma is not None else beta.dtype if beta is not None else torch.float32]
        y, stat = x.new_empty((rows, cols)), x.new_empty((rows, 2), dtype=torch.float32)
        self._check(self.lib.fs_layer_norm(self.h, x.data_ptr(), _DTYPES[x.dtype], rows, cols, _ld(x), w[0], w[1], wt, eps, y.data_ptr(), cols,
                                           stat.data_ptr()), "fs_layer_norm")
        return y, stat

    def fs_layer_norm_grad(self, x: torch.Tensor, gamma: Optional[torch.Tensor], stat: torch.Tensor, dy: torch.Tensor):
        """Gradients of ``fs_layer_norm`` for the gradient ``dy`` of its output; returns (dx, dgamma, dbeta), the last two float32."""
        _matrix(x, "x")
        _matrix(dy, "dy")
        rows, cols = x.shape
        if dy.shape != x.shape or dy.dtype != x.dtype:
            raise ValueError("dy must have the shape and type of x")
        _dev_f32(stat, "stat", (rows, 2))
        g = _weights(gamma, "gamma", cols)
        dx, dw = x.new_empty((rows, cols)), x.new_empty((2, cols), dtype=torch.float32)
        at = dw.data_ptr()
        self._check(self.lib.fs_layer_norm_grad(self.h, x.data_ptr(), _DTYPES[x.dtype], rows, cols, _ld(x), g,
                                                FS_F32 if gamma is None else _DTYPES[gamma.dtype], stat.data_ptr(), dy.data_ptr(), _ld(dy),
                                                dx.data_ptr(), cols, at, at + 4 * cols), "fs_layer_norm_grad")
        return (dx, *dw.unbind(0))

    def fs_points_keep(self, prob: Problem) -> None:
        """Declare the clouds of `prob` unchanged until fs_points_release: later calls reuse their derived copies."""
        self._check(self.lib.fs_points_keep(self.h, ctypes.byref(prob.c)), "fs_points_keep")

    def fs_points_release(self) -> None:
        self._check(self.lib.fs_points_release(self.h), "fs_points_release")

    def fs_debug_set(self, key: str, value: int) -> None:
        """Test and experiment switches of this context (0 = the library decides)."""
        self._check(self.lib.fs_debug_set(self.h, key.encode(), int(value)), "fs_debug_set")

    def fs_debug_get(self, key: str) -> int:
        v = ctypes.c_int64()
        self._check(self.lib.fs_debug_get(self.h, key.encode(), ctypes.byref(v)), "fs_debug_get")
        return v.value

    def fs_profile_enable(self, on: bool) -> None:
        self._check(self.lib.fs_profile_enable(self.h, 1 if on else 0), "fs_profile_enable")

    def fs_profile_read(self):
        avg, cnt, pairs = ctypes.c_double(), ctypes.c_int64(), ctypes.c_double()
        self._check(self.lib.fs_profile_read(self.h, ctypes.byref(avg), ctypes.byref(cnt),
                                             ctypes.byref(pairs)), "fs_profile_read")
        return avg.value, cnt.value, pairs.value


class AdamW:
    """AdamW over many tensors in one call of the library (``fs_adamw``): the weights are updated in place.

    ``state_bits`` 8 keeps m and sqrt(v) as float8 codes under a scale for every 256 weights.  ``master``: float copies of bf16
    weights.  The state is made here unless it is given (``m``, ``v``, ``m_scale``, ``v_scale``, and ``step``, the steps already taken);
    its tensors and the master copies stay the ones of the beginning: another state is copied into them.  A weight may be given
    other memory between steps, of the same size and type; what it had before is kept until the next step.
    """

    def __init__(self, ctx: Context, params, lr: float = 1e-3, betas=(0.9, 0.999), eps: float = 1e-8, weight_decay: float = 0.0,
                 state_bits: int = 32, master=None, m=None, v=None, m_scale=None, v_scale=None, step: int = 0, seed: int = 0):
        if state_bits not in (8, 32):
            raise ValueError("state_bits is 8 or 32")
        self.ctx, self.params, self.step_count, self.seed = ctx, list(params), int(step), int(seed)
        self.lr, self.betas, self.eps, self.weight_decay, self.state_bits = lr, betas, eps, weight_decay, state_bits
        if not self.params:
            raise ValueError("no weights")
        self.p_dtype = self.params[0].dtype
        if self.p_dtype not in _DTYPES:
            raise TypeError("weights must be float32 or bfloat16")
        kind = torch.float32 if state_bits == 32 else torch.float8_e4m3fn

        def made(given, dtype, count, fill):
            if given is None:
                return [torch.full((count(p),), fill, dtype=torch.float32, device=p.device).to(dtype) for p in self.params]
            if len(given) != len(self.params):
                raise ValueError("as many state tensors as weights")
            for t, p in zip(given, self.params):
                if not t.is_cuda or t.dtype != dtype or not t.is_contiguous() or t.numel() != count(p):
                    raise TypeError("a state tensor does not fit its weights")
            return list(given)

        self._check_params()
        self.m = made(m, kind, lambda p: p.numel(), 0.0)
        self.v = made(v, kind, lambda p: p.numel(), 0.0)
        self.m_scale = self.v_scale = self.master = None
        if state_bits == 8:
            self.m_scale = made(m_scale, torch.float32, lambda p: (p.numel() + 255) // 256, 1.0)
            self.v_scale = made(v_scale, torch.float32, lambda p: (p.numel() + 255) // 256, 1.0)
        if master is not None:
            self.master = made(master, torch.float32, lambda p: p.numel(), 0.0)
        self._table = (FsAdamwTensor * len(self.params))()
        lists = ((self.params, "p"), (self.m, "m"), (self.v, "v"), (self.m_scale, "m_scale"), (self.v_scale, "v_scale"), (self.master, "master"))
        for tensors, field in lists:
            for entry, t in zip(self._table, tensors or ()):
                setattr(entry, field, t.data_ptr())
        self._sizes = [p.numel() for p in self.params]
        for entry, n in zip(self._table, self._sizes):
            entry.n = n
        self._at = np.frombuffer(self._table, dtype=np.int64).reshape(len(self.params), 8)   # (the table's addresses: p, g, ...)
        wide = [p.element_size() for p in self.params]
        self._bytes = np.array([(n * w, n * 4 * (self.master is not None), *((n, n, (n + 255) // 256 * 4, (n + 255) // 256 * 4) if state_bits == 8 else
                                                                           (n * 4, n * 4, 0, 0))) for n, w in zip(self._sizes, wide)], dtype=np.int64)
        self._check_apart()
        self._p_at = list(map(torch.Tensor.data_ptr, self.params))
        # The memory behind the table's addresses lives as long as they are in it, whatever the tensors are made to point to meanwhile:
        # so no other tensor has an address of the table, and a weight at its address is the weight that was checked.
        self._held = [t.detach() for tensors, _ in lists for t in tensors or ()]
        self._args = FsAdamwArgs(p_dtype=_DTYPES[self.p_dtype], state_bits=state_bits)

    def _check_params(self):
        for p in self.params:
            if not p.is_cuda or p.dtype != self.p_dtype or not p.is_contiguous():
                raise TypeError("weights must be contiguous GPU tensors of one type")

    def _check_apart(self):
        """What a step writes does not overlap: a weight given twice, or one state for two, would be updated by two at once."""
        first, size = self._at[:, [0, 2, 3, 4, 5, 6]].ravel(), self._bytes.ravel()   # p, master, m, v, m_scale, v_scale
        first, size = first[size > 0], size[size > 0]
        order = np.argsort(first)
        if (first[order][:-1] + size[order][:-1] > first[order][1:]).any():
            raise ValueError("weights or states overlap each other")

    def step(self, grads, grad_scale: Optional[torch.Tensor] = None) -> None:
        """One step with these gradients (one type, contiguous, in the order of the weights).  ``grad_scale``: a float32 GPU scalar
        that they are multiplied by."""
        if len(grads) != len(self.params):
            raise ValueError("as many gradients as weights")
        kind = grads[0].dtype
        if kind not in _DTYPES:
            raise TypeError("gradients must be float32 or bfloat16")
        # (whole lists at a time: with many small tensors these checks are what a step costs)
        if (list(map(torch.Tensor.numel, grads)) != self._sizes or set(map(_get_dtype, grads)) != {kind} or not all(map(_get_is_cuda, grads))
                or not all(map(torch.Tensor.is_contiguous, grads))):
            raise TypeError("a gradient does not fit its weights")
        self._at[:, 1] = list(map(torch.Tensor.data_ptr, grads))
        p_at = list(map(torch.Tensor.data_ptr, self.params))
        if p_at != self._p_at:   # a weight was given other memory
            self._check_params()
            if list(map(torch.Tensor.numel, self.params)) != self._sizes:
                raise ValueError("a weight changed its size")
            before = self._at[:, 0].copy()
            self._at[:, 0] = p_at
            try:
                self._check_apart()
            except ValueError:
                self._at[:, 0] = before
                raise
            self._p_at = p_at
            self._held[:len(p_at)] = [p.detach() for p in self.params]
        a = self._args
        a.lr, (a.beta1, a.beta2), a.eps, a.weight_decay = self.lr, self.betas, self.eps, self.weight_decay
        a.step, a.g_dtype = self.step_count + 1, _DTYPES[kind]
        a.seed = (self.seed + self.step_count + 1) & 0xFFFFFFFF
        if grad_scale is not None and (not grad_scale.is_cuda or grad_scale.dtype != torch.float32 or grad_scale.numel() != 1):
            raise TypeError("grad_scale must be a float32 GPU scalar")
        a.grad_scale = None if grad_scale is None else grad_scale.data_ptr()
        self.ctx._check(self.ctx.lib.fs_adamw(self.ctx.h, ctypes.byref(a), self._table, len(self.params)), "fs_adamw")
        self.step_count += 1


def problem_from_workload(w, device="cuda:0") -> Problem:
    """Upload a ``workloads.Workload`` (host arrays) and wrap it as a Problem."""
    dev = torch.device(device)
    x = torch.from_numpy(w.x).to(dev)
    y = torch.from_numpy(w.y).to(dev)
    if w.storage == "bf16":
        x, y = x.to(torch.bfloat16), y.to(torch.bfloat16)   # exact: values are bf16-representable
    a = torch.from_numpy(w.a).to(dev)
    b = torch.from_numpy(w.b).to(dev)
    compute = FS_COMPUTE_BF16_MFMA if w.compute == "bf16_mfma" else FS_COMPUTE_FP32
    return Problem(x, y, a, b, compute)
