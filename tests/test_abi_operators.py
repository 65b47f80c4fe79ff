"""Host-side checks of the norm, optimizer and few-token calls: arguments are rejected before any launch (no GPU is needed: the
pointers are never followed), sizes are right."""
import ctypes

import pytest

from test_abi import lib

NULL, SHAPE, FORMAT, LAYOUT, WORKSPACE = 1, 2, 3, 4, 5
P = ctypes.c_void_p(0x10000)


@pytest.fixture(scope="module")
def S():
    return lib()


def q(S, rows, cols, fmt=0, codes=0x10000, scales=0x10000, g4=0):
    return S._QTensorC(codes, scales, g4 or None, rows, cols, fmt)


def norm(S, x=P, rows=32, cols=64, ld=64, r=None, ldr=64, w=P, wd=0, eps=1e-5, rule=0, s=None, lds=64, rstd=P, y=P, ldy=64, row=None, col=None):
    ref = lambda t: ctypes.byref(t) if t is not None else None  # noqa: E731
    return S._lib().snip_rms_norm(x, rows, cols, ld, r, ldr, w, wd, eps, rule, s, lds, rstd, y, ldy, ref(row), ref(col), None)


def test_rms_norm(S):
    assert norm(S, x=None) == NULL and norm(S, w=None) == NULL
    assert norm(S, rows=-1) == SHAPE and norm(S, cols=0, ld=0) == SHAPE and norm(S, ld=56) == SHAPE and norm(S, ldy=8) == SHAPE
    assert norm(S, ld=68) == LAYOUT and norm(S, x=ctypes.c_void_p(0x10008)) == LAYOUT and norm(S, w=ctypes.c_void_p(0x10002)) == LAYOUT
    assert norm(S, rstd=ctypes.c_void_p(0x10002)) == LAYOUT
    assert norm(S, wd=2) == FORMAT and norm(S, rule=2) == FORMAT and norm(S, eps=-1e-9) == FORMAT and norm(S, eps=float("inf")) == FORMAT
    assert norm(S, s=P) == NULL                                             # a sum without a residual
    assert norm(S, rstd=None, y=None) == NULL                               # no output
    assert norm(S, r=P, ldr=60) == SHAPE and norm(S, r=P, ldr=68) == LAYOUT
    assert norm(S, row=q(S, 32, 32)) == SHAPE and norm(S, row=q(S, 32, 64, 2)) == FORMAT and norm(S, row=q(S, 32, 64, codes=None)) == NULL
    assert norm(S, row=q(S, 32, 64, codes=0x10004)) == LAYOUT and norm(S, row=q(S, 32, 64, scales=0x10002)) == LAYOUT and norm(S, row=q(S, 32, 64, g4=0x10004)) == LAYOUT
    assert norm(S, cols=40, row=q(S, 32, 40)) == SHAPE and norm(S, rows=24, col=q(S, 64, 24)) == SHAPE and norm(S, cols=63, col=q(S, 63, 32)) == SHAPE
    assert norm(S, rstd=None, col=q(S, 64, 32)) == NULL                      # columns need the rows' norms
    assert norm(S, r=P, col=q(S, 64, 32)) == NULL                            # and what was normed
    assert norm(S, rows=0) == 0 and norm(S, rows=0, x=None, rstd=None, y=None, row=q(S, 0, 64, codes=None, scales=None)) == 0


def test_rms_norm_backward(S):
    def back(dy=P, rows=8, cols=64, ld=64, h=P, w=P, wd=0, rstd=P, ds=None, lds=64, dx=P, ldx=64, dw=P, ws=P, n=1 << 20):
        return S._lib().snip_rms_norm_backward(dy, rows, cols, ld, h, 64, w, wd, rstd, ds, lds, dx, ldx, dw, ws, n, None)
    assert back(dy=None) == NULL and back(h=None) == NULL and back(rstd=None) == NULL and back(dx=None) == NULL and back(w=None) == NULL
    assert back(ld=32) == SHAPE and back(ldx=60) == SHAPE and back(ds=P, lds=60) == SHAPE and back(ds=P, lds=68) == LAYOUT and back(rows=1 << 31) == SHAPE
    assert back(wd=-1) == FORMAT and back(dw=ctypes.c_void_p(0x10002)) == LAYOUT
    assert back(ws=None) == WORKSPACE and back(n=16) == WORKSPACE and back(ws=ctypes.c_void_p(0x10008)) == LAYOUT
    size = S.rms_norm_workspace_bytes
    assert size(0, 64) == 0 and size(-1, 64) == 0 and size(8, 0) == 0
    assert 0 < size(8, 64) <= 8 * 64 * 4 and size(3, 13) == 3 * 16 * 4       # a row of sums for each row at most, of a multiple of 8 columns
    assert size(1 << 20, 4096) == size(1 << 16, 4096) <= 32 << 20


class AdamwC(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("param", "grad", "m", "v", "copy", "m_scale", "v_scale")] + \
               [("n", ctypes.c_int64), ("weight_decay", ctypes.c_float), ("grad_dtype", ctypes.c_int32)]


def test_adamw_step(S):
    def step(count=1, lr=1e-3, b1=0.9, b2=0.95, eps=1e-8, t=1, gs=None, **kw):
        d = dict(param=0x10000, grad=0x10000, m=0x10000, v=0x10000, copy=None, m_scale=None, v_scale=None, n=64, weight_decay=0.0, grad_dtype=0) | kw
        a = (AdamwC * 1)(AdamwC(**d))
        return S._lib().snip_adamw_step(a if count else None, count, lr, b1, b2, eps, t, gs, 0, None)
    assert step(count=0) == 0 and step(count=-1) == SHAPE
    assert S._lib().snip_adamw_step(None, 1, 1e-3, 0.9, 0.95, 1e-8, 1, None, 0, None) == NULL
    for name in ("param", "grad", "m", "v"):
        assert step(**{name: None}) == NULL and step(**{name: 0x10001}) == LAYOUT
    assert step(m_scale=0x10000) == NULL and step(v_scale=0x10000) == NULL and step(m_scale=0x10002, v_scale=0x10000) == LAYOUT
    assert step(copy=0x10001) == LAYOUT and step(grad=0x10002, grad_dtype=1) == LAYOUT and step(gs=ctypes.c_void_p(0x10002)) == LAYOUT
    assert step(n=-1) == SHAPE and step(n=1 << 34) == SHAPE
    for kw in ({"b1": 1.0}, {"b1": -0.1}, {"b2": 1.0}, {"eps": -1.0}, {"eps": float("inf")}, {"lr": float("nan")}, {"t": 0}, {"weight_decay": float("nan")}, {"grad_dtype": 2}):
        assert step(**kw) == FORMAT, kw
    assert step(n=0, param=None, grad=None, m=None, v=None) == 0


def test_gemv(S):
    def gemv(x=P, m=4, k=64, ld=64, w=None, y=0x10000, ldy=16, dt=0, count=1):
        a = (S._QTensorC * 1)(w if w is not None else q(S, 16, 64, 1))
        return S._lib().snip_gemv(x, m, k, ld, a, (ctypes.c_void_p * 1)(y), (ctypes.c_int64 * 1)(ldy), count, dt, None)
    assert gemv(x=None) == NULL and gemv(y=None) == NULL and gemv(w=q(S, 16, 64, 1, codes=None)) == NULL
    assert S._lib().snip_gemv(P, 4, 64, 64, None, None, None, 1, 0, None) == NULL
    assert gemv(m=-1) == SHAPE and gemv(m=65537) == SHAPE and gemv(k=48) == SHAPE and gemv(k=0, ld=0) == SHAPE and gemv(ld=32) == SHAPE and gemv(count=-1) == SHAPE
    assert gemv(ldy=8) == SHAPE and gemv(w=q(S, -1, 64, 1)) == SHAPE and gemv(w=q(S, (1 << 27) + 1, 64, 1), ldy=1 << 28) == SHAPE
    assert gemv(ld=68) == LAYOUT and gemv(w=q(S, 16, 96, 1)) == LAYOUT and gemv(y=0x10008) == LAYOUT and gemv(ldy=20) == LAYOUT and gemv(ldy=18, dt=1) == LAYOUT
    assert gemv(dt=2) == FORMAT and gemv(w=q(S, 16, 64, 2)) == FORMAT
    assert gemv(count=0) == 0 and gemv(m=0, x=None) == 0 and gemv(w=q(S, 0, 64, 1, codes=None, scales=None), y=None) == 0
