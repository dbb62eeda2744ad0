"""include/mx_b128.h and include/mx_norm.h: everything declared is exported, argument validation returns the documented codes before anything
is launched, and the binding refuses what does not fit.  No GPU needed."""
import os
import re

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, NULL, ENUM, SHAPE, ALIGN, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3, 4, 5, 8
P = 0x1000                                    # an aligned address; validation fails before it is used


@pytest.fixture(scope="module")
def L():
    from paper_2310_10537_amd import binding
    if not os.path.exists(binding._LIB_PATH):
        from paper_2310_10537_amd import build
        build.build()
    return binding.lib()


def declared(header):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", header)).read(), flags=re.S)
    return set(re.findall(r"\b(mx_[a-z0-9_]+)\s*\(", text))


def test_exports_match_headers(L):
    assert declared("mx_b128.h") == {"mx_b128_elem_bytes", "mx_b128_scale_count", "mx_quantize_b128", "mx_dequantize_b128", "mx_gemm_b128"}
    assert declared("mx_norm.h") == {"mx_rmsnorm", "mx_rmsnorm_q", "mx_rmsnorm_b128", "mx_rmsnorm_bwd", "mx_rmsnorm_bwd_ws", "mx_rmsnorm_bwd_workspace_bytes"}
    for n in declared("mx_b128.h") | declared("mx_norm.h"):
        assert hasattr(L, n), n


def test_sizes(L):
    assert L.mx_b128_elem_bytes(10, 129, 1) == 10 * 256 and L.mx_b128_elem_bytes(10, 129, 0) == 129 * 128
    assert L.mx_b128_scale_count(300, 129, 1, 0) == 600 and L.mx_b128_scale_count(300, 129, 1, 1) == 6
    assert L.mx_b128_scale_count(300, 129, 0, 0) == 129 * 3 and L.mx_b128_scale_count(300, 129, 0, 1) == 6
    assert L.mx_b128_elem_bytes(-1, 5, 1) == L.mx_b128_elem_bytes(1, 5, 2) == L.mx_b128_scale_count(1, 5, 1, 2) == 0
    assert L.mx_b128_elem_bytes(0, 5, 1) == 0 and L.mx_b128_elem_bytes(1 << 20, 1 << 20, 1) == 1 << 40
    assert L.mx_rmsnorm_bwd_workspace_bytes(0, 100) == 0 and L.mx_rmsnorm_bwd_workspace_bytes(1, 1) >= 4


def test_cast_status_codes(L):
    for q in (lambda src=P, dt=1, rows=64, cols=256, ld=256, axis=1, tile=0, fmt=0, e=P, s=P: L.mx_quantize_b128(src, dt, rows, cols, ld, axis, tile, fmt, e, s, None),
              lambda src=P, dt=1, rows=64, cols=256, ld=256, axis=1, tile=0, fmt=0, e=P, s=P: L.mx_dequantize_b128(e, s, fmt, rows, cols, axis, tile, src, dt, ld, None)):
        for fmt in (-1, 2, 3, 4, 5, 6):
            assert q(fmt=fmt) == ENUM
        assert q(dt=2) == q(axis=2) == q(axis=-1) == q(tile=2) == ENUM
        assert q(rows=-1) == q(cols=-1) == q(ld=255) == SHAPE
        assert q(src=None) == q(e=None) == q(s=None) == NULL
        assert q(src=P + 2) == q(e=P + 8) == q(s=P + 4) == q(ld=260) == ALIGN
        assert q(src=None, rows=0) == q(src=None, cols=0) == OK
    # more tiles, or longer lines, than a launch can number
    assert L.mx_quantize_b128(P, 1, 1 << 40, 256, 256, 1, 1, 0, P, P, None) == UNSUPPORTED
    assert L.mx_quantize_b128(P, 1, 1 << 40, 256, 256, 0, 0, 0, P, P, None) == UNSUPPORTED
    assert L.mx_quantize_b128(P, 1, 1, 1 << 36, 1 << 36, 1, 0, 0, P, P, None) == UNSUPPORTED
    assert L.mx_dequantize_b128(P, P, 0, 1 << 40, 256, 0, 0, P, 1, 256, None) == UNSUPPORTED
    assert L.mx_dequantize_b128(P, P, 0, 1, 1 << 36, 1, 0, P, 1, 1 << 36, None) == UNSUPPORTED


def test_product_status_codes(L):
    def g(M=16, N=32, K=256, a=P, sa=P, ta=0, fa=0, b=P, sb=P, tb=1, fb=0, c=P, dt=1, ldc=32):
        return L.mx_gemm_b128(M, N, K, a, sa, ta, fa, b, sb, tb, fb, c, dt, ldc, None)
    assert g(fa=2) == g(fb=5) == g(fa=-1) == g(dt=2) == g(ta=2) == g(tb=-1) == ENUM
    assert g(K=130) == g(K=64) == g(M=-1) == g(N=-1) == g(K=-128) == g(ldc=31) == SHAPE
    assert g(a=None) == g(sa=None) == g(b=None) == g(sb=None) == g(c=None) == NULL
    assert g(a=P + 8) == g(sa=P + 4) == g(b=P + 8) == g(sb=P + 4) == g(c=P + 8) == ALIGN
    assert g(M=0, a=None) == g(N=0, c=None, ldc=0) == OK
    assert g(K=0, a=None, sa=None, b=None, sb=None, c=None) == NULL
    assert g(M=1 << 30, N=1 << 30, ldc=1 << 30) == g(K=1 << 39) == UNSUPPORTED


def test_norm_status_codes(L):
    def f(which, x=P, ldx=64, r=None, ldr=0, w=P, wdt=0, dt=1, rows=4, cols=64, eps=1e-5, fmt=0, rnd=0, e=P, s=P, h=None, ldh=0, y=P, ldy=64, rstd=None):
        head, tail = (x, ldx, r, ldr, w, wdt, dt, rows, cols, eps), (h, ldh, y, ldy, rstd, None)
        return (L.mx_rmsnorm(*head, *tail) if which == 0 else L.mx_rmsnorm_q(*head, fmt, rnd, e, s, *tail) if which == 1 else L.mx_rmsnorm_b128(*head, fmt, e, s, *tail))
    for k in range(3):
        bad = lambda **kw: f(k, **kw)  # noqa: E731
        assert bad(dt=2) == bad(wdt=3) == bad(eps=-1.0) == bad(eps=float("nan")) == bad(eps=float("inf")) == ENUM
        assert bad(w=None, wdt=3, x=None) == NULL              # the type of an absent weight is not looked at
        assert bad(rows=-1) == bad(cols=-1) == bad(ldx=63) == bad(r=P, ldr=63) == bad(h=P, ldh=8) == bad(ldy=63) == SHAPE
        assert bad(x=None) == NULL
        assert bad(x=P + 2) == bad(ldx=68) == bad(r=P + 8, ldr=64) == bad(r=P, ldr=68) == bad(h=P, ldh=68) == bad(y=P + 4) == bad(w=P + 4) == bad(rstd=P + 2) == ALIGN
        assert bad(rows=0, x=None) == bad(cols=0, x=None) == OK
        assert bad(rows=1 << 31) == bad(cols=1 << 32, ldx=1 << 32, ldy=1 << 32) == UNSUPPORTED
    assert f(0, y=None) == f(1, e=None) == f(1, s=None) == f(2, e=None) == f(2, s=None) == NULL
    assert f(1, e=P + 8) == f(2, s=P + 4) == ALIGN
    assert f(1, fmt=6) == f(1, fmt=-1) == f(1, rnd=3) == f(1, rnd=-1) == f(2, fmt=2) == f(2, fmt=5) == ENUM


def test_gradient_status_codes(L):
    def f(dy=P, lddy=64, h=P, ldh=64, w=P, wdt=0, rstd=P, dh=None, lddh=0, dt=1, rows=4, cols=64, dx=P, lddx=64, dw=P, ws=None, wb=0):
        return L.mx_rmsnorm_bwd_ws(dy, lddy, h, ldh, w, wdt, rstd, dh, lddh, dt, rows, cols, dx, lddx, dw, ws, wb, None)
    assert f(dt=2) == f(wdt=2) == ENUM
    assert f(rows=-1) == f(cols=-1) == f(lddy=63) == f(ldh=63) == f(lddx=63) == f(dh=P, lddh=63) == SHAPE
    assert f(dy=None) == f(h=None) == f(rstd=None) == f(dx=None) == NULL
    assert f(dy=P + 2) == f(h=P + 8) == f(dh=P + 8, lddh=64) == f(dx=P + 4) == f(lddx=68) == f(w=P + 4) == f(dw=P + 4) == f(rstd=P + 1) == ALIGN
    assert f(rows=0, dw=None, dy=None) == f(cols=0, dy=None) == OK
    assert f(rows=1 << 31) == f(cols=1 << 32, lddy=1 << 32, ldh=1 << 32, lddx=1 << 32) == UNSUPPORTED
    assert f(ws=P, wb=8) == WORKSPACE and f(ws=P + 8, wb=1 << 30) == ALIGN
    assert L.mx_rmsnorm_bwd(None, 64, P, 64, P, 0, P, None, 0, 1, 4, 64, P, 64, P, None) == NULL


def test_binding_refuses_host_tensors():
    from paper_2310_10537_amd import binding as mx
    x = torch.zeros((32, 128))
    for call in (lambda: mx.mx_quantize_b128(x, 1, 0), lambda: mx.mx_dequantize_b128(x, x, 0, 32, 128, 1), lambda: mx.mx_gemm_b128(x, x, 0, x, x, 0, 128),
                 lambda: mx.mx_rmsnorm(x, None, 1e-5), lambda: mx.mx_rmsnorm_q(x, None, 1e-5, 0), lambda: mx.mx_rmsnorm_b128(x, None, 1e-5, 0),
                 lambda: mx.mx_rmsnorm_bwd(x, x, None, x[:, 0])):
        with pytest.raises(ValueError):
            call()
