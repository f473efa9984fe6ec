"""Argument checks of the block's operators: they return before anything is launched, so they run without a
GPU.  Pointers here are plain numbers that nothing follows."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def L():
    from paper_2510_27258_gb300 import build, hla
    build.build()
    return hla.lib()


@pytest.fixture(scope="module")
def E():
    from paper_2510_27258_gb300 import hla
    return hla


BIG = 1 << 40


def test_glr_marks(L, E):
    assert [E.hla_glr_marks(n) for n in (0, 1, 32, 33, 64, 1 << 30)] == [0, 1, 1, 2, 2, 1 << 25]
    assert L.hla_glr_marks(-1) == 0


def glr(L, x=256, r=256, g=256, decay=256, y=256, dt=1, B=2, n=8, C=24, xs=24, rs=24, gs=24, ys=24, lengths=None, si=None,
        so=None, marks=None):
    return L.hla_glr_forward(x, r, g, decay, y, dt, B, n, C, xs, rs, gs, ys, lengths, si, so, marks, None)


def test_glr_forward_refuses(L, E):
    bad, no = E.HLA_ERR_INVALID_ARGUMENT, E.HLA_ERR_UNSUPPORTED
    for want, kw in ((bad, dict(x=None)), (bad, dict(r=None)), (bad, dict(g=None)), (bad, dict(decay=None)),
                     (bad, dict(y=None)), (bad, dict(dt=2)), (bad, dict(B=-1)), (bad, dict(n=-1)), (bad, dict(C=0)),
                     (bad, dict(xs=23)), (bad, dict(rs=0)), (bad, dict(gs=-24)), (bad, dict(ys=23)), (bad, dict(x=257)),
                     (bad, dict(decay=260)), (bad, dict(si=8)), (bad, dict(so=264)), (bad, dict(marks=4)),
                     (bad, dict(lengths=258)), (no, dict(B=1 << 20, n=1 << 20)), (no, dict(xs=1 << 39, n=1 << 10)),
                     (no, dict(C=(1 << 31) - 1, xs=1 << 31, rs=1 << 31, gs=1 << 31, ys=1 << 31)),
                     (no, dict(B=1 << 20, C=1 << 13, xs=1 << 13, rs=1 << 13, gs=1 << 13, ys=1 << 13))):
        assert glr(L, **kw) == want, kw
        assert L.hla_last_error()
    assert glr(L, B=0, x=None, r=None, g=None, decay=None, y=None) == E.HLA_OK
    assert glr(L, n=0, x=None, r=None, g=None, decay=None, y=None) == E.HLA_OK and L.hla_last_error() == b""


def test_glr_step_and_backward_refuse(L, E):
    bad = E.HLA_ERR_INVALID_ARGUMENT

    def step(state=256, xs=24, y=256, C=24):
        return L.hla_glr_step(256, 256, 256, 256, y, 1, 2, C, xs, 24, 24, 24, state, None)
    assert step(state=None) == bad and step(state=264) == bad and step(xs=23) == bad and step(y=None) == bad
    assert step(C=-1) == bad

    def back(dy=256, marks=256, dx=256, dr=256, dg=256, dd=256, n=8, dxs=24, drs=24, dgs=24, dys=24, ds=None, di=None, ws=256,
             ws_bytes=BIG):
        return L.hla_glr_backward(256, 256, 256, 256, dy, marks, dx, dr, dg, dd, 1, 2, n, 24, 24, 24, 24, dys, dxs, drs, dgs,
                                  None, ds, di, ws, ws_bytes, None)
    for kw in (dict(dy=None), dict(marks=None), dict(dx=None), dict(dr=None), dict(dg=None), dict(dd=None), dict(dxs=8),
               dict(drs=8), dict(dgs=8), dict(dys=8), dict(ds=8), dict(di=8), dict(dd=260), dict(marks=264), dict(ws=264)):
        assert back(**kw) == bad, kw
    assert back(ws=None) == E.HLA_ERR_WORKSPACE and back(ws_bytes=300) == E.HLA_ERR_WORKSPACE
    assert L.hla_glr_backward_workspace_bytes(2, 8, 24, 1) % 256 == 0
    assert L.hla_glr_backward_workspace_bytes(1, 1 << 16, 24, 0) >= 256 + 4 * 24 * 8  # a sum for each block of the sequence
    for sizes in ((2, 8, 0, 1), (-1, 8, 24, 1), (2, -8, 24, 1), (2, 8, 24, 3), (1 << 20, 1 << 20, 24, 1)):
        assert L.hla_glr_backward_workspace_bytes(*sizes) == 0


def norm(L, x=256, y=256, gate=256, wp=256, sc=256, wr=256, xo=256, h=256, dt=1, rows=8, C=24, xs=24, ys=24, gs=24, xos=24,
         hs=24, post=1, pre=1, act=2, alpha=1.0, eps=1e-6, drop=0.1, seed=1, offset=2):
    return L.hla_block_norm_forward(x, y, gate, wp, sc, wr, xo, h, dt, rows, C, xs, ys, gs, xos, hs, post, pre, act,
                                    ctypes.c_float(alpha), ctypes.c_float(eps), ctypes.c_double(drop), seed, offset, None)


def test_block_norm_refuses(L, E):
    bad, no = E.HLA_ERR_INVALID_ARGUMENT, E.HLA_ERR_UNSUPPORTED
    nan, inf = float("nan"), float("inf")
    for want, kw in ((bad, dict(x=None)), (bad, dict(y=None)), (bad, dict(xo=None)), (bad, dict(h=None)), (bad, dict(dt=5)),
                     (bad, dict(rows=-1)), (bad, dict(C=0)), (bad, dict(xs=23)), (bad, dict(ys=1)), (bad, dict(gs=23)),
                     (bad, dict(xos=0)), (bad, dict(hs=23)), (bad, dict(post=2)), (bad, dict(pre=-1)), (bad, dict(act=3)),
                     (bad, dict(act=-1)), (bad, dict(alpha=inf)), (bad, dict(alpha=nan)), (bad, dict(eps=-1.0)),
                     (bad, dict(eps=nan)), (bad, dict(drop=1.0)), (bad, dict(drop=-0.1)), (bad, dict(drop=nan)),
                     (bad, dict(wp=257)), (bad, dict(sc=257)), (bad, dict(wr=257)), (bad, dict(gate=257)),
                     (no, dict(C=1 << 30, xs=1 << 30, ys=1 << 30, gs=1 << 30, xos=1 << 30, hs=1 << 30)),
                     (no, dict(xs=1 << 38))):
        assert norm(L, **kw) == want, kw
    assert norm(L, rows=0, x=None, y=None, gate=None, xo=None, h=None, wp=None, sc=None, wr=None) == E.HLA_OK
    # a norm that is off asks for nothing of its own
    assert norm(L, rows=0, pre=0, h=None, wr=257) == E.HLA_OK and norm(L, rows=0, post=0, wp=257) == E.HLA_OK


def test_block_norm_backward_refuses(L, E):
    bad = E.HLA_ERR_INVALID_ARGUMENT

    def back(gate=256, dxo=256, dh=256, dx=256, dy=256, dg=256, dwp=256, dsc=256, dwr=256, rows=8, dxs=24, dgs=24, drop=0.0,
             ws=256, ws_bytes=BIG):
        return L.hla_block_norm_backward(256, 256, gate, None, None, None, dxo, dh, dx, dy, dg, dwp, dsc, dwr, 0, rows, 24, 24,
                                         24, 24, 24, 24, dxs, 24, dgs, 1, 1, 2, ctypes.c_float(1), ctypes.c_float(1e-6),
                                         ctypes.c_double(drop), 0, 0, ws, ws_bytes, None)
    for kw in (dict(dxo=None), dict(dh=None), dict(dx=None), dict(dy=None), dict(dg=None), dict(dxs=2), dict(dgs=2),
               dict(dwp=258), dict(dsc=258), dict(dwr=258), dict(drop=1.5), dict(ws=260)):
        assert back(**kw) == bad, kw
    assert back(ws=None) == E.HLA_ERR_WORKSPACE and back(ws_bytes=0) == E.HLA_ERR_WORKSPACE
    assert L.hla_block_norm_backward_workspace_bytes(8, 24, 0) % 256 == 0
    assert L.hla_block_norm_backward_workspace_bytes(8, 0, 0) == L.hla_block_norm_backward_workspace_bytes(8, 24, 2) == 0
    assert L.hla_block_norm_backward_workspace_bytes(-8, 24, 0) == L.hla_block_norm_backward_workspace_bytes(8, 1 << 30, 0) == 0


def test_ffn_refuses(L, E):
    bad, no = E.HLA_ERR_INVALID_ARGUMENT, E.HLA_ERR_UNSUPPORTED

    def fwd(x=256, w=256, out=256, dt=1, M=8, K=24, F=40, xs=24, os=40, act=2, ws=256, ws_bytes=BIG):
        return L.hla_ffn_forward(x, w, out, dt, M, K, F, xs, os, act, ws, ws_bytes, None)
    for want, kw in ((bad, dict(x=None)), (bad, dict(w=None)), (bad, dict(out=None)), (bad, dict(dt=2)), (bad, dict(M=-1)),
                     (bad, dict(K=0)), (bad, dict(F=0)), (bad, dict(xs=23)), (bad, dict(os=39)), (bad, dict(act=3)),
                     (bad, dict(x=257)), (bad, dict(w=257)), (bad, dict(out=257)), (bad, dict(ws=264)),
                     (E.HLA_ERR_WORKSPACE, dict(ws=None)), (E.HLA_ERR_WORKSPACE, dict(ws_bytes=100)),
                     (no, dict(M=(1 << 26) + 1)), (no, dict(K=1 << 27, xs=1 << 27)), (no, dict(F=1 << 27, os=1 << 27)),
                     (no, dict(K=1 << 21, F=1 << 20, xs=1 << 21, os=1 << 20))):
        assert fwd(**kw) == want, kw

    def back(dout=256, dx=256, dw=256, dos=40, dxs=24, ws=256, ws_bytes=BIG):
        return L.hla_ffn_backward(256, 256, dout, dx, dw, 1, 8, 24, 40, 24, dos, dxs, 2, ws, ws_bytes, None)
    for kw in (dict(dout=None), dict(dx=None), dict(dw=None), dict(dos=39), dict(dxs=23), dict(dw=257), dict(ws=264)):
        assert back(**kw) == bad, kw
    assert back(ws=None) == E.HLA_ERR_WORKSPACE and back(ws_bytes=300) == E.HLA_ERR_WORKSPACE
    for f in (L.hla_ffn_workspace_bytes, L.hla_ffn_backward_workspace_bytes):
        assert f(8, 24, 40, 1) % 256 == 0 and f(8, 24, 40, 0) >= 256
        assert f(-8, 24, 40, 1) == f(8, 0, 40, 1) == f(8, 24, 0, 1) == f(8, 24, 40, 2) == 0
    # what the gradient keeps between its products fits
    assert L.hla_ffn_backward_workspace_bytes(300, 24, 41, 1) >= 256 + 2 * 2 * 300 * 48
    assert L.hla_ffn_backward_workspace_bytes(300, 24, 41, 0) >= 256 + 4 * 300 * 82
