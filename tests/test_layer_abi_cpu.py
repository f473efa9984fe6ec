"""Argument checks of the operators around the mixers: they return before anything is launched, so
they run without a GPU.  Pointers here are plain numbers that nothing follows."""
import ctypes

import pytest
import torch


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


def conv(L, x=256, w=256, bias=256, out=256, dt=1, B=2, n=8, C=24, width=4, xs=24, os=24, silu=1, lengths=None,
         si=None, so=None):
    return L.hla_conv_forward(x, w, bias, out, dt, B, n, C, width, xs, os, silu, lengths, si, so, None)


def test_conv_forward_refuses(L, E):
    bad, no = E.HLA_ERR_INVALID_ARGUMENT, E.HLA_ERR_UNSUPPORTED
    for want, kw in ((bad, dict(x=None)), (bad, dict(w=None)), (bad, dict(out=None)), (bad, dict(dt=2)), (bad, dict(B=-1)),
                     (bad, dict(n=-1)), (bad, dict(C=0)), (bad, dict(width=0)), (no, dict(width=5)), (no, dict(width=1)),
                     (bad, dict(xs=23)), (bad, dict(os=23)), (bad, dict(silu=2)), (bad, dict(x=257)), (bad, dict(so=3)),
                     (bad, dict(lengths=2)), (no, dict(B=1 << 20, n=1 << 20)), (no, dict(xs=1 << 39, n=1 << 10))):
        assert conv(L, **kw) == want, kw
        assert L.hla_last_error()
    assert conv(L, B=0, x=None, out=None) == E.HLA_OK
    assert conv(L, n=0, x=None, out=None) == E.HLA_OK and L.hla_last_error() == b""


def test_conv_step_and_backward_refuse(L, E):
    bad = E.HLA_ERR_INVALID_ARGUMENT

    def step(state=256, width=4, xs=24):
        return L.hla_conv_step(256, 256, None, 256, 1, 2, 24, width, xs, 24, 1, state, None)
    assert step(state=None) == bad and step(xs=0) == bad and step(width=6) == E.HLA_ERR_UNSUPPORTED

    def back(dout=256, dx=256, dw=256, ws=256, ws_bytes=BIG, ds=24, B=2):
        return L.hla_conv_backward(256, 256, None, dout, dx, dw, None, 1, B, 8, 24, 4, 24, 24, ds, 1, None, ws, ws_bytes,
                                   None)
    assert back(dout=None) == bad and back(dx=None) == bad and back(dw=None) == bad and back(ds=8) == bad
    assert back(ws=None) == E.HLA_ERR_WORKSPACE and back(ws_bytes=300) == E.HLA_ERR_WORKSPACE
    assert back(ws=264) == bad
    assert L.hla_conv_backward_workspace_bytes(2, 8, 24, 4, 1) % 256 == 0
    assert L.hla_conv_backward_workspace_bytes(2, 8, 24, 5, 1) == 0
    assert L.hla_conv_backward_workspace_bytes(2, 8, 24, 4, 3) == 0


def ssm(L, x=256, delta=256, a=256, b=256, c=256, skip=None, bias=None, y=256, dt=1, B=2, n=8, H=4, P=32, G=2, N=16,
        xs=128, ds=4, bs=32, cs=32, ys=128, softplus=1, lengths=None, si=None, so=None, ws=256, ws_bytes=BIG):
    return L.hla_ssm_forward(x, delta, a, b, c, skip, bias, y, dt, B, n, H, P, G, N, xs, ds, bs, cs, ys, softplus,
                             lengths, si, so, ws, ws_bytes, None)


def test_ssm_forward_refuses(L, E):
    bad, no = E.HLA_ERR_INVALID_ARGUMENT, E.HLA_ERR_UNSUPPORTED
    for want, kw in ((bad, dict(x=None)), (bad, dict(delta=None)), (bad, dict(a=None)), (bad, dict(b=None)),
                     (bad, dict(c=None)), (bad, dict(y=None)), (bad, dict(dt=9)), (bad, dict(G=3)), (bad, dict(H=0)),
                     (no, dict(P=48, xs=192, ys=192)), (no, dict(N=256, bs=512, cs=512)), (bad, dict(xs=127)),
                     (bad, dict(ds=3)), (bad, dict(bs=31)), (bad, dict(cs=31)), (bad, dict(ys=1)), (bad, dict(softplus=7)),
                     (bad, dict(si=8)), (bad, dict(so=8)), (bad, dict(a=257)), (bad, dict(lengths=258)),
                     (E.HLA_ERR_WORKSPACE, dict(ws=None)), (E.HLA_ERR_WORKSPACE, dict(ws_bytes=1)), (bad, dict(ws=272))):
        assert ssm(L, **kw) == want, kw
    assert ssm(L, B=0, x=None, y=None, delta=None, a=None, b=None, c=None) == E.HLA_OK
    assert L.hla_ssm_workspace_bytes(2, 8, 4, 32, 3, 16, 1) == 0
    assert L.hla_ssm_workspace_bytes(2, 8, 4, 24, 2, 16, 1) == 0
    assert L.hla_ssm_workspace_bytes(1, 1 << 16, 4, 32, 2, 16, 0) > L.hla_ssm_workspace_bytes(1, 8, 4, 32, 2, 16, 0) > 0


def test_ssm_path_without_a_device(L, E):
    assert E.hla_ssm_forward_path(8, 2048, 32, 64, 1, 128) == (0, 1)  # no device here: the fp32 kernels
    assert E.hla_ssm_forward_path(1, 2048, 4, 64, 1, 128, dtype=torch.float32) == (0, 3)  # few heads: segments
    assert E.hla_ssm_forward_path(0, 2048, 4, 64, 1, 128) == (0, 0)
    assert E.hla_ssm_forward_path(1, 2048, 4, 48, 1, 128) == (-1, 0)


def test_ssm_step_refuses(L, E):
    def step(state=256, P=32, xs=128, delta=256):
        return L.hla_ssm_step(256, delta, 256, 256, 256, None, None, 256, 1, 2, 4, P, 2, 16, xs, 4, 32, 32, 128, 1, state,
                              None)
    bad = E.HLA_ERR_INVALID_ARGUMENT
    assert step(state=None) == bad and step(state=264) == bad and step(xs=64) == bad and step(delta=None) == bad
    assert step(P=8) == E.HLA_ERR_UNSUPPORTED


def qk(L, q=256, k=256, wq=None, wk=None, cos=256, sin=256, pos=None, qo=256, ko=256, dt=1, B=2, n=8, H=4, Hk=2, d=32,
       rot=16, inter=0, qs=128, ks=64, pos0=0, top=8, eps=1e-6):
    return L.hla_qk_norm_forward(q, k, wq, wk, cos, sin, pos, qo, ko, dt, B, n, H, Hk, d, rot, inter, qs, ks, pos0, top,
                                 ctypes.c_float(eps), None)


def test_qk_norm_refuses(L, E):
    bad, no = E.HLA_ERR_INVALID_ARGUMENT, E.HLA_ERR_UNSUPPORTED
    for want, kw in ((bad, dict(q=None)), (bad, dict(k=None)), (bad, dict(qo=None)), (bad, dict(ko=None)),
                     (bad, dict(cos=None)), (bad, dict(sin=None)), (bad, dict(Hk=3)), (bad, dict(Hk=0)), (bad, dict(rot=40)),
                     (bad, dict(rot=-8)), (no, dict(rot=12)), (no, dict(d=48, qs=192, ks=96)), (bad, dict(qs=64)),
                     (bad, dict(ks=32)), (bad, dict(top=7)), (bad, dict(pos0=1)), (bad, dict(pos0=-1)), (bad, dict(eps=-1.)),
                     (bad, dict(eps=float("nan"))), (bad, dict(inter=3)), (bad, dict(qo=264)), (bad, dict(cos=264)),
                     (bad, dict(pos=258)), (bad, dict(q=257)), (bad, dict(dt=-1))):
        assert qk(L, **kw) == want, kw
    assert qk(L, n=0, q=None, k=None, qo=None, ko=None) == E.HLA_OK

    def back(dqo=256, dq=256, dqs=128, ws=256, ws_bytes=BIG, dwq=256):
        return L.hla_qk_norm_backward(256, 256, None, None, 256, 256, None, dqo, 256, dq, 256, dwq, None, 1, 2, 8, 4, 2, 32,
                                      16, 0, 128, 64, dqs, 64, 0, 8, ctypes.c_float(1e-6), ws, ws_bytes, None)
    assert back(dqo=None) == bad and back(dq=None) == bad and back(dqs=100) == bad and back(dwq=258) == bad
    assert back(ws=None) == E.HLA_ERR_WORKSPACE and back(ws_bytes=0) == E.HLA_ERR_WORKSPACE and back(ws=260) == bad
    assert L.hla_qk_norm_backward_workspace_bytes(2, 8, 4, 3, 32, 1) == 0
    assert L.hla_qk_norm_backward_workspace_bytes(2, 8, 4, 2, 32, 1) % 256 == 0


def test_row_strides_of_the_binding(E):
    T, dev = torch.float32, torch.device("cpu")
    f = lambda t, lead: E._row_stride("t", t, lead, t.shape, T, dev)  # noqa: E731
    wide = torch.zeros(2, 5, 40)
    assert f(wide[..., :24], 2) == 40 and f(wide[:, 0, :24], 1) == 200
    assert f(wide[..., 8:].unflatten(-1, (4, 8)), 2) == 40
    assert f(torch.zeros(3, 1, 7), 2) == 7 and f(torch.zeros(1, 3, 7), 2) == 7
    for t in (wide[..., ::2], wide[:, ::2], wide.transpose(1, 2)):
        with pytest.raises(ValueError):
            f(t, 2)
    with pytest.raises(ValueError):
        E._row_stride("t", wide, 2, (2, 5, 41), T, dev)
    with pytest.raises(ValueError):
        E.hla_conv_forward(wide, torch.zeros(40, 4))  # no CUDA tensor
