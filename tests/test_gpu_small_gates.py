"""fp32 gates far below zero: what a sigmoid of e^v makes there is as exact as elsewhere.  A sigmoid is an exponential (2 units
of 2^-24 of it), a sum, a reciprocal (2 units) and the products around it, less than 8 roundings in all: 2^-21.  (An
exponential as a power of two of a rounded product is off by |v| 2^-23, which is 2^-17 at the ends here.)"""
import pytest
import torch

from test_gpu_block import DEV, on

pytestmark = pytest.mark.gpu
ROOM = 2.0 ** -21


@pytest.fixture(scope="module")
def hla():
    from paper_2510_27258_gb300 import build
    build.build()
    from paper_2510_27258_gb300 import hla as binding
    return binding


def off(got, want):
    return float(((got.double().cpu() - want) / want).abs().max())


def gates(lo, hi, *shape):
    n = 1
    for v in shape:
        n *= v
    return torch.linspace(lo, hi, n).view(*shape)


def test_recurrence(hla):
    """Open decays (a of e^-50 in the first half, of e^-0.01 s in the second), inputs through gates of -43 to 0."""
    B, n, C = 3, 1, 256
    g = gates(-43, 0, B, n, C)
    decay = torch.where(torch.arange(C) % 2 == 0, -50.0, -0.01)
    r = torch.full_like(g, 60.0)
    x = torch.ones_like(g)
    m = (-torch.expm1(2 * decay.double())).sqrt()
    want = torch.sigmoid(g.double()) * m
    assert off(hla.hla_glr_forward(on(x), on(r), on(g), on(decay)), want) <= 2 * ROOM  # (two roots besides)
    state = torch.zeros(B, C, device=DEV)
    assert off(hla.hla_glr_step(on(x[:, 0]), on(r[:, 0]), on(g[:, 0]), on(decay), state), want[:, 0]) <= 2 * ROOM
    marks = torch.zeros(B, 1, C, device=DEV)
    dx, _, dg, _ = hla.hla_glr_backward(on(x), on(r), on(g), on(decay), on(x), marks)
    assert off(dx, want) <= 2 * ROOM and off(dg, want * torch.sigmoid(-g.double())) <= 2 * ROOM
    # what is left of a state through small gates of the decay: 1 - a = 50 sigmoid(r), a sum of 1 - that in y
    r = gates(-12, 4, B, n, C)
    first = torch.ones(B, C)
    y = hla.hla_glr_forward(on(0 * x), on(r), on(g), torch.full((C,), -1.0, device=DEV), state_in=on(first))
    assert off(y, torch.exp(-torch.sigmoid(r.double()))) <= ROOM


@pytest.mark.parametrize("C", [64, 512, 8200])
def test_norms(hla, C):
    gate = gates(-80, 5, 3, C)
    zero, one = torch.zeros_like(gate), torch.ones_like(gate)
    s = torch.sigmoid(gate.double())
    for act, want in ((hla.HLA_SIGMOID, s), (hla.HLA_SILU, s * gate.double())):
        got = hla.hla_block_norm_forward(on(zero), on(one), on(gate), post_norm=False, pre_norm=False, act=act)[0]
        assert off(got, want) <= ROOM
    # the gradient by y is the gate's value, by a gate the slope: s (1 - s) below 0
    dx, dy, dgate = hla.hla_block_norm_backward(on(zero), on(one), on(gate), on(one), post_norm=False, pre_norm=False,
                                                act=hla.HLA_SIGMOID)[:3]
    below = gate < 0
    assert off(dy, s) <= ROOM and off(dgate[on(below)], (s * torch.sigmoid(-gate.double()))[below]) <= ROOM


@pytest.mark.parametrize("M", [1, 40, 300])
def test_feed_forward(hla, M):
    F = 300
    gate = gates(-80, 5, 1, F)
    w = torch.stack([gate.view(F, 1), torch.ones(F, 1)])
    x = torch.ones(M, 1)
    s = torch.sigmoid(gate.double()).expand(M, F)
    assert off(hla.hla_ffn_forward(on(x), on(w), act=hla.HLA_SIGMOID), s) <= ROOM
    assert off(hla.hla_ffn_forward(on(x), on(w), act=hla.HLA_SILU), s * gate.double()) <= ROOM
    _, dw = hla.hla_ffn_backward(on(x), on(w), torch.ones(M, F, device=DEV), act=hla.HLA_SIGMOID)
    # (a sum over tokens of equal values: each step off by half a unit of the sum, M 2^-24 at most)
    assert off(dw[1, :, 0], M * s[0]) <= ROOM + M * 2.0 ** -24
