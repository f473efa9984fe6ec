"""What shapes the binding takes for contiguous tensors, without a GPU (stand-ins of test_binding_streams_cpu.py)."""
import pytest
import torch

from test_binding_streams_cpu import Tensor, world  # noqa: F401


def T(*shape, dtype=torch.float32):
    return Tensor(torch.zeros(*shape, dtype=dtype))


B, n, H, P, G, N, C, W, d = 2, 8, 4, 32, 2, 16, 24, 4, 16


def conv(E, **kw):
    return E.hla_conv_forward(T(B, n, C), T(C, W), **kw)


def conv_step(E, state):
    return E.hla_conv_step(T(B, C), T(C, W), state)


def ssm(E, **kw):
    return E.hla_ssm_forward(T(B, n, H, P), T(B, n, H), kw.pop("a", T(H)), T(B, n, G, N), T(B, n, G, N), **kw)


def ssm_step(E, state):
    return E.hla_ssm_step(T(B, H, P), T(B, H), T(H), T(B, G, N), T(B, G, N), state)


def qk(E, sin=None, **kw):
    return E.hla_qk_norm_forward(T(B, n, H, d), T(B, n, G, d), cos=T(20, 4), sin=T(20, 4) if sin is None else sin, **kw)


def qk_back(E, dq_out):
    return E.hla_qk_norm_backward(T(B, n, H, d), T(B, n, G, d), None, None, None, None, dq_out, T(B, H, n, d))


i32 = torch.int32
# of as many elements as it should have, in another order
WRONG = [lambda E: ssm(E, state_in=T(B, H, P, N)), lambda E: ssm(E, state_out=T(B, H, P, N)),
         lambda E: ssm(E, state_in=T(H, B, N, P)), lambda E: ssm_step(E, T(B, H, P, N)), lambda E: ssm_step(E, T(N, P, B, H)),
         lambda E: conv(E, state_in=T(B, C, W - 1)), lambda E: conv(E, state_out=T(W - 1, B, C)),
         lambda E: conv_step(E, T(B, C, W - 1)), lambda E: qk(E, positions=T(n, B, dtype=i32)), lambda E: qk(E, sin=T(4, 20)),
         lambda E: qk(E, q_out=T(B, n, H, d)), lambda E: qk(E, k_out=T(B, H, d, n)), lambda E: qk_back(E, T(B, n, H, d))]
# ... and in the same one
RIGHT = [lambda E: ssm(E, state_in=T(B, H, N, P), state_out=T(B * H * N * P)), lambda E: ssm(E, state_in=T(B * H, N, P)),
         lambda E: ssm(E, state_in=T(B, H, N * P), a=T(1, H)), lambda E: ssm_step(E, T(B, G, H // G, N, P)),
         lambda E: conv(E, state_in=T(B, 1, W - 1, C), bias=T(C, 1)), lambda E: conv_step(E, T(B * (W - 1), C)),
         lambda E: qk(E, positions=T(B * n, dtype=i32)), lambda E: qk(E, sin=T(1, 20, 4), q_out=T(B * H, n, d)),
         lambda E: qk(E, k_out=T(B, G, H // G, n, d)), lambda E: qk_back(E, T(B, H * n, d))]


@pytest.mark.parametrize("call", range(len(WRONG)))
def test_another_order_is_refused(world, call):  # noqa: F811
    from paper_2510_27258_gb300 import hla as E
    with pytest.raises(ValueError):
        WRONG[call](E)
    assert not world.launched


@pytest.mark.parametrize("call", range(len(RIGHT)))
def test_the_same_order_in_another_shape(world, call):  # noqa: F811
    from paper_2510_27258_gb300 import hla as E
    RIGHT[call](E)
    assert len(world.launched) == 1


@pytest.mark.parametrize("got,want,same", [
    ((2, 3, 4), (2, 3, 4), True), ((24,), (2, 3, 4), True), ((6, 4), (2, 3, 4), True), ((2, 12), (2, 3, 4), True),
    ((2, 4, 3), (2, 3, 4), False), ((3, 2, 4), (2, 3, 4), False), ((8, 3), (2, 3, 4), False), ((2, 3, 2, 2), (2, 3, 4), True),
    ((0, 7), (0, 3), True), ((1, 6), (6, 1), True), ((5,), (6,), False), ((), (1,), True), ((0,), (1,), False)])
def test_same_order(got, want, same):
    from paper_2510_27258_gb300 import hla as E
    assert E._same_order(got, want) is same
