"""The 64-bit references' gradients against central differences of their forwards, and hand values."""
import math

import pytest
import torch

import layer_ref as R

D = torch.float64


def difference(f, tensors, seed):
    """(directional derivative by central differences, directions) of the scalar f(*tensors)."""
    g = torch.Generator().manual_seed(seed)
    vs = [torch.randn(t.shape, generator=g, dtype=D) for t in tensors]
    e = 1e-5
    up, down = (f(*[t + s * e * v for t, v in zip(tensors, vs)]) for s in (1, -1))
    return (up - down) / (2 * e), vs


@pytest.mark.parametrize("W,silu,lengths", [(2, True, None), (3, False, [4, 0, 9]), (4, True, [9, 1, 5])])
def test_conv_gradient_is_the_difference(W, silu, lengths):
    g = torch.Generator().manual_seed(W)
    x, dout = (torch.randn(3, 9, 5, generator=g, dtype=D) for _ in range(2))
    w, bias = torch.randn(5, W, generator=g, dtype=D), torch.randn(5, generator=g, dtype=D)
    want, vs = difference(lambda *t: float((R.conv(t[0], t[1], t[2], silu, lengths)[0] * dout).sum()), [x, w, bias], 1)
    got = sum(float((a * v).sum()) for a, v in zip(R.conv_grad(x, w, bias, dout, silu, lengths), vs))
    # truncation about 1e-10 of the third derivative, rounding 1e-16 / 1e-5 of the sum
    assert abs(got - want) < 1e-8 * (1 + abs(want))


@pytest.mark.parametrize("per,rot,interleaved", [(1, 8, False), (2, 16, True), (4, 0, False)])
def test_qk_gradient_is_the_difference(per, rot, interleaved):
    g = torch.Generator().manual_seed(rot)
    x, w = torch.randn(2, 5, 3, 16, generator=g, dtype=D), torch.randn(16, generator=g, dtype=D)
    dout = torch.randn(2, 3 * per, 5, 16, generator=g, dtype=D)
    angle = torch.randn(7, rot // 2, generator=g, dtype=D)
    at = torch.randint(0, 7, (2, 5), generator=g)
    want, vs = difference(lambda a, b: float((R.qk_norm(a, b, angle.cos(), angle.sin(), at, 3 * per, 1e-6,
                                                       interleaved)[0] * dout).sum()), [x, w], 2)
    dx, dw, _, _ = R.qk_norm_grad(x, w, angle.cos(), angle.sin(), at, dout, 1e-6, interleaved)
    assert abs(float((dx * vs[0]).sum() + (dw * vs[1]).sum()) - want) < 1e-8 * (1 + abs(want))


def test_scan_by_hand():
    """One head, one state, one column: h = e^{a d} h + d b x."""
    one = lambda *v: torch.tensor(v, dtype=D)  # noqa: E731
    y, h, _, _ = R.ssm(one(1., 2.).view(1, 2, 1, 1), one(0.5, 0.25).view(1, 2, 1), one(-2.), one(3., 1.).view(1, 2, 1, 1),
                       one(1., 4.).view(1, 2, 1, 1), skip=one(10.), softplus=False)
    h1 = 0.5 * 3 * 1
    h2 = math.exp(-0.5) * h1 + 0.25 * 1 * 2
    assert torch.allclose(y.flatten(), one(h1 + 10, 4 * h2 + 20)) and abs(float(h) - h2) < 1e-15


def test_conv_by_hand():
    x = torch.tensor([1., 2., 4.]).view(1, 3, 1)
    out, last, _ = R.conv(x, torch.tensor([[0.5, 3.]]), torch.tensor([1.]), silu=False,
                          state=torch.tensor([8.]).view(1, 1, 1))
    assert out.flatten().tolist() == [1 + 4 + 3, 1 + 0.5 + 6, 1 + 1 + 12] and last.flatten().tolist() == [4.]
