"""Rows whose elements, or whose weights', are more than 32-bit indices reach."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def hla():
    from paper_2510_27258_gb300 import build
    build.build()
    from paper_2510_27258_gb300 import hla as binding
    return binding


@pytest.mark.parametrize("C", [430_000_000, 430_000_003])
def test_conv_weight_gradients_of_many_channels(hla, C):
    """(width + 1) C passes 2^31: two tokens, whose products are exact in fp32, so the sums have one rounding."""
    T, W = torch.bfloat16, 4
    g = torch.Generator(device=DEV).manual_seed(1)
    x, dout = (torch.randn(1, 2, C, generator=g, device=DEV, dtype=T) for _ in range(2))
    w = torch.zeros(C, W, dtype=T, device=DEV)
    w[:, W - 1] = 0.5
    dx, dw, db = hla.hla_conv_backward(x, w, dout, torch.zeros(C, dtype=T, device=DEV), silu=False)
    assert torch.equal(dx, dout * 0.5)
    x, dout = x[0], dout[0]
    assert not dw[:, :W - 2].any()
    assert torch.equal(dw[:, W - 2], dout[1].float() * x[0].float())
    assert torch.equal(dw[:, W - 1], dout[0].float() * x[0].float() + dout[1].float() * x[1].float())
    assert torch.equal(db, dout[0].float() + dout[1].float())
