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


MANY = (1 << 24) + 16  # heads: 128 components (or states) of each pass 2^31 elements
ENDS = [0, 1, (1 << 24) - 1, 1 << 24, (1 << 24) + 1, MANY - 1]


def expected(x, delta, b, c, skip, first=0.0, a=-1.0):
    """One token for each head in 64 bits: x [heads, P], delta [heads], b, c [heads, N], first the state's value."""
    x, d, b, c = x.double(), delta.double()[:, None], b.double(), c.double()
    return (d * (b * c).sum(1, keepdim=True) + skip) * x + first * torch.exp(a * d) * c.sum(1, keepdim=True)


@pytest.mark.parametrize("P,G,N", [(128, 1, 16), (16, MANY, 128)])
def test_scan_of_rows_of_more_than_2_31_elements(hla, P, G, N):
    g = torch.Generator(device=DEV).manual_seed(2)
    rand = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
    x, b, c, delta = rand(1, 1, MANY, P), rand(1, 1, G, N), rand(1, 1, G, N), rand(1, 1, MANY).abs_()
    a, skip = torch.full((MANY,), -1.0, device=DEV), torch.full((MANY,), 0.5, device=DEV)
    y = hla.hla_ssm_forward(x, delta, a, b, c, skip=skip, softplus=False)
    group = [h * G // MANY for h in ENDS]
    want = expected(x[0, 0, ENDS], delta[0, 0, ENDS], b[0, 0, group], c[0, 0, group], 0.5)
    assert float((y[0, 0, ENDS].double() - want).abs().max()) <= (2 * N + 8) * 2.0 ** -24 * N * 100
    assert torch.isfinite(y).all()


def test_scan_step_of_rows_of_more_than_2_31_elements(hla):
    P, N = 128, 16
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 170e9:
        pytest.skip("less than 170 GB of memory are free")
    state = torch.full((1, MANY, N, P), 2.0, device=DEV)  # 137 GB
    g = torch.Generator(device=DEV).manual_seed(3)
    rand = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
    x, b, c, delta = rand(1, MANY, P), rand(1, 1, N), rand(1, 1, N), rand(1, MANY).abs_()
    a, skip = torch.full((MANY,), -1.0, device=DEV), torch.full((MANY,), 0.5, device=DEV)
    y = hla.hla_ssm_step(x, delta, a, b, c, state, skip=skip, softplus=False)
    group = [0] * len(ENDS)
    want = expected(x[0, ENDS], delta[0, ENDS], b[0, group], c[0, group], 0.5, first=2.0)
    assert float((y[0, ENDS].double() - want).abs().max()) <= (2 * N + 8) * 2.0 ** -24 * N * 100
    wanted = 2.0 * torch.exp(-delta[0, ENDS].double())[:, None, None] + (
        (delta[0, ENDS].double()[:, None] * b[0, 0].double())[..., None] * x[0, ENDS].double()[:, None])
    assert float((state[0, ENDS].double() - wanted).abs().max()) <= 8 * 2.0 ** -24 * 100
    del state
    torch.cuda.empty_cache()
