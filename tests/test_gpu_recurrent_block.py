"""The block's operators together, as examples/recurrent_block.py runs them."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def E():
    from paper_2510_27258_gb300 import build
    build.build()
    spec = importlib.util.spec_from_file_location("recurrent_block", os.path.join(ROOT, "examples", "recurrent_block.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("dtype,tol", [(torch.float32, 1e-4), (torch.bfloat16, 2e-2)])
@pytest.mark.parametrize("sizes", [(96, 128, 200), (64, 203, 77)])
def test_prompt_then_tokens_equals_the_whole(E, dtype, tol, sizes):
    """bf16: a dozen roundings of 2^-8 along the way fall differently, of which a row's norm keeps about the root of
    their number; fp32: different orders of sums of some hundred terms."""
    block = E.Block(*sizes, dtype=dtype)
    g = torch.Generator().manual_seed(3)
    x = torch.randn(3, 170, sizes[0], generator=g).to("cuda", dtype)
    want = E.prompt(block, x, block.new_state(3))
    state = block.new_state(3)
    got = [E.prompt(block, x[:, :97].contiguous(), state), E.prompt(block, x[:, 97:164].contiguous(), state)]
    got += [E.token(block, x[:, t], state)[:, None] for t in range(164, 170)]
    diff = (torch.cat(got, 1).double() - want.double()).norm(dim=-1)
    assert float((diff / want.double().norm(dim=-1).mean()).max()) < tol


@pytest.mark.parametrize("name", ["tokens", "w_in", "conv_w", "conv_b", "decay", "w_out", "w_ff", "w_down", "w_first",
                                  "w_post", "w_pre", "w_last", "scale", "scale_last"])
def test_gradients_are_differences(E, name):
    """The step's gradient along a direction against central differences of the fp32 forward (its own rounding,
    1e-6 of the terms over a difference of 1e-2, and the third derivative's 1e-4: 1e-2 together), dropout on.

    decay's elements go from -0.84 to -0.008 and enter as sqrt(1 - a^2), about sqrt(-2 decay s): a central difference of a
    square root is off by (step / value)^2 / 8 of it (its third derivative is 3/4 / value^2 of the first, over 6).  A
    hundredth of the norm is a step of 0.004 on average, half of the smallest value and more: 3 % and more there.  A
    thousandth leaves 3e-4, and 1e-3 of rounding."""
    block = E.Block(40, 48, 36, dtype=torch.float32, dropout=0.25)
    g = torch.Generator().manual_seed(5)
    x = torch.randn(2, 37, 40, generator=g).cuda()
    dout = torch.randn(2, 37, 40, generator=g).cuda()
    grads = E.gradients(block, x, dout, seed=9)
    part = x if name == "tokens" else getattr(block, name)
    assert grads[name].shape == part.shape
    v = torch.randn(part.shape, generator=g).cuda()
    v = v * ((1e-3 if name == "decay" else 1e-2) * float(part.norm() / v.norm()))

    def loss():
        return float((E.prompt(block, x, block.new_state(2), seed=9).double() * dout.double()).sum())

    keep = part.clone()
    part.copy_(keep + v)
    up = loss()
    part.copy_(keep - v)
    down = loss()
    part.copy_(keep)
    want = (up - down) / 2
    got = float((grads[name].double() * v.double()).sum())
    scale = float(grads[name].double().norm() * v.double().norm()) / v.numel() ** 0.5
    assert abs(got - want) < 1e-2 * max(abs(want), scale)
