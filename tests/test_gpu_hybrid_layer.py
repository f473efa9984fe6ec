"""The operators together, as examples/hybrid_layer.py runs them."""
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
    spec = importlib.util.spec_from_file_location("hybrid_layer", os.path.join(ROOT, "examples", "hybrid_layer.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("dtype,tol", [(torch.float32, 1e-4), (torch.bfloat16, 2e-2)])
@pytest.mark.parametrize("kw", [dict(), dict(H=4, Hk=1, d=32, S=6, P=32, G=2, N=16), dict(H=2, Hk=2, d=128, S=3, P=128, N=64)])
def test_prompt_then_tokens_equals_the_whole(E, dtype, tol, kw):
    """bf16: the layer's intermediate roundings (2^-8 each) differ between the ways; 2e-2 is the bar of the
    HLA forward itself.  fp32: different orders of sums over a few hundred tokens."""
    layer = E.Layer(96, dtype=dtype, **kw)
    g = torch.Generator().manual_seed(3)
    tokens = torch.randn(3, 170, 96, generator=g).to("cuda", dtype)
    want = E.prompt(layer, tokens, layer.new_state(3))
    state = layer.new_state(3)
    got = [E.prompt(layer, tokens[:, :97], state), E.prompt(layer, tokens[:, 97:164], state)]
    got += [E.token(layer, tokens[:, t], state)[:, None] for t in range(164, 170)]
    diff = (torch.cat(got, 1).double() - want.double()).norm(dim=-1)
    assert float((diff / want.double().norm(dim=-1).mean()).max()) < tol


@pytest.mark.parametrize("name", ["tokens", "w_in", "conv_w", "conv_b", "wq", "wk"])
def test_gradients_are_differences(E, name):
    """The step's gradient along a direction against central differences of the fp32 forward (its own
    rounding, 1e-7 of the terms over a difference of 1e-2, and the third derivative's 1e-4: 1e-2 together)."""
    layer = E.Layer(48, H=2, Hk=1, d=16, dtype=torch.float32)
    g = torch.Generator().manual_seed(5)
    tokens = torch.randn(2, 21, 48, generator=g).cuda()
    dout = torch.randn(2, 2, 21, 16, generator=g).cuda()
    grads = E.gradients(layer, tokens, dout)
    used = sum(layer.parts[:3])
    cut = {"w_in": (slice(None), slice(0, used)), "conv_w": slice(0, used), "conv_b": slice(0, used)}
    target = tokens if name == "tokens" else getattr(layer, name)
    part = target[cut[name]] if name in cut else target
    assert grads[name].shape == part.shape
    v = torch.randn(part.shape, generator=g).cuda()
    e = 1e-2 * float(part.norm() / v.norm())
    v = v * e

    def loss():
        return float((E.hla_half(layer, tokens)[0].double() * dout.double()).sum())

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
