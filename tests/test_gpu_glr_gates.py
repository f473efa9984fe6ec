"""The gated recurrence where both of a token's gates are shut: such a token leaves the state as it is, exactly, and its
gradients are zero.  e^-v leaves the range of fp32 at v = 88.7, its square at 44.4, and the sigmoid of -87.4 and below
is 0."""
import pytest
import torch

import block_ref as R
from test_gpu_block import DEV, TYPES, gen, glr_case, near, on, randn

pytestmark = pytest.mark.gpu
INF = float("inf")
SHUT = [(-1e4, -1e4), (-100.0, -50.0), (-88.0, -45.0), (-87.5, -44.5), (-INF, -INF), (-INF, -1e4), (-100.0, -INF),
        ("lowest", "lowest"), (-60.0, -1e4), (-1e4, -44.0)]


@pytest.fixture(scope="module")
def hla():
    from paper_2510_27258_gb300 import build
    build.build()
    from paper_2510_27258_gb300 import hla as binding
    return binding


def values(pair, T):
    return [torch.finfo(T).min if v == "lowest" else v for v in pair]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pair", SHUT)
@pytest.mark.parametrize("decay", [-0.01, -50.0])
@pytest.mark.parametrize("B,n,C", [(2, 70, 64), (1, 2000, 24), (40, 40, 520)])
def test_tokens_with_both_gates_shut_keep_the_state(hla, dtype, pair, decay, B, n, C):
    """(blocks of a sequence alone and in clusters)  With r = -60 the decay is e^(-50 e^-60), 1 in fp32."""
    T = TYPES[dtype]
    g = gen(n)
    gate_r, gate_g = values(pair, T)
    x, first = on(randn(g, B, n, C, T=T, scale=3.0)), on(randn(g, B, C))
    r, gt, dec = torch.full_like(x, gate_r), torch.full_like(x, gate_g), torch.full((C,), decay, device=DEV)
    state, marks = first.clone(), torch.full((B, hla.hla_glr_marks(n), C), float("nan"), device=DEV)
    y = hla.hla_glr_forward(x, r, gt, dec, state_in=state, state_out=state, marks=marks)
    assert torch.equal(state, first)
    assert torch.equal(y, first.to(T)[:, None].expand_as(y)) and torch.equal(marks, first[:, None].expand_as(marks))
    out = hla.hla_glr_step(x[:, 0], r[:, 0], gt[:, 0], dec, state)
    assert torch.equal(state, first) and torch.equal(out, first.to(T))
    dy, dl = on(randn(g, B, n, C, T=T)), on(randn(g, B, C))
    back = torch.empty_like(dl)
    dx, dr, dg, ddecay = hla.hla_glr_backward(x, r, gt, dec, dy, marks, dstate_out=dl, dstate_in=back)
    if gate_r < -80:
        assert not dx.any() and not dr.any() and not dg.any() and not ddecay.any()
    else:  # s = e^-60: dr and ddecay are sums of up to n values of 50 s |G h| <= 5e-25 n^2
        assert not dx.any() and not dg.any() and float(dr.float().abs().max()) < 1e-16 and float(ddecay.abs().max()) < 1e-13
    # all of dy comes to the state: sums of n values, each step off by 2^-24 of the magnitudes
    want = dl.double() + dy.double().sum(1)
    room = (n + 2) * 2.0 ** -24 * (dl.double().abs() + dy.double().abs().sum(1))
    assert bool(((back.double() - want).abs() <= room).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pair", [(-1e4, -1e4), (-100.0, -50.0), ("lowest", "lowest")])
@pytest.mark.parametrize("B,n,C", [(3, 130, 203), (1, 1500, 66), (40, 70, 264)])
def test_shut_tokens_among_others(hla, dtype, pair, B, n, C):
    """Half of the tokens, and whole runs of them, masked by both gates: the others are what the definition gives."""
    T = TYPES[dtype]
    g, v, _ = glr_case(C, B, n, C, T, False)
    shut = torch.rand(B, n, 1, generator=g) < 0.5
    shut[:, 20:37] = True
    for k, to in zip(("r", "g"), values(pair, T)):
        v[k] = torch.where(shut, torch.tensor(to, dtype=T), v[k])
    want, last, bound, last_bound = R.glr(v["x"], v["r"], v["g"], v["decay"], v["state"])
    x, r, gt, dec = (on(v[k]) for k in ("x", "r", "g", "decay"))
    state, marks = on(v["state"]), torch.empty(B, hla.hla_glr_marks(n), C, device=DEV)
    near("y", hla.hla_glr_forward(x, r, gt, dec, state_in=state, state_out=state, marks=marks), want, bound)
    near("state", state, last, last_bound)
    state = on(v["state"])
    for t in range(24):
        near("token", hla.hla_glr_step(x[:, t], r[:, t], gt[:, t], dec, state), want[:, t], bound[:, t])
    dy = randn(g, B, n, C, T=T)
    grads = hla.hla_glr_backward(x, r, gt, dec, on(dy), marks)
    assert all(torch.isfinite(t).all() for t in grads)
    there = on(shut).expand_as(x)
    assert not any(t[there].any() for t in grads[:3])
