"""The selective scan on the GPU where its tiles and segments depend on one another, against the 64-bit recurrence:
slow decays and large states over many tiles, decays so strong that sums of exponents lose their small terms, NaN and
infinities in tokens, and waits that run out.

b, c, x, skip and the states are positive here, so that a sum's value is the magnitude its rounding errors scale
with: a bound of a few 2^-8 resolves a carried part of one percent."""
import pytest
import torch

import layer_ref as R

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U16, U32 = 2.0 ** -8, 2.0 ** -24
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
TILE = 128


@pytest.fixture(scope="module")
def hla():
    from paper_2510_27258_gb300 import build
    build.build()
    from paper_2510_27258_gb300 import hla as binding
    return binding


def near(got, want, bound):
    excess = (got.double() - want).abs() - bound
    assert torch.isfinite(got).all()
    assert float(excess.max()) <= 0, (float(excess.max()), float((got - want).abs().max()))


def positive(g, *shape, T=torch.float32):
    return torch.rand(*shape, generator=g, device=DEV).add_(0.1).to(T)


def inputs(seed, B, n, H, P, G, N, T):
    """x, delta, a, b, c, skip, state: steps of softplus(delta - 6), about 2.5e-3, and a in -2 .. -0.5, so that a
    head forgets over hundreds of tokens."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    x, b, c = positive(g, B, n, H, P, T=T), positive(g, B, n, G, N, T=T), positive(g, B, n, G, N, T=T)
    delta = (torch.randn(B, n, H, generator=g, device=DEV) * 0.5).to(T)
    a = -0.5 - 1.5 * torch.rand(H, generator=g, device=DEV)
    return x, delta, a, b, c, positive(g, H), 4 * positive(g, B, H, N, P)


def reference(*args, **kw):
    with torch.device(DEV):
        return R.ssm(*args, **kw)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,n,H,P,G,N,lens,cuts", [
    (2, 890, 3, 64, 1, 128, [890, 700], (1, 7)),        # tiles of one CTA
    (2, 1100, 152, 64, 1, 64, [900, 1100], (1, 9)),
    (1, 3015, 76, 64, 2, 64, None, (4, 6)),             # segments of several tiles
    (1, 3015, 76, 64, 1, 128, None, (4, 6)),
    (1, 2048, 38, 128, 2, 32, None, (4, 4)),
    (1, 2048, 38, 128, 1, 128, None, (4, 4)),
    (2, 3000, 38, 64, 1, 128, [3000, 1037], (4, 6)),    # ... of which some count in part, or not at all
    (2, 3000, 19, 128, 1, 16, [130, 2999], (4, 6))])
def test_a_state_carried_over_tiles_and_segments(hla, dtype, B, n, H, P, G, N, lens, cuts):
    """Rounding of the state of bf16 tokens: w X as bf16 pairs (2^-16); exponents of up to 16 (what lies further back
    weighs nothing) whose steps and sums are good to 2^-21; and for each tile 32 accumulations of 2^-23 and the
    tile's decay."""
    T = TYPES[dtype]
    if T == torch.bfloat16:
        segments, tiles = cuts
        assert segments * tiles * TILE >= n > (segments - 1) * tiles * TILE
        assert hla.hla_ssm_forward_path(B, n, H, P, G, N) == (1, 1 if segments == 1 else 3)
        if segments > 1:  # the workspace holds a state for each
            assert hla.hla_ssm_workspace_bytes(B, n, H, P, G, N, T) // (4 * B * H * (N * P + 1)) == segments
    x, delta, a, b, c, skip, state = inputs(n + N, B, n, H, P, G, N, T)
    bias = torch.full((H,), -6.0, device=DEV)
    lengths = None if lens is None else torch.tensor(lens, dtype=torch.int32, device=DEV)
    y, h, ym, hm = reference(x, delta, a, b, c, skip, bias, True, lengths, state)
    st = state.clone()
    out = hla.hla_ssm_forward(x, delta, a, b, c, skip=skip, delta_bias=bias, lengths=lengths, state_in=st, state_out=st)
    if T == torch.bfloat16:
        rel = 2.0 ** -16 + 16 * 2.0 ** -21 + 64 * (n / TILE + 2) * U32
        near(out, y, U16 * y.abs() + (2 * U16 + rel) * ym)
    else:
        rel = (6 * n + 2 * N + 64) * U32
        near(out, y, rel * ym)
    near(st, h, rel * hm)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("P,N", [(64, 16), (16, 128), (128, 64)])
def test_weights_behind_a_very_strong_decay(hla, dtype, P, N):
    """Steps that wipe a state out leave the weights among the tokens after them as they are, in the same
    32-token block too, up to steps whose exponent is beyond fp32's range."""
    T, (B, n, H, G) = TYPES[dtype], (1, 300, 4, 2)
    x, delta, a, b, c, skip, state = inputs(P + N, B, n, H, P, G, N, T)
    a = a * 8
    a[-1] = -1e6  # (times 1e34: beyond fp32's range)
    delta = (delta.float().abs() * 0.05 + 0.01).to(T)
    for t, big in ((3, 3e4), (36, 1e6), (37, 2e4), (63, 3e5), (130, 1e34), (200, 1e30), (259, 3e4)):
        delta[:, t] = big
    x[:, 130:] *= 1e-3
    y, h, ym, hm = reference(x, delta, a, b, c, skip, softplus=False, state=state)
    st = state.clone()
    out = hla.hla_ssm_forward(x, delta, a, b, c, skip=skip, softplus=False, state_in=st, state_out=st)
    serial = (6 * n + 2 * N + 64) * U32
    if T == torch.bfloat16:
        near(out, y, U16 * y.abs() + (2 * U16 + serial) * ym)
        near(st, h, (2.0 ** -16 + serial) * hm)
    else:
        near(out, y, serial * ym)
        near(st, h, serial * hm)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("B,n,H,P,G,N", [(2, 520, 3, 64, 1, 128), (2, 520, 3, 32, 3, 64), (1, 520, 2, 128, 1, 16),
                                         (1, 520, 2, 128, 2, 128), (1, 2500, 38, 64, 1, 64)])
def test_no_token_reaches_an_earlier_one(hla, dtype, bad, B, n, H, P, G, N):
    """A token that is not finite leaves what comes before it, and the columns of a state that it does not
    enter, as they are."""
    T = TYPES[dtype]
    x, delta, a, b, c, skip, state = inputs(7 * P + N, B, n, H, P, G, N, T)
    bias = torch.full((H,), -6.0, device=DEV)
    y, _, ym, _ = reference(x, delta, a, b, c, skip, bias, True, None, state)
    rel = 2.0 ** -16 + 16 * 2.0 ** -21 + 64 * (n / TILE + 2) * U32
    bound = U16 * y.abs() + (2 * U16 + rel) * ym if T == torch.bfloat16 else (6 * n + 2 * N + 64) * U32 * ym

    def run(x, delta, b, c, state):
        return hla.hla_ssm_forward(x, delta, a, b, c, skip=skip, delta_bias=bias, state_in=state)

    def check(out, free):
        """What is finite by the formula (`free`) is right, all else is not finite."""
        assert torch.isfinite(out[free]).all() and not torch.isfinite(out[~free]).any()
        assert bool(((out.double() - y).abs() <= bound)[free].all())

    every = torch.ones(B, n, H, P, dtype=torch.bool, device=DEV)
    # single elements of x, several in a tile, in neighbouring tiles, one column twice
    places = [(0, 5, 0, 0), (0, 70, H - 1, P - 1), (B - 1, 127, 0, 1), (B - 1, 128, H - 1, 2), (0, 300, 1, P // 2),
              (0, 310, 1, P // 2), (0, 290, 1, P // 2 + 1), (0, n - 2, 0, 3)]
    x2, free = x.clone(), every.clone()
    for s, t, h, p in places:
        x2[s, t, h, p] = bad
        free[s, t:, h, p] = False
    check(run(x2, delta, b, c, state), free)
    # c: its own token alone
    c2, free = c.clone(), every.clone()
    c2[0, 77, G - 1, 3] = bad
    free[0, 77, (G - 1) * (H // G):] = False
    check(run(x, delta, b, c2, state), free)
    # b: every later token of its group's heads
    b2, free = b.clone(), every.clone()
    b2[0, 200, 0, 5] = bad
    free[0, 200:, :H // G] = False
    check(run(x, delta, b2, c, state), free)
    # a step (minus infinity is one of zero)
    if bad != float("-inf"):
        d2, free = delta.clone(), every.clone()
        d2[B - 1, 259, H - 1] = bad
        free[B - 1, 259:, H - 1] = False
        check(run(x, d2, b, c, state), free)
    # a state
    s2, free = state.clone(), every.clone()
    s2[0, 0, 2, 1] = bad
    free[0, :, 0, 1] = False
    check(run(x, delta, b, c, s2), free)


@pytest.mark.parametrize("B,n,H,P,G,N,launches", [(2, 890, 3, 64, 1, 128, 1), (2, 890, 3, 64, 1, 64, 1),
                                                  (1, 3015, 38, 128, 1, 32, 3)])
def test_a_wait_that_runs_out_is_reported(hla, monkeypatch, B, n, H, P, G, N, launches):
    """Copies of x that bring half of the bytes that are waited for (set up on the host): the waits run out (2 s each),
    the kernels finish, hla_poll_error reports HLA_ERR_TIMEOUT, and the workspace works again."""
    T = torch.bfloat16
    assert hla.hla_ssm_forward_path(B, n, H, P, G, N) == (1, launches)
    x, delta, a, b, c, skip, state = inputs(n + N, B, n, H, P, G, N, T)
    bias = torch.full((H,), -6.0, device=DEV)
    ws = hla.alloc_workspace(hla.hla_ssm_workspace_bytes(B, n, H, P, G, N, T), DEV)
    so = torch.empty_like(state)
    run = lambda: hla.hla_ssm_forward(x, delta, a, b, c, skip=skip, delta_bias=bias, state_in=state,  # noqa: E731
                                      state_out=so, workspace=ws)
    want, state_want = run(), so.clone()
    assert hla.hla_poll_error(ws) == hla.HLA_OK
    monkeypatch.setenv("HLA_TEST_SHORT_COPY", "1")
    run()
    assert hla.hla_poll_error(ws) == hla.HLA_ERR_TIMEOUT
    monkeypatch.delenv("HLA_TEST_SHORT_COPY")
    assert torch.equal(run(), want) and torch.equal(so, state_want)
    assert hla.hla_poll_error(ws) == hla.HLA_OK
