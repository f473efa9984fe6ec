"""The operators around the mixers on the GPU against their definitions in 64 bits.

Every bound is elementwise and follows from the arithmetic: u16 = 2^-8 for the one rounding of a bf16
output, 2^-24 for each fp32 operation, times the magnitude of what was summed.  The device
exponential (2 + 1.2 |x| units in the last place) and division give the sigmoid 2^-19 over the values
used here."""
import pytest
import torch

import layer_ref as R

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U16, U32 = 2.0 ** -8, 2.0 ** -24
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def hla():
    from paper_2510_27258_gb300 import build
    build.build()
    from paper_2510_27258_gb300 import hla as binding
    return binding


def unit(T):
    return U16 if T == torch.bfloat16 else 0.0


def near(got, want, bound):
    """Every element within its bound (and finite)."""
    got = got.double().cpu()
    assert got.shape == want.shape
    assert torch.isfinite(got).all()
    excess = (got - want).abs() - bound - 1e-30
    assert float(excess.max()) <= 0 if excess.numel() else True, (float(excess.max()), float((got - want).abs().max()))


def sliced(t, extra=8, at=0):
    """`t` on the GPU as a slice of rows that are wider by `extra` elements (NaN), from element `at` on."""
    flat = t.flatten(2) if t.dim() > 2 else t
    wide = torch.full(flat.shape[:-1] + (flat.shape[-1] + extra,), float("nan"), dtype=t.dtype, device=DEV)
    wide[..., at:at + flat.shape[-1]] = flat.to(DEV)
    return wide[..., at:at + flat.shape[-1]].unflatten(-1, t.shape[2:]) if t.dim() > 2 else \
        wide[..., at:at + flat.shape[-1]]


def gen(seed):
    return torch.Generator().manual_seed(seed)


def randn(g, *shape, T=torch.float32, scale=1.0):
    return (torch.randn(*shape, generator=g) * scale).to(T)


def ragged(g, B, n):
    lens = [n, 0, 1] + [int(v) for v in torch.randint(0, n + 1, (max(B - 3, 0),), generator=g)]
    return torch.tensor(lens[:B], dtype=torch.int32)


def poison(t, lens):
    """NaN and infinities at and after each length: nothing there may be read into a result."""
    for i, m in enumerate(lens.tolist()):
        t[i, m:] = float("nan")
        t[i, m + 1:m + 2] = float("inf")
    return t


# ---------------------------------------------------------------------------------- convolution

def conv_case(seed, B, n, C, W, T, with_lengths):
    g = gen(seed)
    x, w, bias = randn(g, B, n, C, T=T), randn(g, C, W, T=T, scale=0.5), randn(g, C, T=T)
    state = randn(g, B, W - 1, C, T=T)
    lens = ragged(g, B, n) if with_lengths else None
    return g, x, w, bias, state, lens


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,n,C,W,silu,lens,extra,at", [
    (1, 1, 8, 4, True, False, 8, 0), (3, 2, 24, 4, True, True, 8, 0), (4, 37, 264, 3, False, True, 8, 8),
    (2, 130, 203, 4, True, False, 5, 3), (5, 64, 257, 2, True, True, 0, 0), (1, 1000, 64, 4, True, False, 8, 0),
    (2, 300, 520, 4, True, True, 1, 1), (1, 5, 1, 3, True, False, 3, 2)])
def test_conv_forward(hla, dtype, B, n, C, W, silu, lens, extra, at):
    T = TYPES[dtype]
    _, x, w, bias, state, lengths = conv_case(n + C, B, n, C, W, T, lens)
    want, last, mag = R.conv(x, w, bias, silu, lengths, state)
    if lengths is not None:
        poison(x, lengths)
    on = lambda t: None if t is None else t.to(DEV)  # noqa: E731
    st = on(state)
    out = hla.hla_conv_forward(sliced(x, extra, at), on(w), on(bias), silu=silu, lengths=on(lengths), state_in=st,
                               state_out=st)  # the state in place
    near(out, want, unit(T) * want.abs() + 2.0 ** -19 * (1 + mag))
    assert torch.equal(st.cpu().double(), last)  # copied, not computed
    # no bias, no state, a strided output
    want, last, mag = R.conv(torch.where(torch.isfinite(x), x, torch.zeros((), dtype=T)), w, None, silu, lengths)
    wide = torch.zeros(B, n, C + 7, dtype=T, device=DEV)
    so = torch.full_like(st, float("nan"))
    hla.hla_conv_forward(on(x), on(w), out=wide[..., 3:3 + C], silu=silu, lengths=on(lengths), state_out=so)
    near(wide[..., 3:3 + C], want, unit(T) * want.abs() + 2.0 ** -19 * (1 + mag))
    assert torch.equal(so.cpu().double(), last)
    assert not wide[..., :3].any() and not wide[..., 3 + C:].any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,C,W,silu,extra,at", [(1, 8, 4, True, 8, 0), (7, 203, 3, True, 3, 1), (64, 264, 2, False, 8, 0),
                                                 (33, 1, 4, True, 0, 0)])
def test_conv_step_continues_the_prompt(hla, dtype, B, C, W, silu, extra, at):
    """A prompt and then single tokens equal the whole sequence at once."""
    T = TYPES[dtype]
    _, x, w, bias, _, _ = conv_case(B + C, B, 12, C, W, T, False)
    want, last, mag = R.conv(x, w, bias, silu)
    st = torch.empty(B, W - 1, C, dtype=T, device=DEV)
    hla.hla_conv_forward(x[:, :7].contiguous().to(DEV), w.to(DEV), bias.to(DEV), silu=silu, state_out=st)
    for t in range(7, 12):
        tok = sliced(x[:, t], extra, at)
        out = hla.hla_conv_step(tok, w.to(DEV), st, bias.to(DEV), tok if t % 2 else None, silu=silu)
        near(out, want[:, t], unit(T) * want[:, t].abs() + 2.0 ** -19 * (1 + mag[:, t]))
    assert torch.equal(st.cpu().double(), last)


def test_conv_empty_prompt_keeps_the_state(hla):
    st = torch.randn(2, 3, 16, device=DEV)
    keep = st.clone()
    w = torch.randn(16, 4, device=DEV)
    hla.hla_conv_forward(torch.empty(2, 0, 16, device=DEV), w, state_in=st, state_out=st)
    assert torch.equal(st, keep)
    hla.hla_conv_forward(torch.empty(2, 0, 16, device=DEV), w, state_out=st)
    assert not st.any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,n,C,W,silu,lens,extra,at", [
    (1, 1, 8, 4, True, False, 8, 0), (4, 37, 264, 3, False, True, 8, 8), (2, 130, 203, 4, True, False, 5, 3),
    (5, 64, 132, 2, True, True, 0, 0), (1, 2100, 64, 4, True, False, 8, 0), (3, 3, 12, 4, True, True, 4, 4)])
def test_conv_backward(hla, dtype, B, n, C, W, silu, lens, extra, at):
    T = TYPES[dtype]
    g, x, w, bias, _, lengths = conv_case(n * C, B, n, C, W, T, lens)
    dout = randn(g, B, n, C, T=T)
    dx, dw, db = R.conv_grad(x, w, bias, dout, silu, lengths)
    # g carries a sigmoid's error times |dout| (1 + |pre|); dx sums W of them, dw up to B n
    mag = R.conv(x, w, bias, silu, lengths)[2]
    gm = dout.double().abs() * (1 + mag) ** 2
    if lengths is not None:
        gm = torch.where(torch.arange(n)[None, :, None] < lengths.view(B, 1, 1), gm, torch.zeros((), dtype=R.D))
    dxm, dwm, dbm = R.conv_grad(x.double().abs(), w.double().abs(), None, gm, False, lengths)
    if lengths is not None:
        poison(x, lengths), poison(dout, lengths)
    run = lambda: hla.hla_conv_backward(sliced(x, extra, at), w.to(DEV), sliced(dout, extra, at), bias.to(DEV),  # noqa: E731
                                        silu=silu, lengths=None if lengths is None else lengths.to(DEV))
    got = run()
    near(got[0], dx, unit(T) * dx.abs() + 2.0 ** -18 * dxm)
    terms = 32 + 16 + B * n / 32 / 8 / 8 + 8  # a strip, the block, the partial rows
    near(got[1], dw, (2.0 ** -18 + terms * U32) * dwm)
    near(got[2], db, (2.0 ** -18 + terms * U32) * dbm)
    for a, b in zip(got, run()):
        assert torch.equal(a, b)  # a fixed order of sums


# ---------------------------------------------------------------------------------- selective scan

def ssm_case(seed, B, n, H, P, G, N, T, with_lengths, strong=False):
    g = gen(seed)
    x, b, c = randn(g, B, n, H, P, T=T), randn(g, B, n, G, N, T=T), randn(g, B, n, G, N, T=T)
    delta = randn(g, B, n, H, T=T)
    a = -(torch.rand(H, generator=g) * 15 + 1)
    if strong:
        a = a * 20
    bias = randn(g, H, scale=0.5) + (0.0 if strong else -3.0)
    skip = randn(g, H)
    state = randn(g, B, H, N, P)
    return x, delta, a, b, c, skip, bias, state, ragged(g, B, n) if with_lengths else None


def ssm_bounds(T, n, N, y, ym, hm, step=False):
    """fp32 tokens (and the step): the serial recurrence in fp32, a few roundings a token and N
    products a sum.  bf16 prompts: the weights C B^T and the carried state are rounded to bf16 once for
    the outputs (2 u16 of the magnitude); the state itself takes bf16 pairs (2^-16)."""
    serial = (6.0 * n + 2 * N + 64) * U32
    if T == torch.float32 or step:
        return unit(T) * y.abs() + serial * ym, serial * hm
    return U16 * y.abs() + (2 * U16 + serial) * ym, (2.0 ** -16 + serial) * hm


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,n,H,P,G,N,lens,extra,at,strong", [
    (1, 1, 1, 16, 1, 16, False, 8, 0, False), (3, 5, 4, 32, 2, 32, True, 8, 8, False),
    (2, 127, 2, 64, 1, 128, False, 0, 0, False), (2, 129, 4, 64, 2, 64, False, 8, 0, True),
    (4, 200, 3, 64, 3, 128, True, 8, 0, False), (1, 513, 2, 128, 1, 64, False, 8, 0, False),
    (3, 300, 2, 128, 2, 128, True, 3, 1, False), (1, 1500, 1, 64, 1, 128, False, 8, 0, False),
    (3, 700, 2, 32, 1, 16, True, 8, 0, False), (2, 640, 2, 16, 1, 128, True, 8, 0, True)])
def test_ssm_forward(hla, dtype, B, n, H, P, G, N, lens, extra, at, strong):
    T = TYPES[dtype]
    x, delta, a, b, c, skip, bias, state, lengths = ssm_case(n + N, B, n, H, P, G, N, T, lens, strong)
    y, h, ym, hm = R.ssm(x, delta, a, b, c, skip, bias, True, lengths, state)
    if lengths is not None:
        for t in (x, delta, b, c):
            poison(t, lengths)
    on = lambda t: None if t is None else t.to(DEV)  # noqa: E731
    st = on(state)
    ws = hla.alloc_workspace(hla.hla_ssm_workspace_bytes(B, n, H, P, G, N, T), DEV)
    ws.fill_(255)
    run = lambda st, so: hla.hla_ssm_forward(  # noqa: E731
        sliced(x, extra, at), sliced(delta, extra, at), on(a), sliced(b, extra, at), sliced(c, extra, at), skip=on(skip),
        delta_bias=on(bias), lengths=on(lengths), state_in=st, state_out=so, workspace=ws)
    out = run(st, st)  # the state in place
    assert hla.hla_poll_error(ws) == 0
    by, bh = ssm_bounds(T, n, N, y, ym, hm)
    near(out, y, by)
    near(st, h, bh)
    so = torch.empty_like(st)
    assert torch.equal(run(on(state), so), out) and torch.equal(so, st)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_ssm_forward_plain_options(hla, dtype):
    """No skip, no bias, no softplus, no states, an output that is a slice."""
    T, (B, n, H, P, G, N) = TYPES[dtype], (2, 150, 4, 64, 2, 128)
    x, delta, a, b, c, _, _, _, _ = ssm_case(3, B, n, H, P, G, N, T, False)
    delta = (delta.float().abs() * 0.05).to(T)
    y, h, ym, hm = R.ssm(x, delta, a, b, c, softplus=False)
    wide = torch.zeros(B, n, H * P + 24, dtype=T, device=DEV)
    hla.hla_ssm_forward(*(t.to(DEV) for t in (x, delta, a, b, c)), wide[..., 8:8 + H * P].unflatten(-1, (H, P)),
                        softplus=False)
    near(wide[..., 8:8 + H * P].unflatten(-1, (H, P)), y, ssm_bounds(T, n, N, y, ym, hm)[0])
    assert not wide[..., :8].any() and not wide[..., 8 + H * P:].any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,H,P,G,N,extra,at", [(1, 1, 16, 1, 16, 8, 0), (3, 4, 32, 2, 32, 3, 1), (2, 6, 64, 3, 128, 8, 0),
                                                (80, 4, 128, 1, 64, 8, 0), (400, 1, 64, 1, 16, 8, 0)])
def test_ssm_step_continues_the_prompt(hla, dtype, B, H, P, G, N, extra, at):
    T, n = TYPES[dtype], 9
    x, delta, a, b, c, skip, bias, _, _ = ssm_case(P + N, B, n, H, P, G, N, torch.float32, False)
    x, delta, b, c = (t.to(T) for t in (x, delta, b, c))
    y, h, ym, hm = R.ssm(x, delta, a, b, c, skip, bias)
    on = lambda t: t.to(DEV)  # noqa: E731
    st = torch.empty(B, H, N, P, device=DEV)
    cut = lambda t: t[:, :5].contiguous().to(DEV)  # noqa: E731
    hla.hla_ssm_forward(cut(x), cut(delta), on(a), cut(b), cut(c), skip=on(skip), delta_bias=on(bias), state_out=st)
    part = ssm_bounds(T, n, N, y, ym, hm)[1] if T == torch.bfloat16 else None
    for t in range(5, n):
        tok = sliced(x[:, t].flatten(1), extra, at).unflatten(-1, (H, P))
        dt = sliced(delta[:, t], extra, at)
        bt, ct = (sliced(v[:, t].flatten(1), extra, at).unflatten(-1, (G, N)) for v in (b, c))
        out = hla.hla_ssm_step(tok, dt, on(a), bt, ct, st, tok if t % 2 else None, skip=on(skip), delta_bias=on(bias))
        # the prompt's state may carry its 2^-16 of the magnitude
        extra_y = 0.0 if part is None else 2.0 ** -16 * ym[:, t]
        near(out, y[:, t], ssm_bounds(T, n, N, y[:, t], ym[:, t], hm, step=True)[0] + extra_y)
    near(st, h, ssm_bounds(T, n, N, y, ym, hm, step=True)[1] if part is None else part)


def test_ssm_prompt_in_two_parts(hla):
    """A prompt cut anywhere and continued from its state equals the whole."""
    B, n, H, P, G, N = 2, 260, 2, 64, 1, 64
    x, delta, a, b, c, skip, bias, _, _ = ssm_case(8, B, n, H, P, G, N, torch.bfloat16, False)
    y, h, ym, hm = R.ssm(x, delta, a, b, c, skip, bias)
    st = None
    parts = []
    for lo, hi in ((0, 97), (97, 98), (98, n)):
        so = torch.empty(B, H, N, P, device=DEV) if st is None else st
        cut = lambda t: t[:, lo:hi].contiguous().to(DEV)  # noqa: E731, B023
        parts.append(hla.hla_ssm_forward(cut(x), cut(delta), a.to(DEV), cut(b), cut(c), skip=skip.to(DEV),
                                         delta_bias=bias.to(DEV), state_in=st, state_out=so))
        st = so
    by, bh = ssm_bounds(torch.bfloat16, n, N, y, ym, hm)
    near(torch.cat(parts, 1), y, by + 3 * 2.0 ** -16 * ym)
    near(st, h, 3 * bh)


def test_ssm_path(hla):
    assert hla.hla_ssm_forward_path(8, 2048, 32, 64, 1, 128) == (1, 1)
    assert hla.hla_ssm_forward_path(1, 32768, 16, 64, 2, 64) == (1, 3)  # few heads: cut along the sequence
    assert hla.hla_ssm_forward_path(8, 2048, 32, 64, 1, 128, dtype=torch.float32)[0] == 0
    assert hla.hla_ssm_forward_path(8, 2048, 32, 64, 1, 128, aligned_rows=False)[0] == 0


def test_ssm_empty_prompt(hla):
    B, H, P, G, N = 2, 2, 32, 1, 16
    z = lambda *s: torch.empty(*s, device=DEV)  # noqa: E731
    st = torch.randn(B, H, N, P, device=DEV)
    so = torch.empty_like(st)
    args = (z(B, 0, H, P), z(B, 0, H), -torch.ones(H, device=DEV), z(B, 0, G, N), z(B, 0, G, N))
    hla.hla_ssm_forward(*args, state_in=st, state_out=so)
    assert torch.equal(so, st)
    hla.hla_ssm_forward(*args, state_out=so)
    assert not so.any()


# ---------------------------------------------------------------------------------- q/k norm

def qk_case(seed, B, n, H, Hk, d, rot, T, weights=True):
    g = gen(seed)
    q, k = randn(g, B, n, H, d, T=T), randn(g, B, n, Hk, d, T=T)
    wq, wk = (randn(g, d, T=T), randn(g, d, T=T)) if weights else (None, None)
    angle = torch.randn(n + 5, rot // 2, generator=g)
    return g, q, k, wq, wk, angle.cos(), angle.sin()


QK = [(1, 1, 1, 1, 16, 0, False, 8, 0), (2, 5, 4, 2, 16, 8, False, 8, 0), (2, 7, 4, 4, 16, 16, True, 8, 8),
      (1, 33, 6, 2, 32, 24, False, 8, 0), (3, 130, 4, 1, 64, 64, False, 8, 0), (2, 65, 8, 2, 64, 32, True, 3, 1),
      (2, 40, 4, 4, 128, 64, False, 1, 0), (64, 1, 4, 2, 128, 128, True, 8, 0), (1, 300, 3, 3, 128, 72, False, 8, 0)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,n,H,Hk,d,rot,inter,extra,at", QK)
@pytest.mark.parametrize("given", [False, True])
def test_qk_norm_forward(hla, dtype, B, n, H, Hk, d, rot, inter, extra, at, given):
    T = TYPES[dtype]
    g, q, k, wq, wk, cos, sin = qk_case(n + d, B, n, H, Hk, d, rot, T, weights=not given)
    q[0, 0, 0] = 0.0  # a row of zeros
    pos = torch.randint(0, n + 5, (B, n), generator=g, dtype=torch.int32) if given else None
    where = pos.long() if given else (torch.arange(n) + 5).expand(B, n)
    on = lambda t: None if t is None else t.to(DEV)  # noqa: E731
    got = hla.hla_qk_norm_forward(sliced(q, extra, at), sliced(k, extra, at), on(wq), on(wk), on(cos), on(sin),
                                  positions=on(pos), pos0=0 if given else 5, eps=1e-5, interleaved=inter)
    for out, x, w in zip(got, (q, k), (wq, wk)):
        want, mag = R.qk_norm(x, w, cos, sin, where, H, 1e-5, inter)
        near(out, want, unit(T) * want.abs() + (d / 2 + 16) * U32 * mag)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,n,H,Hk,d,rot,inter,extra,at", QK)
def test_qk_norm_backward(hla, dtype, B, n, H, Hk, d, rot, inter, extra, at):
    T = TYPES[dtype]
    g, q, k, wq, wk, cos, sin = qk_case(3 * n + d, B, n, H, Hk, d, rot, T)
    dqo, dko = randn(g, B, H, n, d, T=T), randn(g, B, H, n, d, T=T)
    pos = torch.randint(0, n + 5, (B, n), generator=g, dtype=torch.int32)
    on = lambda t: t.to(DEV)  # noqa: E731
    run = lambda: hla.hla_qk_norm_backward(sliced(q, extra, at), sliced(k, extra, at), on(wq), on(wk), on(cos), on(sin),  # noqa: E731
                                           on(dqo), on(dko), positions=on(pos), eps=1e-5, interleaved=inter)
    got = run()
    for dx, dw, x, w, go in ((got[0], got[2], q, wq, dqo), (got[1], got[3], k, wk, dko)):
        wx, ww, mx, mw = R.qk_norm_grad(x, w, cos, sin, pos.long(), go, 1e-5, inter)
        near(dx, wx, unit(T) * wx.abs() + (2 * d + 32) * U32 * mx)
        near(dw, ww, (d + 32 + H + 256 + B * n * H / 256) * U32 * mw)
    for a, b in zip(got, run()):
        assert torch.equal(a, b)


def test_qk_norm_position_outside_the_tables(hla):
    """Only the rotated components of that token become NaN."""
    B, n, H, d, rot = 1, 4, 2, 32, 16
    _, q, k, wq, wk, cos, sin = qk_case(1, B, n, H, H, d, rot, torch.float32)
    pos = torch.tensor([[0, 9, -1, 8]], dtype=torch.int32)  # the tables have rows 0 .. 8
    out, _ = hla.hla_qk_norm_forward(*(t.to(DEV) for t in (q, k, wq, wk, cos, sin)), positions=pos.to(DEV))
    nan = torch.isnan(out[0, 0])
    assert nan[1:3, :rot].all() and not nan[1:3, rot:].any() and not nan[0].any() and not nan[3].any()


def test_qk_norm_empty(hla):
    z = torch.empty(2, 0, 2, 32, device=DEV)
    w = torch.ones(32, device=DEV)
    assert hla.hla_qk_norm_forward(z, z, w, w)[0].shape == (2, 2, 0, 32)
    e = torch.empty(2, 2, 0, 32, device=DEV)
    _, _, dwq, dwk = hla.hla_qk_norm_backward(z, z, w, w, None, None, e, e)
    assert not dwq.any() and not dwk.any()


# ---------------------------------------------------------------------------------- all of them

def test_another_stream(hla):
    """Calls go to the stream they are given, here one that first waits for the inputs."""
    s = torch.cuda.Stream()
    B, n, H, P, N = 2, 300, 4, 64, 64
    x, delta, a, b, c, skip, bias, _, _ = (None if t is None else t.to(DEV) for t in
                                           ssm_case(5, B, n, H, P, 1, N, torch.bfloat16, False))
    w = torch.randn(H * P, 4, device=DEV).to(torch.bfloat16)
    want_c = hla.hla_conv_forward(x.flatten(2), w)
    want_y = hla.hla_ssm_forward(want_c.unflatten(-1, (H, P)), delta, a, b, c)
    want_q = hla.hla_qk_norm_forward(x, x)[0]
    torch.cuda.synchronize()
    late = torch.zeros_like(x)
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        torch.cuda._sleep(20_000_000)
        late.copy_(x)
        got_c = hla.hla_conv_forward(late.flatten(2), w)
        got_y = hla.hla_ssm_forward(got_c.unflatten(-1, (H, P)), delta, a, b, c)
    got_q = hla.hla_qk_norm_forward(late, late, stream=s)[0]
    s.synchronize()
    assert torch.equal(got_c, want_c) and torch.equal(got_y, want_y) and torch.equal(got_q, want_q)


def test_in_a_cuda_graph(hla):
    """Every operator captured once and replayed on new inputs equals direct calls."""
    T, (B, n, H, P, N) = torch.bfloat16, (1, 700, 4, 64, 64)
    x, delta, a, b, c, skip, bias, _, _ = (None if t is None else t.to(DEV) for t in
                                           ssm_case(21, B, n, H, P, 1, N, T, False))
    w = torch.randn(H * P, 4, device=DEV).to(T)
    ws = [torch.empty(1 << 22, dtype=torch.uint8, device=DEV) for _ in range(3)]
    state = torch.empty(B, H, N, P, device=DEV)

    def run():
        y = hla.hla_conv_forward(x.flatten(2), w)
        z = hla.hla_ssm_forward(y.unflatten(-1, (H, P)), delta, a, b, c, state_out=state, workspace=ws[0])
        q, k = hla.hla_qk_norm_forward(z, z)
        dq, dk, _, _ = hla.hla_qk_norm_backward(z, z, None, None, None, None, q, k, workspace=ws[1])
        return (z, q, k, dq, dk, state) + hla.hla_conv_backward(x.flatten(2), w, dq.flatten(2), workspace=ws[2])[:2]

    assert hla.hla_ssm_workspace_bytes(B, n, H, P, 1, N, T) <= ws[0].numel()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        run()
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run()
    for seed in (1, 2):
        x.copy_(torch.randn(x.shape, generator=gen(seed)).to(T))
        graph.replay()
        torch.cuda.synchronize()
        kept = [t.clone() for t in got]
        for p, q in zip(kept, run()):
            assert torch.equal(p, q)


@pytest.mark.parametrize("captured", [False, True])
@pytest.mark.parametrize("B,n,H,Hk,d", [(1, 8, 2, 1, 64), (2, 300, 8, 4, 64), (4, 1024, 16, 16, 128)])
def test_calls_in_a_row(hla, captured, B, n, H, Hk, d):
    """Calls begin while those before them end: chains of calls through the same few buffers, with other
    kernels, a fill and another stream's work between them, give what they give with a wait after each."""
    T, C = torch.bfloat16, (H + Hk) * d
    g = torch.Generator(device=DEV).manual_seed(7)
    rand = lambda *s: torch.randn(*s, generator=g, device=DEV)
    x0, w, token0 = rand(B, n, C).to(T), (rand(C, 4) / 2).to(T), rand(B, C).to(T)
    delta, bm, a = rand(B, H).to(T), rand(B, 1, d).to(T), -rand(H).abs()
    x, y, dx = (torch.empty(B, n, C, dtype=T, device=DEV) for _ in range(3))
    token, conv_state, state = torch.empty_like(token0), torch.empty(B, 3, C, dtype=T, device=DEV), torch.empty(B, H, d, d, device=DEV)
    qo, ko = (torch.empty(B, H, n, d, dtype=T, device=DEV) for _ in range(2))
    tok_out = torch.empty(B, H, d, dtype=T, device=DEV)
    ws = [torch.empty(max(hla.hla_conv_backward_workspace_bytes(B, n, C, 4, T),
                          hla.hla_qk_norm_backward_workspace_bytes(B, n, H, Hk, d, T)), dtype=torch.uint8, device=DEV)]
    heads = lambda t: (t[..., :H * d].unflatten(-1, (H, d)), t[..., H * d:].unflatten(-1, (Hk, d)))
    side = torch.cuda.Stream()

    def chain(wait):
        kept = []

        def did(*results):
            wait()
            kept.extend(results)

        x.copy_(x0), token.copy_(token0), conv_state.zero_(), state.zero_()
        did()
        for _ in range(3):
            hla.hla_conv_forward(x, w, out=y)
            did()
            hla.hla_qk_norm_forward(*heads(y), q_out=qo, k_out=ko)
            did()
            dq, dk, _, _ = hla.hla_qk_norm_backward(*heads(y), None, None, None, None, ko, qo, workspace=ws[0])
            did()
            dx.zero_()
            hla.hla_conv_backward(x, w, y, dx=dx, workspace=ws[0])
            did()
            torch.add(x, dx, out=x)  # what the calls before it read
            x.clamp_(-4, 4)
            did(dq.clone(), dk.clone())
            for _ in range(3):
                hla.hla_conv_step(token, w, conv_state, out=token)
                did()
                hla.hla_ssm_step(token[:, :H * d].unflatten(-1, (H, d)), delta, a, bm, bm, state, tok_out)
                did()
                token[:, :H * d].copy_(tok_out.flatten(1))
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                token.clamp_(-2, 2)
            torch.cuda.current_stream().wait_stream(side)
            hla.hla_conv_step(token, w, conv_state, out=token)
            did(qo.clone(), ko.clone(), token.clone())
        return kept + [x, state, conv_state]

    want = [t.clone() for t in chain(torch.cuda.synchronize)]
    torch.cuda.synchronize()
    if captured:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = chain(lambda: None)
    for _ in range(5):
        if captured:
            graph.replay()
        else:
            got = chain(lambda: None)
        torch.cuda.synchronize()
        for p, r in zip(got, want):
            assert torch.equal(p, r)


@pytest.mark.parametrize("captured", [False, True])
@pytest.mark.parametrize("B,n,H,P,N,T", [(1, 3000, 2, 64, 64, torch.bfloat16), (4, 300, 32, 64, 128, torch.bfloat16),
                                         (1, 700, 2, 32, 16, torch.float32), (8, 40, 40, 16, 32, torch.float32)])
def test_scans_in_a_row(hla, captured, B, n, H, P, N, T):
    """The same for scans (one launch, or segments) whose inputs and states the calls before them write."""
    x0, delta, a, b, c, skip, bias, _, _ = (None if t is None else t.to(DEV) for t in
                                            ssm_case(33, B, n, H, P, 1, N, T, False))
    w = torch.randn(H * P, 4, generator=gen(3)).to(DEV).to(T)
    ws = torch.empty(hla.hla_ssm_workspace_bytes(B, n, H, P, 1, N, T), dtype=torch.uint8, device=DEV)
    x, y, state = torch.empty_like(x0), torch.empty_like(x0), torch.empty(B, H, N, P, device=DEV)

    def chain(wait):
        kept = []
        x.copy_(x0), state.zero_()
        wait()
        for _ in range(4):
            hla.hla_conv_forward(x.flatten(2), w, out=y.flatten(2))
            wait()
            hla.hla_ssm_forward(y, delta, a, b, c, out=x, state_in=state, state_out=state, workspace=ws)
            wait()
            hla.hla_ssm_step(x[:, -1], delta[:, -1], a, b[:, -1], c[:, -1], state, y[:, 0].contiguous())
            wait()
            hla.hla_ssm_forward(x, delta, a, b, c, out=y, state_in=state, state_out=state, workspace=ws)
            wait()
            x.copy_(y).clamp_(-2, 2)
            state.mul_(0.5)
            kept += [y.clone(), state.clone()]
            wait()
        return kept

    want = chain(torch.cuda.synchronize)
    torch.cuda.synchronize()
    if captured:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = chain(lambda: None)
    for _ in range(5):
        if captured:
            graph.replay()
        else:
            got = chain(lambda: None)
        torch.cuda.synchronize()
        for p, r in zip(got, want):
            assert torch.equal(p, r)


def test_rows_beyond_32_bit_offsets(hla):
    """Row offsets past 2^31 elements: the last rows equal those of a compact copy."""
    n, C, stride, T = 33000, 64, 1 << 16, torch.bfloat16  # 2.16e9 elements, 4.3 GB
    wide = torch.zeros(1, n, stride, dtype=T, device=DEV)
    g = torch.Generator(device=DEV).manual_seed(1)
    x = torch.randn(1, n, 3 * C, generator=g, device=DEV).to(T)
    wide[..., stride - 3 * C:] = x
    far = wide[..., stride - 3 * C:]
    w = torch.randn(C, 4, generator=g, device=DEV).to(T)
    assert torch.equal(hla.hla_conv_forward(far[..., :C], w), hla.hla_conv_forward(x[..., :C].contiguous(), w))
    for p, q in zip(hla.hla_qk_norm_forward(far[..., :C].unflatten(-1, (1, C)), far[..., C:2 * C].unflatten(-1, (1, C))),
                    hla.hla_qk_norm_forward(x[..., :C].unflatten(-1, (1, C)), x[..., C:2 * C].unflatten(-1, (1, C)))):
        assert torch.equal(p, q)
    heads = lambda t, i: t[..., i * C:(i + 1) * C].unflatten(-1, (1, C))  # noqa: E731
    a = -torch.ones(1, device=DEV)
    run = lambda t: hla.hla_ssm_forward(heads(t, 0), t[..., :1], a, heads(t, 1), heads(t, 2))  # noqa: E731
    assert torch.equal(run(far), run(x))


def test_refusals_of_the_binding(hla):
    x = torch.zeros(2, 4, 16, device=DEV)
    w = torch.zeros(16, 4, device=DEV)
    for kw in (dict(x=x.transpose(1, 2)), dict(weight=w.half()), dict(weight=w[:8]), dict(lengths=torch.zeros(2, device=DEV)),
               dict(state_in=torch.zeros(2, 4, 16, device=DEV)), dict(bias=torch.zeros(16))):
        with pytest.raises(ValueError):
            hla.hla_conv_forward(**{"x": x, "weight": w, **kw})
    with pytest.raises(TypeError):
        hla.hla_conv_forward(x.half(), w.half())
    with pytest.raises(hla.HLAError):
        hla.hla_conv_forward(x, torch.zeros(16, 7, device=DEV))
    y = torch.zeros(2, 4, 2, 32, device=DEV)
    with pytest.raises(hla.HLAError):
        hla.hla_qk_norm_forward(y, y, cos=torch.zeros(3, 8, device=DEV), sin=torch.zeros(3, 8, device=DEV))
    with pytest.raises(hla.HLAError):
        hla.hla_ssm_forward(torch.zeros(1, 4, 2, 24, device=DEV), torch.zeros(1, 4, 2, device=DEV),
                            -torch.ones(2, device=DEV), torch.zeros(1, 4, 1, 16, device=DEV),
                            torch.zeros(1, 4, 1, 16, device=DEV))
