"""The block's operators (gated recurrence, norms around a block, gated feed-forward projections) on the GPU
against their definitions in 64 bits, element by element within the bounds of block_ref.  A bf16 output
adds its one rounding, 2^-9 of the next power of two: 2^-8 of the value."""
import numpy as np
import pytest
import torch

import block_ref as R

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def hla():
    from paper_2510_27258_gb300 import build
    build.build()
    from paper_2510_27258_gb300 import hla as binding
    return binding


def gen(seed):
    return torch.Generator().manual_seed(seed)


def randn(g, *shape, T=torch.float32, scale=1.0):
    return (torch.randn(*shape, generator=g) * scale).to(T)


def near(name, got, want, bound):
    """Every element within its bound and the rounding of its type."""
    unit = 2.0 ** -8 if got.dtype == torch.bfloat16 else 2.0 ** -24
    got = got.double().cpu()
    assert got.shape == want.shape, name
    assert torch.isfinite(got).all(), name
    excess = (got - want).abs() - bound * (1 + unit) - unit * want.abs() - 1e-30
    assert not excess.numel() or float(excess.max()) <= 0, (name, float(excess.max()), float((got - want).abs().max()))


def sliced(t, extra=8, at=0, fill=float("nan")):
    """`t` on the GPU as a slice of rows that are wider by `extra` elements, from element `at` on."""
    wide = torch.full(t.shape[:-1] + (t.shape[-1] + extra,), fill, dtype=t.dtype, device=DEV)
    wide[..., at:at + t.shape[-1]] = t.to(DEV)
    return wide[..., at:at + t.shape[-1]]


def ragged(g, B, n):
    lens = [n, 0, 1] + [int(v) for v in torch.randint(0, n + 1, (max(B - 3, 0),), generator=g)]
    return torch.tensor(lens[:B], dtype=torch.int32)


def poison(t, lens):
    """A copy with NaN and infinities at and after each length: nothing there may be read into a result."""
    t = t.clone()
    for i, m in enumerate(lens.tolist()):
        t[i, m:] = float("nan")
        t[i, m + 1:m + 2] = float("inf")
    return t


def on(t):
    return None if t is None else t.to(DEV)


# ---------------------------------------------------------------------------------- recurrence

def glr_case(seed, B, n, C, T, ragged_lengths, slow=True):
    g = gen(seed)
    v = {k: randn(g, B, n, C, T=T, scale=1.5) for k in ("x", "r", "g")}
    v["decay"] = 8 * torch.log(0.9 + 0.0999 * torch.rand(C, generator=g)) if slow else -20 * torch.rand(C, generator=g) - 1e-3
    v["state"] = randn(g, B, C)
    return g, v, ragged(g, B, n) if ragged_lengths else None


GLR = [(1, 1, 8, False, 0, 0, True), (3, 2, 24, True, 8, 0, True), (4, 37, 264, True, 8, 8, True),
       (2, 130, 203, False, 5, 3, False), (5, 64, 130, True, 0, 0, True), (1, 1000, 64, False, 8, 0, True),
       (2, 600, 70, True, 1, 1, False), (1, 65, 1, False, 3, 2, True), (40, 33, 66, True, 0, 0, True),
       (1, 2500, 100, False, 0, 0, True), (70, 5, 640, False, 0, 0, True), (40, 32, 520, True, 8, 0, False),
       (120, 9, 203, True, 3, 1, True), (304, 1, 30, True, 0, 0, True)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,n,C,lens,extra,at,slow", GLR)
def test_glr_forward(hla, dtype, B, n, C, lens, extra, at, slow):
    T = TYPES[dtype]
    _, v, lengths = glr_case(n + C, B, n, C, T, lens, slow)
    want, last, bound, last_bound = R.glr(v["x"], v["r"], v["g"], v["decay"], v["state"], lengths)
    x, r, g = ((v[k] if lengths is None else poison(v[k], lengths)) for k in ("x", "r", "g"))
    st = on(v["state"])
    out = hla.hla_glr_forward(sliced(x, extra, at), sliced(r, extra, at), sliced(g, extra, at), on(v["decay"]),
                              lengths=on(lengths), state_in=st, state_out=st)  # the state in place
    near("y", out, want, bound)
    near("state", st, last, last_bound)
    # from no state, into a strided output, with marks: the states before every 32nd token
    want, last, bound, last_bound = R.glr(v["x"], v["r"], v["g"], v["decay"], None, lengths)
    wide = torch.zeros(B, n, C + 7, dtype=T, device=DEV)
    marks = torch.full((B, hla.hla_glr_marks(n), C), float("nan"), device=DEV)
    so = torch.full_like(st, float("nan"))
    hla.hla_glr_forward(on(x), on(r), on(g), on(v["decay"]), wide[..., 3:3 + C], lengths=on(lengths), state_out=so,
                        marks=marks)
    near("y", wide[..., 3:3 + C], want, bound)
    near("state", so, last, last_bound)
    assert not wide[..., :3].any() and not wide[..., 3 + C:].any()
    for k in range(0, marks.shape[1], 3):
        part = None if lengths is None else lengths.clamp(max=32 * k)
        _, at_mark, _, mark_bound = R.glr(*(v[m][:, :32 * k] for m in ("x", "r", "g")), v["decay"], None, part)
        near("marks", marks[:, k], at_mark, mark_bound)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,n,C,lens,extra,at,slow", GLR)
def test_glr_backward(hla, dtype, B, n, C, lens, extra, at, slow):
    T = TYPES[dtype]
    gn, v, lengths = glr_case(n * C, B, n, C, T, lens, slow)
    dy, dl = randn(gn, B, n, C, T=T), randn(gn, B, C)
    want = R.glr_grad(v["x"], v["r"], v["g"], v["decay"], dy, v["state"], dl, lengths)
    x, r, g, dy = ((t if lengths is None else poison(t, lengths)) for t in (v["x"], v["r"], v["g"], dy))
    xs, rs, gs, ds = (sliced(t, extra, at) for t in (x, r, g, dy))
    marks = torch.full((B, hla.hla_glr_marks(n), C), float("nan"), device=DEV)
    hla.hla_glr_forward(xs, rs, gs, on(v["decay"]), lengths=on(lengths), state_in=on(v["state"]), marks=marks)
    state = on(dl)

    def run():
        state.copy_(dl)
        return hla.hla_glr_backward(xs, rs, gs, on(v["decay"]), ds, marks, dstate_out=state, dstate_in=state,
                                    lengths=on(lengths))
    got = run()
    for name, t in zip(("dx", "dr", "dg", "ddecay"), got):
        near(name, t, *want[name])
    near("dstate", state, *want["dstate"])
    again = run()
    assert all(torch.equal(a, b) for a, b in zip(got, again))  # sums in a fixed order
    # gradients side by side, no gradient of the state
    want = R.glr_grad(v["x"], v["r"], v["g"], v["decay"], torch.where(R.live(lengths, B, n), dy, torch.zeros((), dtype=T)),
                      v["state"], None, lengths)
    rows = torch.zeros(B, n, 3 * C + 1, dtype=T, device=DEV)
    got = hla.hla_glr_backward(on(x), on(r), on(g), on(v["decay"]), on(dy), marks, rows[..., :C], rows[..., C:2 * C],
                               rows[..., 2 * C:3 * C], lengths=on(lengths))
    for name, t in zip(("dx", "dr", "dg", "ddecay"), got):
        near(name, t, *want[name])
    assert not rows[..., 3 * C:].any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,C,extra,at", [(1, 8, 8, 0), (7, 203, 3, 1), (64, 264, 8, 0), (33, 1, 0, 0)])
def test_glr_step_continues_the_prompt(hla, dtype, B, C, extra, at):
    """A prompt and then single tokens equal the whole sequence at once."""
    T = TYPES[dtype]
    _, v, _ = glr_case(B + C, B, 12, C, T, False)
    want, last, bound, last_bound = R.glr(v["x"], v["r"], v["g"], v["decay"], v["state"])
    st = on(v["state"])
    hla.hla_glr_forward(*(v[k][:, :7].contiguous().to(DEV) for k in ("x", "r", "g")), on(v["decay"]), state_in=st, state_out=st)
    for t in range(7, 12):
        x, r, g = (sliced(v[k][:, t], extra, at) for k in ("x", "r", "g"))
        out = hla.hla_glr_step(x, r, g, on(v["decay"]), st, (None, x, r, g, None)[t - 7])
        near("y", out, want[:, t], bound[:, t])
    near("state", st, last, last_bound)


def test_glr_empty_prompt_keeps_the_state(hla):
    st, decay, none = torch.randn(2, 16, device=DEV), -torch.ones(16, device=DEV), torch.empty(2, 0, 16, device=DEV)
    keep = st.clone()
    hla.hla_glr_forward(none, none, none, decay, state_in=st, state_out=st)
    assert torch.equal(st, keep)
    back = torch.empty_like(st)
    grads = hla.hla_glr_backward(none, none, none, decay, none, torch.empty(2, 0, 16, device=DEV), dstate_out=st, dstate_in=back)
    assert torch.equal(back, keep) and not grads[3].any()
    hla.hla_glr_forward(none, none, none, decay, state_out=st)
    assert not st.any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_glr_extreme_gates(hla, dtype):
    """Gates that are shut or open as far as the type goes: no NaN, and what the limits say."""
    T = TYPES[dtype]
    for r, g, keeps, adds in ((-1e4, 0.0, True, False), (-200.0, 1e4, True, False), (0.0, -1e4, False, False),
                              (1e4, 1e4, False, True), (-float("inf"), float("inf"), True, False)):
        x = torch.full((1, 70, 64), 2.0, dtype=T, device=DEV)
        st, decay = torch.ones(1, 64, device=DEV), torch.full((64,), -50.0, device=DEV)
        y = hla.hla_glr_forward(x, torch.full_like(x, r), torch.full_like(x, g), decay, state_in=st)
        want = 1.0 if keeps else 2.0 if adds else 0.0
        # (shut at r = 0: the state decays by e^-25 a token, which is below 2^-24 after one)
        assert torch.isfinite(y).all() and float((y[:, 1:] - want).abs().max()) <= 2.0 ** -23
        marks = torch.empty(1, 3, 64, device=DEV)
        hla.hla_glr_forward(x, torch.full_like(x, r), torch.full_like(x, g), decay, state_in=st, marks=marks)
        grads = hla.hla_glr_backward(x, torch.full_like(x, r), torch.full_like(x, g), decay, x, marks)
        assert all(torch.isfinite(t).all() for t in grads)


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("which", ["x", "r", "g"])
def test_glr_is_causal_for_tokens_that_are_not_finite(hla, which, bad):
    _, v, _ = glr_case(9, 2, 300, 130, torch.float32, False)
    clean = hla.hla_glr_forward(on(v["x"]), on(v["r"]), on(v["g"]), on(v["decay"]))
    v[which][0, 150, 7] = bad
    got = hla.hla_glr_forward(on(v["x"]), on(v["r"]), on(v["g"]), on(v["decay"]))
    if bad != bad:
        assert torch.isnan(got[0, 150:, 7]).all()
    got[0, 150:, 7] = clean[0, 150:, 7]
    assert torch.equal(got, clean)


@pytest.mark.parametrize("B,n,C", [(1, 3000, 66), (2, 700, 130), (40, 70, 66)])
def test_glr_states_that_are_nan(hla, B, n, C):
    """NaN in every channel: the states of a whole sequence turn to NaN, and blocks of one sequence still meet."""
    _, v, _ = glr_case(n, B, n, C, torch.float32, False)
    x, r, g, decay = (on(v[k]) for k in ("x", "r", "g", "decay"))
    marks = torch.empty(B, hla.hla_glr_marks(n), C, device=DEV)
    clean = hla.hla_glr_forward(x, r, g, decay, marks=marks)
    grads = hla.hla_glr_backward(x, r, g, decay, x, marks)
    bad, at = x.clone(), n // 3
    bad[0, at] = float("nan")
    state = torch.empty(B, C, device=DEV)
    y = hla.hla_glr_forward(bad, r, g, decay, state_out=state)
    assert torch.isnan(y[0, at:]).all() and torch.isnan(state[0]).all()
    assert torch.equal(y[0, :at], clean[0, :at]) and torch.equal(y[1:], clean[1:])
    got = hla.hla_glr_backward(x, r, g, decay, bad, marks)  # a gradient that is NaN there, in tokens before it
    for a, b in zip(got[:3], grads):
        assert torch.isnan(a[0, :at + 1]).all()
        assert torch.equal(a[0, at + 1:], b[0, at + 1:]) and torch.equal(a[1:], b[1:])
    assert torch.isnan(got[3]).all()


# ---------------------------------------------------------------------------------- norms

NORM = [((1, 1), dict()), ((5, 8), dict(dropout=0.5)), ((37, 203), dict(dropout=0.1, gate=False)),
        ((300, 256), dict(dropout=0.25, act=R.SIGMOID)), ((64, 260), dict(dropout=0.1)),
        ((700, 2048), dict(dropout=0.1, alpha=0.75)), ((9, 2100), dict(act=R.LINEAR, post=False)),
        ((11, 4104), dict(pre=False, dropout=0.1)), ((3, 8192), dict(dropout=0.1)), ((2, 1023), dict(weights=False)),
        ((2, 8201), dict(dropout=0.1)), ((3, 20000), dict(post=False)), ((2, 8200), dict(pre=False, gate=False)),
        ((400, 24), dict(post=False, pre=False)), ((33, 1022), dict(dropout=0.1)), ((77, 30), dict(dropout=0.25)),
        ((2000, 32), dict(dropout=0.1)), ((51, 60), dict(dropout=0.5)), ((131, 100), dict(dropout=0.1)),
        ((41, 250), dict(dropout=0.1, gate=False)), ((3000, 49), dict(dropout=0.1)), ((9, 8190), dict(dropout=0.1))]


def norm_case(seed, rows, C, T, gate=True, weights=True, **kw):
    g = gen(seed)
    v = {"x": randn(g, rows, C, T=T), "y": randn(g, rows, C, T=T, scale=0.5), "gate": randn(g, rows, C, T=T) if gate else None}
    for k in ("w_post", "scale", "w_pre"):
        v[k] = randn(g, C, T=T) if weights else None
    kw = {"alpha": 1.0, "eps": 1e-6, "dropout": 0.0, "act": R.SILU, "post": True, "pre": True, **kw}
    kw["seed"], kw["offset"] = 2 ** 63 + 12345 * seed, 2 ** 40 + seed
    own = {("post_norm" if k == "post" else "pre_norm" if k == "pre" else k): x for k, x in kw.items()}
    return g, v, kw, own


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size,opts", NORM)
@pytest.mark.parametrize("extra,at", [(8, 0), (3, 1)])
def test_block_norm(hla, dtype, size, opts, extra, at):
    T = TYPES[dtype]
    rows, C = size
    g, v, kw, own = norm_case(rows + C, rows, C, T, **opts)
    dx_out, dh = randn(g, rows, C, T=T), randn(g, rows, C, T=T) if kw["pre"] else None
    want = R.norm(**v, dx_out=dx_out, dh=dh, **kw)
    w = {k: on(v[k]) for k in ("w_post", "scale", "w_pre")}
    cut = lambda t: None if t is None else sliced(t, extra, at)  # noqa: E731
    x, y, gate = cut(v["x"]), cut(v["y"]), cut(v["gate"])
    h = sliced(torch.zeros(rows, C, dtype=T), extra, at, 7.0)
    x_out, h = hla.hla_block_norm_forward(x, y, gate, None, h, **w, **own)
    near("x_out", x_out, *want["x_out"])
    assert (h is None) == (not kw["pre"])
    if h is not None:
        near("h", h, *want["h"])
        base = h._base
        assert (base[:, :at] == 7).all() and (base[:, at + C:] == 7).all()
    same = x.clone()
    again, _ = hla.hla_block_norm_forward(same, y, gate, same, **w, **own)  # in place
    assert again is same and torch.equal(same, x_out)

    def run():
        return hla.hla_block_norm_backward(x, y, gate, cut(dx_out), cut(dh), **w, **own)
    got = run()
    for name, t in zip(("dx", "dy", "dgate", "dw_post", "dscale", "dw_pre"), got):
        if name == "dgate" and v["gate"] is None or name.startswith("d") and name[1:] in v and v[name[1:]] is None:
            assert t is None
        elif name[1:] in ("w_post", "w_pre") and not kw[name[3:]]:
            assert t is None
        else:
            near(name, t, *want[name])
    assert all(a is b is None or torch.equal(a, b) for a, b in zip(got, run()))
    d = on(dx_out)
    got2 = hla.hla_block_norm_backward(x, y, gate, d, cut(dh), d, **w, **own)  # dx over dx_out
    assert got2[0] is d and torch.equal(d, got[0]) and torch.equal(got2[1], got[1])


def test_block_norm_batches_and_masks(hla):
    """[B, n, C] is the same rows, and a value's bits depend on row, column, seed and offset alone."""
    _, v, _, own = norm_case(5, 24, 256, torch.float32, dropout=0.5)
    args = [on(v[k]) for k in ("x", "y", "gate")]
    a = hla.hla_block_norm_forward(*args, **own)
    b = hla.hla_block_norm_forward(*(t.view(4, 6, 256) for t in args), **own)
    assert all(torch.equal(s, t.view(24, 256)) for s, t in zip(a, b))
    kept = (a[0] != args[0])
    other = hla.hla_block_norm_forward(*args, **{**own, "offset": own["offset"] + 1})[0] != args[0]
    # two masks of one half each: they agree on 0.5 +- 4.5 deviations of sqrt(1 / 4 / 6144) = 0.0064
    assert abs(float(kept.float().mean()) - 0.5) < 0.03 and abs(float((kept == other).float().mean()) - 0.5) < 0.03
    strided = hla.hla_block_norm_forward(*(sliced(v[k], 1, 1) for k in ("x", "y", "gate")), **own)[0]
    assert torch.equal(strided != args[0], kept)


@pytest.mark.parametrize("C", [24, 203, 256, 2048, 2047, 8200])
def test_block_norm_dropped_values_that_are_not_finite(hla, C):
    """What y and gate hold where a value is dropped reaches nothing, in either direction."""
    g, v, kw, own = norm_case(11, 40, C, torch.bfloat16, dropout=0.5, post=False)
    x, y, gate, dx_out, dh = (on(t) for t in (v["x"], v["y"], v["gate"], randn(g, 40, C, T=torch.bfloat16),
                                              randn(g, 40, C, T=torch.bfloat16)))
    dropped = on(torch.from_numpy(R.words(40, C, kw["seed"], kw["offset"]) < np.uint64(2 ** 31)))
    odd = torch.arange(C, device=DEV) % 2 == 1
    bad_y = torch.where(dropped, torch.where(odd, float("nan"), float("inf")).to(y.dtype), y)
    bad_gate = torch.where(dropped, torch.where(odd, -float("inf"), float("nan")).to(y.dtype), gate)
    w = {k: on(v[k]) for k in ("w_post", "scale", "w_pre")}
    assert all(torch.equal(a, b) for a, b in zip(hla.hla_block_norm_forward(x, y, gate, **w, **own),
                                                 hla.hla_block_norm_forward(x, bad_y, bad_gate, **w, **own)))
    for a, b in zip(hla.hla_block_norm_backward(x, y, gate, dx_out, dh, **w, **own),
                    hla.hla_block_norm_backward(x, bad_y, bad_gate, dx_out, dh, **w, **own)):
        assert a is b is None or torch.equal(a, b)


def test_block_norm_rows_of_zeros(hla):
    """eps keeps a row of zeros finite, forwards and backwards."""
    z = torch.zeros(3, 512, device=DEV)
    x, h = hla.hla_block_norm_forward(z, z, z)
    assert not x.any() and not h.any()
    grads = hla.hla_block_norm_backward(z, z, z, z + 1, z + 1)
    assert all(t is None or torch.isfinite(t).all() for t in grads)
    none = torch.empty(0, 512, device=DEV)
    grads = hla.hla_block_norm_backward(none, none, None, none, none, w_post=z[0], scale=z[0], w_pre=z[0])
    assert grads[0].shape == (0, 512) and not any(t.any() for t in grads[3:])


# ---------------------------------------------------------------------------------- feed-forward

FFN = [(1, 8, 8, R.SILU), (3, 1, 1, R.SILU), (16, 264, 520, R.SIGMOID), (129, 130, 67, R.SILU), (333, 260, 103, R.LINEAR),
       (300, 512, 1032, R.SILU), (1, 2056, 384, R.SILU), (64, 33, 2050, R.SIGMOID), (520, 64, 328, R.SILU),
       (17, 1000, 77, R.SILU), (256, 320, 136, R.SILU), (257, 72, 200, R.SILU), (100, 1600, 72, R.SIGMOID),
       (5, 2048, 1288, R.SILU), (9, 700, 1100, R.SILU), (32, 1030, 600, R.SIGMOID), (31, 64, 50, R.SILU),
       (8, 4100, 70, R.LINEAR), (1030, 520, 2600, R.SILU)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,K,F,act", FFN)
@pytest.mark.parametrize("extra,at", [(8, 0), (3, 1)])
def test_ffn(hla, dtype, M, K, F, act, extra, at):
    T = TYPES[dtype]
    g = gen(M + K + F)
    x, w, dout = randn(g, M, K, T=T), randn(g, 2, F, K, T=T, scale=K ** -0.5), randn(g, M, F, T=T)
    # bf16 keeps the projections' gradients as bf16 between the products: half a step, 2^-8
    want = R.ffn(x, w, dout, act, 2.0 ** -8 if dtype == "bf16" else 0.0)
    cut = lambda t, fill=float("nan"): sliced(t, extra, at, fill)  # noqa: E731
    out = cut(torch.zeros_like(dout), 7.0)
    hla.hla_ffn_forward(cut(x), on(w), out, act=act)
    near("out", out, *want["out"])
    assert (out._base[:, :at] == 7).all() and (out._base[:, at + F:] == 7).all()
    dx = cut(torch.zeros_like(x), 7.0)

    def run():
        return hla.hla_ffn_backward(cut(x), on(w), cut(dout), dx, act=act)
    got = [t.clone() for t in run()]
    near("dx", got[0], *want["dx"])
    near("dw", got[1], *want["dw"])
    assert (dx._base[:, :at] == 7).all() and (dx._base[:, at + K:] == 7).all()
    assert all(torch.equal(a, b) for a, b in zip(got, run()))


def test_ffn_batches_and_none(hla):
    x, w = torch.randn(2, 5, 64, device=DEV), torch.randn(2, 96, 64, device=DEV)
    out = hla.hla_ffn_forward(x, w)
    assert out.shape == (2, 5, 96) and torch.equal(out.view(10, 96), hla.hla_ffn_forward(x.view(10, 64), w))
    none = torch.empty(0, 64, device=DEV)
    assert hla.hla_ffn_forward(none, w).shape == (0, 96)
    dx, dw = hla.hla_ffn_backward(none, w, torch.empty(0, 96, device=DEV))
    assert dx.shape == (0, 64) and not dw.any()


# ---------------------------------------------------------------------------------- as they are used

def chain(hla, v, ws):
    """A block: norm, recurrence, norm with gate and residual, feed-forward."""
    y = hla.hla_glr_forward(v["x"], v["r"], v["g"], v["decay"])
    x1, h = hla.hla_block_norm_forward(v["x"], y, v["r"], scale=v["scale"], dropout=0.1, seed=3)
    f = hla.hla_ffn_forward(h, v["w"], workspace=ws)
    return hla.hla_block_norm_forward(x1, f, None, pre_norm=False)[0]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_chain_on_other_streams_and_in_graphs(hla, dtype):
    T = TYPES[dtype]
    g = gen(1)
    C = 256
    v = {k: randn(g, 2, 150, C, T=T).to(DEV) for k in ("x", "r", "g")}
    v["decay"], v["scale"] = -torch.rand(C, generator=g).to(DEV) - 0.01, randn(g, C, T=T).to(DEV)
    v["w"] = randn(g, 2, C, C, T=T, scale=C ** -0.5).to(DEV)
    ws = hla.alloc_workspace(hla.hla_ffn_workspace_bytes(300, C, C, T), DEV)
    want = chain(hla, v, ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = [chain(hla, v, ws) for _ in range(3)]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            captured = chain(hla, v, ws)
        captured.zero_()
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(t, want) for t in got) and torch.equal(captured, want)


def test_long_sequences_of_few_channels(hla):
    """Blocks of a cluster that hand their runs on many times, with both shapes of a block."""
    for B, n, C in ((1, 9000, 24), (1, 5000, 600), (2, 3001, 40), (3, 1500, 1100)):
        g, v, lengths = glr_case(n, B, n, C, torch.bfloat16, B > 2)
        want, last, bound, last_bound = R.glr(v["x"], v["r"], v["g"], v["decay"], v["state"], lengths)
        so = torch.empty(B, C, device=DEV)
        marks = torch.empty(B, hla.hla_glr_marks(n), C, device=DEV)
        y = hla.hla_glr_forward(on(v["x"]), on(v["r"]), on(v["g"]), on(v["decay"]), lengths=on(lengths),
                                state_in=on(v["state"]), state_out=so, marks=marks)
        near("y", y, want, bound)
        near("state", so, last, last_bound)
        dy, dl = randn(g, B, n, C, T=torch.bfloat16), randn(g, B, C)
        want = R.glr_grad(v["x"], v["r"], v["g"], v["decay"], dy, v["state"], dl, lengths)
        di = torch.empty(B, C, device=DEV)
        got = hla.hla_glr_backward(on(v["x"]), on(v["r"]), on(v["g"]), on(v["decay"]), on(dy), marks, dstate_out=on(dl),
                                   dstate_in=di, lengths=on(lengths))
        for name, t in zip(("dx", "dr", "dg", "ddecay", "dstate"), got + (di,)):
            near(name, t, *want[name])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_more_than_2_31_elements_apart(hla, dtype):
    """Offsets inside the tensors pass 32 bits: the same values in rows that are 2^29 and a bit elements apart."""
    T, step, n, C = TYPES[dtype], (1 << 29) + 64, 6, 40
    if torch.cuda.mem_get_info()[0] < 40e9:
        pytest.skip("the device's memory is in use")
    buf = torch.empty(n * step, dtype=T, device=DEV)
    places = iter(range(0, 1 << 28, 1 << 20))

    def far(values=None):
        t = buf.as_strided((1, n, C), (n * step, step, 1), next(places))
        return t if values is None else t.copy_(values)
    g = gen(4)
    x, r, gt, dy = (randn(g, 1, n, C, T=T).to(DEV) for _ in range(4))
    decay = -torch.rand(C, generator=g).to(DEV) - 0.1
    marks = torch.empty(1, 1, C, device=DEV)
    fx, fr, fg, fdy = (far(t) for t in (x, r, gt, dy))
    assert torch.equal(hla.hla_glr_forward(fx, fr, fg, decay, far(), marks=marks), hla.hla_glr_forward(x, r, gt, decay))
    want = hla.hla_glr_backward(x, r, gt, decay, dy, marks)
    got = hla.hla_glr_backward(fx, fr, fg, decay, fdy, marks, far(), far(), far())
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    w = randn(g, C, T=T).to(DEV)
    kw = dict(w_post=w, scale=w, w_pre=w, dropout=0.25, seed=5)
    want = hla.hla_block_norm_forward(x, r, gt, **kw)
    got = hla.hla_block_norm_forward(fx, fr, fg, far(), far(), **kw)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    want = hla.hla_block_norm_backward(x, r, gt, dy, x, **kw)
    got = hla.hla_block_norm_backward(fx, fr, fg, fdy, fx, far(), far(), far(), **kw)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    wf = randn(g, 2, C, C, T=T).to(DEV)
    assert torch.equal(hla.hla_ffn_forward(fx, wf, far()), hla.hla_ffn_forward(x, wf))
    want, got = hla.hla_ffn_backward(x, wf, dy), hla.hla_ffn_backward(fx, wf, fdy, far())
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_used_workspaces(hla, dtype):
    """What a workspace held before does not matter, and a call leaves no error in it."""
    T = TYPES[dtype]
    for M, K, F in ((40, 72, 136), (300, 130, 260)):
        g = gen(M)
        x, w, d = randn(g, M, K, T=T).to(DEV), randn(g, 2, F, K, T=T).to(DEV), randn(g, M, F, T=T).to(DEV)
        y, gate = randn(g, M, K, T=T).to(DEV), randn(g, M, K, T=T).to(DEV)
        decay, marks = -torch.ones(K, device=DEV), torch.empty(1, hla.hla_glr_marks(M), K, device=DEV)
        seq = [t[None] for t in (x, y, gate)]
        hla.hla_glr_forward(*seq, decay, marks=marks)
        for size, call in (
                (hla.hla_ffn_workspace_bytes(M, K, F, T), lambda ws: [hla.hla_ffn_forward(x, w, workspace=ws)]),
                (hla.hla_ffn_backward_workspace_bytes(M, K, F, T), lambda ws: hla.hla_ffn_backward(x, w, d, workspace=ws)),
                (hla.hla_block_norm_backward_workspace_bytes(M, K, T),
                 lambda ws: hla.hla_block_norm_backward(x, y, gate, y, x, w_pre=x[0], workspace=ws)),
                (hla.hla_glr_backward_workspace_bytes(1, M, K, T),
                 lambda ws: hla.hla_glr_backward(*seq, decay, seq[0], marks, workspace=ws))):
            ws = hla.alloc_workspace(size, DEV)
            want = [t.clone() for t in call(ws) if t is not None]
            ws.fill_(255)
            got = [t for t in call(ws) if t is not None]
            assert all(torch.equal(a, b) for a, b in zip(got, want))
            hla.hla_poll_error(ws)


def test_calls_on_another_stream_without_a_workspace(hla):
    """Scratch and outputs of a call on another stream, while the current one goes on allocating and writing."""
    g = torch.Generator(device=DEV).manual_seed(3)
    rand = lambda *s: torch.randn(*s, generator=g, device=DEV).to(torch.bfloat16)  # noqa: E731
    x, r, gt, dy, w = rand(1, 700, 264), rand(1, 700, 264), rand(1, 700, 264), rand(1, 700, 264), rand(2, 520, 264)
    decay, few = -torch.rand(264, generator=g, device=DEV) - 0.01, x[0, :20]
    w_pre = decay.to(x.dtype)  # (an input lives as long as the kernels that read it)
    marks = torch.empty(1, hla.hla_glr_marks(700), 264, device=DEV)
    hla.hla_glr_forward(x, r, gt, decay, marks=marks)
    calls = [lambda s: hla.hla_glr_forward(x, r, gt, decay, stream=s),
             lambda s: hla.hla_glr_backward(x, r, gt, decay, dy, marks, stream=s),
             lambda s: hla.hla_block_norm_forward(x, r, gt, dropout=0.5, seed=1, stream=s),
             lambda s: hla.hla_block_norm_backward(x, r, gt, dy, x, w_pre=w_pre, stream=s),
             lambda s: hla.hla_ffn_forward(x, w, stream=s), lambda s: hla.hla_ffn_backward(x, w, rand_out, stream=s),
             lambda s: hla.hla_ffn_forward(few, w, stream=s), lambda s: hla.hla_ffn_backward(few, w, rand_out[0, :20], stream=s)]
    rand_out = rand(1, 700, 520)
    tensors = lambda out: [t for t in (out if isinstance(out, tuple) else (out,)) if t is not None]  # noqa: E731
    want = [[t.clone() for t in tensors(call(None))] for call in calls]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(40_000_000)  # the calls' kernels run well after the calls return
    got = []
    for call in calls:
        got.append(tensors(call(side)))
        for size in (1 << 12, 1 << 18, 1 << 20, 1 << 22):
            for _ in range(4):
                torch.empty(size, dtype=torch.uint8, device=DEV).fill_(255)
    torch.cuda.current_stream().wait_stream(side)
    assert [all(torch.equal(a, b) for a, b in zip(p, q)) for p, q in zip(got, want)] == [True] * len(calls)


def test_gradients_in_graphs(hla):
    """A training step captured twice, each graph with workspaces of its own, replayed by turns on new inputs."""
    g = gen(8)
    B, n, C, F, T = 2, 100, 136, 264, torch.bfloat16
    v = {k: randn(g, B, n, C, T=T).to(DEV) for k in ("x", "r", "g", "dy")}
    w, decay, wr = randn(g, 2, F, C, T=T).to(DEV), -torch.rand(C, generator=g).to(DEV) - 0.01, randn(g, C, T=T).to(DEV)
    dout = randn(g, B, n, F, T=T).to(DEV)

    def step():
        marks = torch.empty(B, hla.hla_glr_marks(n), C, device=DEV)
        y = hla.hla_glr_forward(v["x"], v["r"], v["g"], decay, marks=marks)
        kw = dict(w_pre=wr, scale=wr, dropout=0.1, seed=2, offset=3)
        x1, h = hla.hla_block_norm_forward(v["x"], y, v["g"], **kw)
        dh, dw = hla.hla_ffn_backward(h, w, dout)
        dn = hla.hla_block_norm_backward(v["x"], y, v["g"], v["dy"], dh, **kw)
        return [hla.hla_ffn_forward(h, w), x1, dw] + [t for t in dn if t is not None] + list(
            hla.hla_glr_backward(v["x"], v["r"], v["g"], decay, dn[1], marks))
    step()
    graphs, outs = [], []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(step())
        graphs.append(graph)
    for turn in range(4):
        v["x"].normal_(), dout.normal_()
        want = step()
        graphs[turn % 2].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs[turn % 2], want))
