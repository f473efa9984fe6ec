"""The block's operators on either side of the sizes where another kernel takes over, and far along each dimension."""
import pytest
import torch

import block_ref as R
from test_gpu_block import DEV, TYPES, gen, glr_case, near, norm_case, on, randn

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def hla():
    from paper_2510_27258_gb300 import build
    build.build()
    from paper_2510_27258_gb300 import hla as binding
    return binding


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,K,F", [(16, 72, 9600), (16, 72, 9601), (3, 40, 28672), (128, 136, 520), (129, 136, 520), (32, 200, 300),
                                   (33, 200, 300), (5, 20000, 72), (16, 130, 4000), (17, 130, 4000), (40000, 24, 40), (9, 8, 40000)])
def test_feed_forward(hla, dtype, M, K, F):
    T = TYPES[dtype]
    g = gen(M + K + F)
    x, w, dout = randn(g, M, K, T=T), randn(g, 2, F, K, T=T, scale=K ** -0.5), randn(g, M, F, T=T)
    want = R.ffn(x, w, dout, R.SILU, 2.0 ** -8 if dtype == "bf16" else 0.0)
    near("out", hla.hla_ffn_forward(on(x), on(w)), *want["out"])
    dx, dw = hla.hla_ffn_backward(on(x), on(w), on(dout))
    near("dx", dx, *want["dx"])
    near("dw", dw, *want["dw"])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,C", [(30000, 24), (7, 256), (7, 257), (5, 2048), (5, 2049), (5, 4096), (5, 4097), (3, 8192), (3, 8193),
                                    (3, 12288), (400, 8200), (2, 65536)])
def test_norms(hla, dtype, rows, C):
    T = TYPES[dtype]
    g, v, kw, own = norm_case(rows + C, rows, C, T, dropout=0.1)
    dx_out, dh = randn(g, rows, C, T=T), randn(g, rows, C, T=T)
    want = R.norm(**v, dx_out=dx_out, dh=dh, **kw)
    x, y, gate = (on(v[k]) for k in ("x", "y", "gate"))
    w = {k: on(v[k]) for k in ("w_post", "scale", "w_pre")}
    for name, t in zip(("x_out", "h"), hla.hla_block_norm_forward(x, y, gate, **w, **own)):
        near(name, t, *want[name])
    got = hla.hla_block_norm_backward(x, y, gate, on(dx_out), on(dh), **w, **own)
    for name, t in zip(("dx", "dy", "dgate", "dw_post", "dscale", "dw_pre"), got):
        near(name, t, *want[name])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,n,C", [(3000, 3, 40), (1, 3, 20000), (2, 129, 4096), (152, 33, 64), (153, 33, 64), (1, 64, 2048),
                                   (1, 65, 2048), (5, 1000, 32), (5, 1000, 33), (1, 4100, 32)])
def test_recurrence(hla, dtype, B, n, C):
    T = TYPES[dtype]
    gn, v, _ = glr_case(n + C, B, n, C, T, False)
    want, last, bound, last_bound = R.glr(v["x"], v["r"], v["g"], v["decay"], v["state"])
    x, r, g, decay = (on(v[k]) for k in ("x", "r", "g", "decay"))
    state, marks = on(v["state"]), torch.full((B, hla.hla_glr_marks(n), C), float("nan"), device=DEV)
    near("y", hla.hla_glr_forward(x, r, g, decay, state_in=state, state_out=state, marks=marks), want, bound)
    near("state", state, last, last_bound)
    dy, dl = randn(gn, B, n, C, T=T), randn(gn, B, C)
    want = R.glr_grad(v["x"], v["r"], v["g"], v["decay"], dy, v["state"], dl)
    back = torch.empty(B, C, device=DEV)
    got = hla.hla_glr_backward(x, r, g, decay, on(dy), marks, dstate_out=on(dl), dstate_in=back)
    for name, t in zip(("dx", "dr", "dg", "ddecay", "dstate"), got + (back,)):
        near(name, t, *want[name])
