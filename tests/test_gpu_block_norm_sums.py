"""The weights' gradients of the block norms through the C entry point, which takes a pointer for each whether or not its
norm is on: zeros where it is off."""
import ctypes

import pytest
import torch

import block_ref as R
from test_gpu_block import DEV, TYPES, near, norm_case, on, randn

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def hla():
    from paper_2510_27258_gb300 import build
    build.build()
    from paper_2510_27258_gb300 import hla as binding
    return binding


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("post,pre", [(0, 1), (1, 0), (0, 0), (1, 1)])
@pytest.mark.parametrize("rows,C", [(37, 24), (9, 203), (64, 260), (40, 2048), (11, 2047), (5, 4104), (3, 8192), (3, 8200)])
def test_sums_of_norms_that_are_off(hla, dtype, post, pre, rows, C):
    T = TYPES[dtype]
    g, v, kw, _ = norm_case(rows + C, rows, C, T, dropout=0.1, post=bool(post), pre=bool(pre))
    dx_out, dh = randn(g, rows, C, T=T), randn(g, rows, C, T=T)
    want = R.norm(**v, dx_out=dx_out, dh=dh, **kw)
    t = {k: on(x) for k, x in (*v.items(), ("dx_out", dx_out), ("dh", dh))}
    out = [torch.empty(rows, C, dtype=T, device=DEV) for _ in range(3)]
    sums = {k: torch.full((C,), float("nan"), device=DEV) for k in ("dw_post", "dscale", "dw_pre")}
    ws = hla.alloc_workspace(hla.hla_block_norm_backward_workspace_bytes(rows, C, T), DEV)
    code = hla.lib().hla_block_norm_backward(
        *(t[k].data_ptr() for k in ("x", "y", "gate", "w_post", "scale", "w_pre", "dx_out", "dh")),
        *(o.data_ptr() for o in out), *(s.data_ptr() for s in sums.values()), 1 if dtype == "bf16" else 0, rows, C,
        *[C] * 8, post, pre, kw["act"], ctypes.c_float(kw["alpha"]), ctypes.c_float(kw["eps"]),
        ctypes.c_double(kw["dropout"]), kw["seed"], kw["offset"], ws.data_ptr(), ws.numel(),
        torch.cuda.current_stream().cuda_stream)
    assert code == hla.HLA_OK
    near("dscale", sums["dscale"], *want["dscale"])
    for name, norm in (("dw_post", post), ("dw_pre", pre)):
        if norm:
            near(name, sums[name], *want[name])
        else:
            assert torch.equal(sums[name], torch.zeros_like(sums[name])), name
    for name, o in zip(("dx", "dy", "dgate"), out):
        near(name, o, *want[name])
