"""The fp32 feed-forward products keep 32 bits: the norm of their error, which products of fewer bits exceed by far."""
import pytest

import block_ref as R
import ffn_precision as P
from test_ffn_precision_cpu import case, grads

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def hla():
    from paper_2510_27258_gb300 import build
    build.build()
    from paper_2510_27258_gb300 import hla as binding
    return binding


@pytest.mark.parametrize("M,K,F", P.SIZES)
def test_norm_of_the_error(hla, M, K, F):
    x, w, dout = case(M, K, F)
    exact, bounds = grads(x, w, dout, None), P.bounds(M, K, F)
    x, w, dout = (t.to("cuda:0") for t in (x, w, dout))
    dx, dw = hla.hla_ffn_backward(x, w, dout, act=R.SILU)
    got = {"out": hla.hla_ffn_forward(x, w, act=R.SILU), "dx": dx, "dw": dw}
    off = {k: P.off(t, exact[k]) for k, t in got.items()}
    assert all(off[k] <= bounds[k] for k in off), (off, bounds)
