"""The bounds of ffn_precision.py tell products in 32 bits from products of fewer: operands with 10 bits of mantissa, as tensor
cores take fp32, and with 13, are outside them."""
import pytest
import torch

import block_ref as R
import ffn_precision as P


@pytest.fixture(autouse=True, scope="module")
def one_thread():
    """(tests of several processes fork this one, which is safe while no pool of threads has been started)"""
    threads = torch.get_num_threads()
    torch.set_num_threads(1)
    yield
    torch.set_num_threads(threads)


def cut(t, bits):
    """Rounded to `bits` bits of mantissa."""
    m, e = torch.frexp(t.double())
    return torch.ldexp(torch.round(m * 2.0 ** (bits + 1)) / 2.0 ** (bits + 1), e)


def case(M, K, F):
    g = torch.Generator().manual_seed(M + K + F)
    randn = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    return randn(M, K), randn(2, F, K) * K ** -0.5, randn(M, F)


def grads(x, w, dout, bits):
    """(out, dx, dw) with the operands of every product cut."""
    c = (lambda t: cut(t, bits)) if bits else (lambda t: t.double())
    x, w = c(x), c(w)
    zg, zu = x @ w[0].t(), x @ w[1].t()
    a, slope = R.act_of(R.SILU, zg)
    dz = c(torch.cat([dout.double() * zu * slope, dout.double() * a], 1))
    return {"out": a * zu, "dx": dz @ w.reshape(-1, w.shape[2]), "dw": (dz.t() @ x).view(w.shape)}


@pytest.mark.parametrize("M,K,F", P.SIZES)
def test_fewer_bits_are_outside(M, K, F):
    x, w, dout = case(M, K, F)
    exact, bounds = grads(x, w, dout, None), P.bounds(M, K, F)
    for bits in (10, 13):
        got = grads(x, w, dout, bits)
        assert all(P.off(got[k], exact[k]) > 3 * bounds[k] for k in got), {k: (P.off(got[k], exact[k]), bounds[k]) for k in got}


@pytest.mark.parametrize("M,K,F", P.SIZES)
def test_sums_in_32_bits_are_inside(M, K, F):
    """The same by elementary operations in fp32, each sum formed one product after another."""
    x, w, dout = case(M, K, F)

    def product(a, b):  # a b^T
        sums = torch.zeros(a.shape[0], b.shape[0])
        for k in range(a.shape[1]):
            sums += a[:, k:k + 1] * b[:, k]
        return sums
    zg, zu = product(x, w[0]), product(x, w[1])
    a, slope = R.act_of(R.SILU, zg)
    dz = torch.cat([dout * zu * slope, dout * a], 1)
    got = {"out": a * zu, "dx": product(dz, w.reshape(-1, K).t()), "dw": product(dz.t(), x.t()).view(w.shape)}
    exact, bounds = grads(x, w, dout, None), P.bounds(M, K, F)
    assert all(P.off(got[k], exact[k]) <= bounds[k] for k in got), {k: (P.off(got[k], exact[k]), bounds[k]) for k in got}
