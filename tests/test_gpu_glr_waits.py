"""The gated recurrence where a wait between the blocks of a sequence runs out: one block of each cluster waits for more bytes
than come (set up on the host), so its waits end at their limit of 2 s, and with several turns the others' after it.  The
kernels finish, what is not known is NaN, the state among it, and the next call is as before."""
import pytest
import torch

from test_gpu_block import DEV, TYPES, gen, on, randn

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def hla():
    from paper_2510_27258_gb300 import build
    build.build()
    from paper_2510_27258_gb300 import hla as binding
    return binding


def known(got, want, name):
    """NaN or what it was without the wait: whether anything is NaN."""
    bad = torch.isnan(got)
    assert torch.equal(torch.where(bad, want, got), want), name
    return bool(bad.any())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,turns", [(700, 1), (9000, 2)])
def test_a_wait_that_runs_out(hla, monkeypatch, dtype, n, turns):
    B, C, T = 2, 66, TYPES[dtype]
    g = gen(n)
    x, r, gt, dy = (on(randn(g, B, n, C, T=T)) for _ in range(4))
    decay, first, dl = on(-torch.rand(C, generator=g) - 0.01), on(randn(g, B, C)), on(randn(g, B, C))
    ws = hla.alloc_workspace(hla.hla_glr_backward_workspace_bytes(B, n, C, T), DEV)

    def forward():
        state, marks = torch.zeros(B, C, device=DEV), torch.zeros(B, hla.hla_glr_marks(n), C, device=DEV)
        return hla.hla_glr_forward(x, r, gt, decay, state_in=first, state_out=state, marks=marks), state, marks

    def backward(marks):
        back = torch.zeros(B, C, device=DEV)
        return hla.hla_glr_backward(x, r, gt, decay, dy, marks, dstate_out=dl, dstate_in=back, workspace=ws) + (back,)
    want = forward()
    want_grads = backward(want[2])
    assert hla.hla_poll_error(ws) == hla.HLA_OK
    monkeypatch.setenv("HLA_TEST_SHORT_COPY", "1")
    y, state, marks = forward()
    grads = backward(want[2])
    assert hla.hla_poll_error(ws) == hla.HLA_ERR_TIMEOUT
    monkeypatch.delenv("HLA_TEST_SHORT_COPY")
    assert torch.isnan(state).all() and known(y, want[0], "y") and known(marks, want[2], "marks")
    assert torch.isnan(grads[4]).all() and torch.isnan(grads[3]).all()
    assert all([known(a, b, k) for a, b, k in zip(grads, want_grads, ("dx", "dr", "dg"))])
    if turns > 1:  # (from the second turn on)
        assert torch.isnan(y[:, -1]).all() and all(torch.isnan(t[:, 0]).all() for t in grads[:3])
    else:  # the other blocks have what they need
        assert not torch.isnan(y[:, -1]).any()
    again = forward()
    assert all(torch.equal(a, b) for a, b in zip(again, want))
    assert all(torch.equal(a, b) for a, b in zip(backward(again[2]), want_grads))
    assert hla.hla_poll_error(ws) == hla.HLA_OK
