"""A host thread whose first CUDA call is one of the library's: the tensor maps of the tensor-core kernels are made by a call of
the driver, for which the thread has to have a context."""
import threading

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV, T = "cuda:0", torch.bfloat16


@pytest.fixture(scope="module")
def hla():
    from paper_2510_27258_gb300 import build
    build.build()
    from paper_2510_27258_gb300 import hla as binding
    return binding


def rand(*shape, scale=1.0, seed=1):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return (torch.randn(*shape, generator=g, device=DEV) * scale).to(T)


def second_order(hla):
    q, out = rand(1, 2, 256, 64, scale=0.1), torch.empty(1, 2, 256, 64, dtype=T, device=DEV)
    ws = hla.alloc_workspace(hla.hla2_workspace_bytes(1, 2, 256, 64, 64, 128, T), DEV)
    assert hla.hla2_forward_path(1, 2, 256, 64, 64)[0] == 1
    return lambda: hla.hla2_forward(q, q, q, out, workspace=ws)


def second_order_gradient(hla):
    q = rand(1, 2, 256, 64, scale=0.1)
    ws = hla.alloc_workspace(hla.hla2_backward_workspace_bytes(1, 2, 256, 64, 64, 64, T), DEV)
    assert hla.hla2_backward_path(1, 2, 256, 64, 64) == 1
    return lambda: hla.hla2_backward(q, q, q, q, workspace=ws)


def ahla(hla):
    q, out = rand(1, 2, 256, 64, scale=0.1), torch.empty(1, 2, 256, 64, dtype=T, device=DEV)
    ws = hla.alloc_workspace(hla.lib().ahla_workspace_bytes(1, 2, 256, 64, 64, 64, hla.HLA_BF16), DEV)
    assert hla.ahla_forward_path(1, 2, 256, 64, 64) == 1
    return lambda: hla.ahla_forward(q, q, q, out, workspace=ws)


def scan(hla):
    x, b, delta = rand(1, 300, 2, 64), rand(1, 300, 1, 64), rand(1, 300, 2)
    a, out = -torch.ones(2, device=DEV), torch.empty(1, 300, 2, 64, dtype=T, device=DEV)
    ws = hla.alloc_workspace(hla.hla_ssm_workspace_bytes(1, 300, 2, 64, 1, 64, T), DEV)
    assert hla.hla_ssm_forward_path(1, 300, 2, 64, 1, 64)[0] == 1
    return lambda: hla.hla_ssm_forward(x, delta, a, b, b, out, workspace=ws)


def feed_forward(hla, M):
    x, w, out = rand(M, 256), rand(2, 512, 256, scale=0.1), torch.empty(M, 512, dtype=T, device=DEV)
    ws = hla.alloc_workspace(hla.hla_ffn_workspace_bytes(M, 256, 512, T), DEV)
    return lambda: hla.hla_ffn_forward(x, w, out, workspace=ws)


def feed_forward_gradient(hla, M):
    x, w, d = rand(M, 256), rand(2, 512, 256, scale=0.1), rand(M, 512, seed=2)
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    ws = hla.alloc_workspace(hla.hla_ffn_backward_workspace_bytes(M, 256, 512, T), DEV)
    return lambda: hla.hla_ffn_backward(x, w, d, dx, dw, workspace=ws)


CALLS = {"second_order": second_order, "second_order_gradient": second_order_gradient, "ahla": ahla, "scan": scan,
         "feed_forward_few": lambda hla: feed_forward(hla, 16), "feed_forward": lambda hla: feed_forward(hla, 300),
         "feed_forward_gradient": lambda hla: feed_forward_gradient(hla, 300),
         "feed_forward_gradient_few": lambda hla: feed_forward_gradient(hla, 16)}


@pytest.mark.parametrize("name", CALLS)
def test_first_call_of_a_thread(hla, name):
    call, got = CALLS[name](hla), []
    tensors = lambda out: [t.clone() for t in (out if isinstance(out, tuple) else (out,))]  # noqa: E731
    want = tensors(call())
    torch.cuda.synchronize()

    def run():
        try:
            got.append(call())
        except Exception as e:  # noqa: BLE001
            got.append(repr(e))
    thread = threading.Thread(target=run)
    thread.start()
    thread.join()
    torch.cuda.synchronize()
    assert not isinstance(got[0], str), got[0]
    assert all(torch.equal(a, b) for a, b in zip(tensors(got[0]), want))
