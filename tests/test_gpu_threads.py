"""Two host threads that call the same kernels with sizes that need different amounts of shared memory, each on a stream and
with a workspace of its own: how much a kernel may be launched with is a setting of the kernel that both share."""
import threading

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def hla():
    from paper_2510_27258_gb300 import build
    build.build()
    from paper_2510_27258_gb300 import hla as binding
    return binding


def both(calls, times):
    """Runs the calls side by side, each in a thread with a stream of its own: what they raised."""
    failed, start = [], threading.Barrier(len(calls))

    def run(call):
        with torch.cuda.stream(torch.cuda.Stream()):
            try:
                start.wait()
                for _ in range(times):
                    call()
            except Exception as e:  # noqa: BLE001
                failed.append(repr(e))
            torch.cuda.current_stream().synchronize()
    threads = [threading.Thread(target=run, args=(c,)) for c in calls]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    return failed


def feed_forward(hla, M):
    x, w = (torch.randn(*s, device=DEV).to(torch.bfloat16) for s in ((M, 256), (2, 512, 256)))
    out = torch.empty(M, 512, dtype=x.dtype, device=DEV)
    ws = hla.alloc_workspace(hla.hla_ffn_workspace_bytes(M, 256, 512, x.dtype), DEV)
    return lambda: hla.hla_ffn_forward(x, w, out, workspace=ws)


def norm_gradient(hla, C, T):
    x = torch.randn(8, C, device=DEV).to(T)
    ws = hla.alloc_workspace(hla.hla_block_norm_backward_workspace_bytes(8, C, T), DEV)
    dx, dy = torch.empty_like(x), torch.empty_like(x)
    return lambda: hla.hla_block_norm_backward(x, x, None, x, x, dx, dy, workspace=ws)


def second_order(hla, d, chunk):
    q = torch.randn(1, 2, 64, d, device=DEV) / 8
    ws, out = hla.alloc_workspace(hla.hla2_workspace_bytes(1, 2, 64, d, d, chunk, q.dtype), DEV), torch.empty_like(q)
    return lambda: hla.hla2_forward(q, q, q, out, chunk=chunk, workspace=ws)


def second_order_gradient(hla, d, chunk):
    q = torch.randn(1, 2, 64, d, device=DEV) / 8
    return lambda: hla.hla2_backward(q, q, q, q, normalized=False, chunk=chunk)


def third_order(hla, d):
    q = torch.randn(1, 2, 16, d, device=DEV) / 8
    return lambda: hla.hla3_forward(q, q, q, masked=False)


def ahla(hla, d):
    q = torch.randn(1, 2, 64, d, device=DEV) / 8
    return lambda: hla.ahla_forward(q, q, q)


def token(hla, d):
    q = torch.randn(1, 2, d, device=DEV) / 8
    state = torch.zeros(1, 2, hla.hla2_state_floats(d, d), device=DEV)
    return lambda: hla.hla2_step(q, q, q, state)


def ahla_token(hla, d):
    q = torch.randn(1, 2, d, device=DEV) / 8
    state = torch.zeros(1, 2, hla.ahla_state_floats(d, d), device=DEV)
    return lambda: hla.ahla_step(q, q, q, state)


PAIRS = {
    "feed_forward": lambda hla: (feed_forward(hla, 128), feed_forward(hla, 96)),
    "norm_gradient_bf16": lambda hla: (norm_gradient(hla, 2048, torch.bfloat16), norm_gradient(hla, 1160, torch.bfloat16)),
    "norm_gradient_f32": lambda hla: (norm_gradient(hla, 2048, torch.float32), norm_gradient(hla, 1040, torch.float32)),
    "norm_gradient_wide_rows": lambda hla: (norm_gradient(hla, 8192, torch.bfloat16), norm_gradient(hla, 4200, torch.bfloat16)),
    "second_order": lambda hla: (second_order(hla, 128, 64), second_order(hla, 128, 32)),
    "second_order_gradient": lambda hla: (second_order_gradient(hla, 64, 64), second_order_gradient(hla, 64, 32)),
    "third_order": lambda hla: (third_order(hla, 64), third_order(hla, 16)),
    "ahla": lambda hla: (ahla(hla, 128), ahla(hla, 64)),
    "token": lambda hla: (token(hla, 128), token(hla, 64)),
    "ahla_token": lambda hla: (ahla_token(hla, 128), ahla_token(hla, 64)),
}


@pytest.mark.parametrize("name", PAIRS)
def test_calls_of_two_threads(hla, name):
    calls = PAIRS[name](hla)
    for call in calls:
        call()
    torch.cuda.synchronize()
    assert both(calls, 2000) == []
