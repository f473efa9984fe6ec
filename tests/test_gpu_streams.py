"""Calls on another stream than the current one, without a workspace of the caller's, while the current stream goes on
allocating and writing."""
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


def test_scratch_and_outputs_of_a_call_on_another_stream(hla):
    g = torch.Generator(device=DEV).manual_seed(3)
    rand = lambda *s: torch.randn(*s, generator=g, device=DEV).to(torch.bfloat16)  # noqa: E731
    B, n, H, P, N = 1, 3000, 4, 64, 64
    x, delta, b, c, w = rand(B, n, H, P), rand(B, n, H), rand(B, n, 1, N), rand(B, n, 1, N), rand(H * P, 4)
    a, wq = -torch.rand(H, generator=g, device=DEV), rand(P)
    q = rand(B, H, n, P) / 8
    assert hla.hla_ssm_forward_path(B, n, H, P, 1, N)[1] == 3
    calls = [lambda s: hla.hla_ssm_forward(x, delta, a, b, c, stream=s),
             lambda s: hla.hla_conv_backward(x.flatten(2), w, x.flatten(2), stream=s),
             lambda s: hla.hla_qk_norm_backward(x, x, wq, wq, None, None, q, q, stream=s),
             lambda s: hla.hla2_forward(q, q, q, stream=s), lambda s: hla.hla2_backward(q, q, q, q, stream=s),
             lambda s: hla.ahla_forward(q, q, q, stream=s)]
    tensors = lambda r: [t for t in (r if isinstance(r, tuple) else (r,)) if t is not None]  # noqa: E731
    want = [[t.clone() for t in tensors(call(None))] for call in calls]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for stream in (side, side.cuda_stream):
        got = []
        with torch.cuda.stream(side):
            torch.cuda._sleep(40_000_000)  # the calls' kernels run well after the calls return
        for call in calls:
            got.append(tensors(call(stream)))
            for size in (1 << 12, 1 << 18, 1 << 20, 1 << 22, 1 << 24):
                for _ in range(4):
                    torch.empty(size, dtype=torch.uint8, device=DEV).fill_(255)
        torch.cuda.current_stream().wait_stream(side)
        for p, r in zip(got, want):
            for t, u in zip(p, r):
                assert torch.equal(t, u)
