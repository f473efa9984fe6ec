"""The block's operators on four streams at once, each call with outputs and a workspace of its own: the same bits as alone."""
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


def rand(seed, *shape, T=torch.bfloat16, scale=1.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return (torch.randn(*shape, generator=g, device=DEV) * scale).to(T)


def recurrence(hla, B, n, C, T):
    x, r, g, dy = (rand(k, B, n, C, T=T) for k in range(4))
    decay, state = -torch.rand(C, device=DEV) - 0.01, torch.zeros(B, C, device=DEV)
    y, marks = torch.empty_like(x), torch.empty(B, hla.hla_glr_marks(n), C, device=DEV)
    grads = [torch.empty_like(x) for _ in range(3)]
    ws = hla.alloc_workspace(hla.hla_glr_backward_workspace_bytes(B, n, C, T), DEV)

    def call():
        hla.hla_glr_forward(x, r, g, decay, y, state_out=state, marks=marks)
        return [y, state, marks] + list(hla.hla_glr_backward(x, r, g, decay, dy, marks, *grads, workspace=ws))
    return call


def norms(hla, rows, C, T):
    x, y, gate, dx, dh = (rand(k, rows, C, T=T) for k in range(5))
    w = rand(9, C, T=T)
    out, grads = [torch.empty_like(x) for _ in range(2)], [torch.empty_like(x) for _ in range(3)]
    ws = hla.alloc_workspace(hla.hla_block_norm_backward_workspace_bytes(rows, C, T), DEV)
    kw = dict(w_post=w, scale=w, w_pre=w, dropout=0.1, seed=3)

    def call():
        hla.hla_block_norm_forward(x, y, gate, *out, **kw)
        return out + list(hla.hla_block_norm_backward(x, y, gate, dx, dh, *grads, workspace=ws, **kw))
    return call


def feed_forward(hla, M, K, F, T):
    x, w, d = rand(1, M, K, T=T), rand(2, 2, F, K, T=T, scale=K ** -0.5), rand(3, M, F, T=T)
    out, dx, dw = torch.empty_like(d), torch.empty_like(x), torch.empty_like(w)
    ws = [hla.alloc_workspace(size(M, K, F, T), DEV)
          for size in (hla.hla_ffn_workspace_bytes, hla.hla_ffn_backward_workspace_bytes)]

    def call():
        hla.hla_ffn_forward(x, w, out, workspace=ws[0])
        return [out] + list(hla.hla_ffn_backward(x, w, d, dx, dw, workspace=ws[1]))
    return call


def test_four_streams(hla):
    bf16, f32 = torch.bfloat16, torch.float32
    rows = [[recurrence(hla, 2, 3000, 264, bf16), feed_forward(hla, 16, 1024, 1408, bf16), norms(hla, 500, 2048, bf16)],
            [feed_forward(hla, 700, 512, 1032, bf16), recurrence(hla, 40, 70, 520, bf16), norms(hla, 64, 8192, f32)],
            [norms(hla, 900, 203, bf16), feed_forward(hla, 20, 512, 700, f32), recurrence(hla, 1, 5000, 66, f32)],
            [feed_forward(hla, 128, 512, 1032, bf16), feed_forward(hla, 200, 260, 500, f32), recurrence(hla, 1, 9000, 600, bf16)]]
    want = [[[t.clone() for t in call()] for call in row] for row in rows]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in rows]
    got = [[None] * len(row) for row in rows]
    for turn in range(20):
        for k in range(3):
            for i, s in enumerate(streams):
                with torch.cuda.stream(s):
                    got[i][k] = rows[i][k]()
    torch.cuda.synchronize()
    for i, row in enumerate(want):
        for k, tensors in enumerate(row):
            assert all(torch.equal(a, b) for a, b in zip(got[i][k], tensors)), (i, k)
