"""The binding of the block's operators without a GPU: streams, GPUs and shapes (stand-ins of
test_binding_streams_cpu.py)."""
import pytest
import torch

import test_binding_streams_cpu as S
from test_binding_streams_cpu import Tensor, world  # noqa: F401

B, n, C, K, F = 2, 64, 24, 16, 32


class Like(Tensor):
    """A stand-in that makes tensors of its own kind."""
    world = None

    def new_empty(self, shape):
        return Like.world.empty(shape, dtype=self.dtype, device=self.device)


def T(*shape, dtype=torch.float32, index=S.GPU):
    return Like(torch.zeros(*shape, dtype=dtype), index)


def calls(E, **t):
    """name -> call(stream); t: tensors in the place of the right ones."""
    g = lambda name, *shape: t.get(name, T(*shape))  # noqa: E731
    x = T(B, n, C)
    return {
        "hla_glr_forward": lambda s: E.hla_glr_forward(x, g("r", B, n, C), g("g", B, n, C), g("decay", C),
                                                       state_in=g("state", B, C), marks=g("marks", B, 2, C), stream=s),
        "hla_glr_step": lambda s: E.hla_glr_step(T(B, C), T(B, C), T(B, C), g("decay", C), g("state", B, C), stream=s),
        "hla_glr_backward": lambda s: E.hla_glr_backward(x, x, x, g("decay", C), g("dout", B, n, C), g("marks", B, 2, C),
                                                         dstate_in=g("state", B, C), stream=s),
        "hla_block_norm_forward": lambda s: E.hla_block_norm_forward(x, g("y", B, n, C), g("gate", B, n, C),
                                                                     scale=g("scale", C), stream=s),
        "hla_block_norm_backward": lambda s: E.hla_block_norm_backward(x, g("y", B, n, C), g("gate", B, n, C), x,
                                                                       g("dh", B, n, C), w_pre=g("w_pre", C), stream=s),
        "hla_ffn_forward": lambda s: E.hla_ffn_forward(T(B, n, K), g("w", 2, F, K), stream=s),
        "hla_ffn_backward": lambda s: E.hla_ffn_backward(T(B, n, K), g("w", 2, F, K), g("dout", B, n, F), stream=s),
    }


NAMES = ["hla_glr_forward", "hla_glr_step", "hla_glr_backward", "hla_block_norm_forward", "hla_block_norm_backward",
         "hla_ffn_forward", "hla_ffn_backward"]


@pytest.fixture
def E(world, monkeypatch):  # noqa: F811
    from paper_2510_27258_gb300 import hla
    Like.world = world
    monkeypatch.setattr(hla, "hla_glr_marks", lambda k: -(-k // 32))
    return hla


@pytest.mark.parametrize("name", NAMES)
def test_memory_of_the_stream_that_runs(E, world, name):  # noqa: F811
    """Outputs and scratch are the memory of the stream that the call runs on, the current one or another."""
    calls(E)[name](None)
    assert world.made and all(stream == world.stream for _, stream in world.made)
    assert [S.handle_of(s) for _, s, _ in world.launched] == [world.stream]
    world.made.clear(), world.launched.clear()
    other = S.Stream(77)
    calls(E)[name](other)
    assert world.made and all(stream == 77 for _, stream in world.made)
    assert [S.handle_of(s) for _, s, _ in world.launched] == [77]


@pytest.mark.parametrize("name", NAMES)
def test_launched_on_the_gpu_of_the_tensors(E, world, name):  # noqa: F811
    world.device = S.GPU + 1
    calls(E)[name](None)
    assert [d for _, _, d in world.launched] == [S.GPU] and world.device == S.GPU + 1


@pytest.mark.parametrize("name,wrong", [
    ("hla_glr_forward", dict(r=T(B, n, C + 1))), ("hla_glr_forward", dict(decay=T(C + 1))),
    ("hla_glr_forward", dict(state=T(C, B))), ("hla_glr_forward", dict(marks=T(B, 3, C))),
    ("hla_glr_forward", dict(marks=T(2, B, C, dtype=torch.bfloat16))), ("hla_glr_forward", dict(g=T(n, B, C))),
    ("hla_glr_forward", dict(r=T(B, n, C, dtype=torch.bfloat16))), ("hla_glr_forward", dict(r=T(B, n, C, index=S.GPU + 1))),
    ("hla_glr_step", dict(state=T(C, B))), ("hla_glr_step", dict(decay=T(C, dtype=torch.bfloat16))),
    ("hla_glr_backward", dict(dout=T(B, n, C - 1))), ("hla_glr_backward", dict(marks=T(2, C, B))),
    ("hla_glr_backward", dict(state=T(B, C + 1))),
    ("hla_block_norm_forward", dict(y=T(B, n, C + 1))), ("hla_block_norm_forward", dict(gate=T(B * n, C))),
    ("hla_block_norm_forward", dict(scale=T(C - 1))), ("hla_block_norm_backward", dict(w_pre=T(C, dtype=torch.bfloat16))),
    ("hla_block_norm_backward", dict(dh=T(n, B, C))), ("hla_block_norm_backward", dict(dh=None)),
    ("hla_ffn_forward", dict(w=T(2, F, K + 1))), ("hla_ffn_forward", dict(w=T(F, K))),
    ("hla_ffn_forward", dict(w=T(2, F, K, dtype=torch.bfloat16))), ("hla_ffn_backward", dict(dout=T(B, n, K))),
    ("hla_ffn_backward", dict(dout=T(B * n, F)))])
def test_shapes_that_are_refused(E, world, name, wrong):  # noqa: F811
    with pytest.raises(ValueError):
        calls(E, **wrong)[name](None)
    assert not world.launched


def test_rows_of_a_projection(E, world):  # noqa: F811
    """Slices of wider rows are taken, rows that are not equally spaced are not."""
    wide = torch.zeros(B, n, 3 * C)
    x, r, g = (Like(wide[..., i * C:(i + 1) * C], S.GPU) for i in range(3))
    E.hla_glr_forward(x, r, g, T(C))
    E.hla_block_norm_forward(x, r, g)
    assert len(world.launched) == 2
    for bad in (torch.zeros(B, n + 1, C)[:, 1:], torch.zeros(B, C, n).transpose(1, 2)):
        with pytest.raises(ValueError):
            E.hla_glr_forward(Like(bad, S.GPU), r, g, T(C))
    with pytest.raises(ValueError):
        E.hla_block_norm_forward(T(2, 2, 2, C), T(2, 2, 2, C))
    with pytest.raises(TypeError):
        E.hla_ffn_forward(T(B, K, dtype=torch.float16), T(2, F, K, dtype=torch.float16))
