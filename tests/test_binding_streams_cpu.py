"""Which stream's memory and which GPU the binding's calls use, without a GPU: the library, the streams and the
allocator are stand-ins that write down what they are asked for."""
import pytest
import torch

GPU = 0


class Stream:
    def __init__(self, handle, device=GPU):
        self.cuda_stream, self.device_index = handle, device

    def __eq__(self, other):
        return self.cuda_stream == other.cuda_stream


class Tensor:
    """A CPU tensor that says it is on a GPU."""

    def __init__(self, t, index=GPU):
        self.t, self.index, self.recorded = t, index, []

    is_cuda = True
    dtype = property(lambda self: self.t.dtype)
    shape = property(lambda self: self.t.shape)
    device = property(lambda self: torch.device("cuda", self.index))

    def get_device(self):
        return self.index

    def record_stream(self, stream):
        self.recorded.append(stream.cuda_stream)

    def __getattr__(self, name):
        return getattr(self.t, name)


class World:
    """The current stream and device, and what was allocated and launched under which."""

    def __init__(self):
        self.stream, self.device, self.made, self.launched = 16, GPU, [], []

    def on(self, stream):
        world = self

        class On:
            def __enter__(self):
                self.kept, world.stream = world.stream, stream.cuda_stream

            def __exit__(self, *_):
                world.stream = self.kept
        return On()

    def use(self, index):
        world = self

        class Use:
            def __enter__(self):
                self.kept, world.device = world.device, index

            def __exit__(self, *_):
                world.device = self.kept
        return Use()

    def empty(self, *shape, dtype=None, device=None):
        t = Tensor(torch.zeros(*shape, dtype=dtype), torch.device(device).index)
        self.made.append((t, self.stream))
        return t

    def __getattr__(self, name):  # the library: sizes, and calls whose last argument is the stream
        def call(*args):
            if name.endswith("_bytes"):
                return 512
            if name.endswith("_floats"):
                return 8
            self.launched.append((name, args[-1], self.device))
            return 0
        return call


@pytest.fixture
def world(monkeypatch):
    from paper_2510_27258_gb300 import hla
    w = World()
    monkeypatch.setattr(hla, "lib", lambda: w)
    monkeypatch.setattr(hla, "_ptr", lambda t: None if t is None else t.data_ptr())
    monkeypatch.setattr(torch, "empty", w.empty)
    monkeypatch.setattr(torch, "empty_like", lambda t: w.empty(t.shape, dtype=t.dtype, device=t.device))
    monkeypatch.setattr(torch.cuda, "Stream", Stream)
    monkeypatch.setattr(torch.cuda, "ExternalStream", Stream)
    monkeypatch.setattr(torch.cuda, "default_stream", lambda d=None: Stream(0))
    monkeypatch.setattr(torch.cuda, "stream", w.on)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda d=None: Stream(w.stream))
    monkeypatch.setattr(torch.cuda, "current_device", lambda: w.device)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: w.device, raising=False)
    monkeypatch.setattr(torch.cuda, "device", w.use)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda i: w.stream, raising=False)
    return w


def calls(E, index=GPU):
    """name -> call(stream) for every call of the binding that takes a stream and makes outputs or scratch."""
    T = lambda *s: Tensor(torch.zeros(*s), index)  # noqa: E731
    x, w, h, tok = T(2, 8, 4, 16), T(64, 4), T(2, 4, 8, 16), T(2, 4, 16)
    ssm = (x, T(2, 8, 4), T(4), T(2, 8, 1, 16), T(2, 8, 1, 16))
    one = (tok, T(2, 4), T(4), T(2, 1, 16), T(2, 1, 16), T(2, 4, 16, 16))
    c = T(2, 8, 64)
    return {
        "hla_conv_forward": lambda s: E.hla_conv_forward(c, w, stream=s),
        "hla_conv_step": lambda s: E.hla_conv_step(T(2, 64), w, T(2, 3, 64), stream=s),
        "hla_conv_backward": lambda s: E.hla_conv_backward(c, w, c, T(64), stream=s),
        "hla_ssm_forward": lambda s: E.hla_ssm_forward(*ssm, stream=s),
        "hla_ssm_step": lambda s: E.hla_ssm_step(*one, stream=s),
        "hla_qk_norm_forward": lambda s: E.hla_qk_norm_forward(x, x, stream=s),
        "hla_qk_norm_backward": lambda s: E.hla_qk_norm_backward(x, x, T(16), T(16), None, None, h, h, stream=s),
        "hla2_forward": lambda s: E.hla2_forward(h, h, h, stream=s),
        "hla3_forward": lambda s: E.hla3_forward(h, h, h, stream=s),
        "hla2_forward_noalloc": lambda s: E.hla2_forward_noalloc(h, h, h, stream=s),
        "hla2_backward": lambda s: E.hla2_backward(h, h, h, h, stream=s),
        "ahla_forward": lambda s: E.ahla_forward(h, h, h, stream=s),
        "hla2_step": lambda s: E.hla2_step(tok, tok, tok, T(2, 4, 8), stream=s),
        "ahla_step": lambda s: E.ahla_step(tok, tok, tok, T(2, 4, 8), stream=s),
        "hla2_step_sde": lambda s: E.hla2_step_sde(tok, tok, tok, T(2, 4, 8), stream=s),
        "hla2_state_to_sde": lambda s: E.hla2_state_to_sde(T(2, 4, 8), 16, 16, stream=s),
    }


NAMES = ["hla_conv_forward", "hla_conv_step", "hla_conv_backward", "hla_ssm_forward", "hla_ssm_step",
         "hla_qk_norm_forward", "hla_qk_norm_backward", "hla2_forward", "hla3_forward", "hla2_forward_noalloc",
         "hla2_backward", "ahla_forward", "hla2_step", "ahla_step", "hla2_step_sde", "hla2_state_to_sde"]


def handle_of(v):
    return getattr(v, "value", v)


@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("given", ["object", "number"])
def test_memory_of_the_stream_that_runs(world, name, given):
    """What a call allocates belongs to the stream it runs on: scratch is released when the call returns, while
    that stream still uses it, and goes to the next allocation of the stream it belongs to.  Outputs that the
    caller takes to the current stream are kept for that one."""
    from paper_2510_27258_gb300 import hla as E
    result = calls(E)[name](Stream(32) if given == "object" else 32)
    assert [(n, handle_of(s)) for n, s, _ in world.launched] == [(name, 32)]
    assert world.made and all(stream == 32 for _, stream in world.made)
    outputs = [t for t in (result if isinstance(result, tuple) else (result,)) if t is not None]
    assert outputs and all(t.recorded == [16] for t in outputs)


@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("stream", [None, 16])
def test_memory_of_the_current_stream(world, name, stream):
    from paper_2510_27258_gb300 import hla as E
    calls(E)[name](None if stream is None else Stream(stream))
    assert [(n, handle_of(s)) for n, s, _ in world.launched] == [(name, 16)]
    assert world.made and all(stream == 16 and not t.recorded for t, stream in world.made)


def test_default_stream_by_its_numbers(world):
    from paper_2510_27258_gb300 import hla as E
    for number in (0, 1):
        world.made.clear()
        calls(E)["hla_ssm_forward"](number)
        assert world.made and all(stream == 0 for _, stream in world.made)


def test_a_stream_of_another_gpu(world):
    from paper_2510_27258_gb300 import hla as E
    with pytest.raises(ValueError):
        calls(E)["hla_conv_forward"](Stream(32, device=1))
    assert not world.launched


@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("index", [0, 1])
def test_launched_on_the_gpu_of_the_tensors(world, name, index):
    """Whichever GPU is the current one, a call is made with its tensors' one, and leaves the current one as it was."""
    from paper_2510_27258_gb300 import hla as E
    calls(E, index)[name](None)
    assert [(n, device) for n, _, device in world.launched] == [(name, index)]
    assert world.device == 0 and all(t.index == index for t, _ in world.made)
