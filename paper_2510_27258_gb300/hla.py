"""Thin ctypes binding of the HLA C ABI (include/hla.h).

Every function has the name of the C entry point it calls and does argument
marshalling only: it checks tensor shapes/devices, takes raw pointers and the
current CUDA stream from PyTorch, and calls the library.  All arithmetic runs in
the CUDA kernels of ``libhla.so``.  If the library is missing the calls raise;
there is no fallback.
"""
from __future__ import annotations

import ctypes
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libhla.so")

HLA_OK, HLA_ERR_INVALID_ARGUMENT, HLA_ERR_UNSUPPORTED, HLA_ERR_CUDA, HLA_ERR_TIMEOUT, HLA_ERR_WORKSPACE = range(6)
HLA_F32, HLA_BF16 = 0, 1

# every symbol include/hla.h declares
EXPORTS = ("hla_status_string", "hla_last_error", "hla2_state_floats", "hla2_workspace_bytes", "hla2_forward",
           "hla2_forward_path", "hla2_step", "hla3_state_floats", "hla3_workspace_bytes", "hla3_forward",
           "hla3_forward_path", "hla2_backward_path",
           "hla2_forward_noalloc", "hla_poll_error_noalloc", "hla_poll_error", "hla2_sde_state_floats",
           "hla2_state_to_sde", "hla2_step_sde", "ahla_state_floats", "ahla_workspace_bytes", "ahla_forward",
           "ahla_step", "hla2_backward_workspace_bytes", "hla2_backward", "ahla_forward_path",
           "hla_conv_forward", "hla_conv_step", "hla_conv_backward_workspace_bytes", "hla_conv_backward",
           "hla_ssm_workspace_bytes", "hla_ssm_forward", "hla_ssm_forward_path", "hla_ssm_step", "hla_qk_norm_forward",
           "hla_qk_norm_backward_workspace_bytes", "hla_qk_norm_backward")

_lib = None


class HLAError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        detail = lib().hla_last_error().decode(errors="replace")
        super().__init__("%s: %s%s" % (where, hla_status_string(code), (" (" + detail + ")") if detail else ""))


def lib():
    """Load libhla.so (built by ``paper_2510_27258_gb300.build``); raise if it is missing."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError("libhla.so is not built: run `python -c \"import __graft_entry__ as g; g.build()\"` "
                               "or `python paper_2510_27258_gb300/build.py`")
        L = ctypes.CDLL(LIB_PATH)
        vp, i, f, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_size_t
        L.hla_status_string.argtypes = [i]
        L.hla_status_string.restype = ctypes.c_char_p
        L.hla_last_error.argtypes = []
        L.hla_last_error.restype = ctypes.c_char_p
        for name in ("hla2_state_floats", "hla3_state_floats"):
            getattr(L, name).argtypes = [i, i]
            getattr(L, name).restype = sz
        L.ahla_state_floats.argtypes = [i, i]
        L.ahla_state_floats.restype = sz
        L.ahla_forward.argtypes = [vp, vp, vp, vp, i, i, i, i, i, i, i, f, i, vp, vp, vp, sz, vp]
        L.ahla_forward.restype = i
        L.ahla_step.argtypes = [vp, vp, vp, vp, i, i, i, i, i, i, f, vp, vp]
        L.ahla_step.restype = i
        L.ahla_forward_path.argtypes = [i, i, i, i, i, i, i, i, i, i]
        L.ahla_forward_path.restype = i
        L.hla2_backward_path.argtypes = [i, i, i, i, i, i, i, i]
        L.hla2_backward_path.restype = i
        L.hla2_backward.argtypes = [vp, vp, vp, vp, vp, vp, vp, i, i, i, i, i, i, i, f, i, vp, sz, vp]
        L.hla2_backward.restype = i
        for name in ("hla2_workspace_bytes", "hla3_workspace_bytes", "ahla_workspace_bytes",
                     "hla2_backward_workspace_bytes"):
            getattr(L, name).argtypes = [i, i, i, i, i, i, i]
            getattr(L, name).restype = sz
        for name in ("hla2_forward", "hla3_forward"):
            getattr(L, name).argtypes = [vp, vp, vp, vp, i, i, i, i, i, i, i, i, f, i, vp, vp, vp, sz, vp]
            getattr(L, name).restype = i
        L.hla2_forward_noalloc.argtypes = [vp, vp, vp, vp, i, i, i, i, i, i, i, i, f, i, vp, vp]
        L.hla2_forward_noalloc.restype = i
        for name in ("hla2_forward_path", "hla3_forward_path"):
            getattr(L, name).argtypes = [i, i, i, i, i, i, i, i, i, i, i, ctypes.POINTER(i)]
            getattr(L, name).restype = i
        L.hla2_step.argtypes = [vp, vp, vp, vp, i, i, i, i, i, i, i, f, vp, vp]
        L.hla2_step.restype = i
        L.hla_poll_error.argtypes = [vp, vp]
        L.hla_poll_error.restype = i
        L.hla_poll_error_noalloc.argtypes = [vp]
        L.hla_poll_error_noalloc.restype = i
        L.hla2_sde_state_floats.argtypes = [i, i]
        L.hla2_sde_state_floats.restype = sz
        L.hla2_state_to_sde.argtypes = [vp, vp, i, i, i, i, vp]
        L.hla2_state_to_sde.restype = i
        L.hla2_step_sde.argtypes = [vp, vp, vp, vp, i, i, i, i, i, i, f, vp, vp]
        L.hla2_step_sde.restype = i
        ll = ctypes.c_longlong
        L.hla_conv_forward.argtypes = [vp] * 4 + [i] * 5 + [ll, ll, i] + [vp] * 4
        L.hla_conv_step.argtypes = [vp] * 4 + [i] * 4 + [ll, ll, i] + [vp] * 2
        L.hla_conv_backward_workspace_bytes.argtypes = [i] * 5
        L.hla_conv_backward.argtypes = [vp] * 7 + [i] * 5 + [ll] * 3 + [i, vp, vp, sz, vp]
        L.hla_ssm_workspace_bytes.argtypes = [i] * 7
        L.hla_ssm_forward.argtypes = [vp] * 8 + [i] * 7 + [ll] * 5 + [i] + [vp] * 4 + [sz, vp]
        L.hla_ssm_step.argtypes = [vp] * 8 + [i] * 6 + [ll] * 5 + [i, vp, vp]
        L.hla_qk_norm_forward.argtypes = [vp] * 9 + [i] * 8 + [ll, ll, i, i, f, vp]
        L.hla_qk_norm_backward_workspace_bytes.argtypes = [i] * 6
        L.hla_qk_norm_backward.argtypes = [vp] * 13 + [i] * 8 + [ll] * 4 + [i, i, f, vp, sz, vp]
        L.hla_ssm_forward_path.argtypes = [i] * 8 + [ctypes.POINTER(i)]
        L.hla_ssm_forward_path.restype = i
        for name in ("hla_conv_backward_workspace_bytes", "hla_ssm_workspace_bytes",
                     "hla_qk_norm_backward_workspace_bytes"):
            getattr(L, name).restype = sz
        for name in ("hla_conv_forward", "hla_conv_step", "hla_conv_backward", "hla_ssm_forward", "hla_ssm_step",
                     "hla_qk_norm_forward", "hla_qk_norm_backward"):
            getattr(L, name).restype = i
        _lib = L
    return _lib


def hla_status_string(code: int) -> str:
    return lib().hla_status_string(int(code)).decode()


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.bfloat16:
        return HLA_BF16
    if t.dtype == torch.float32:
        return HLA_F32
    raise TypeError("HLA tokens must be bfloat16 or float32, got %s" % t.dtype)


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(stream):
    if stream is None:
        stream = torch.cuda.current_stream()
    return ctypes.c_void_p(stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream))


def _check(code: int, where: str):
    if code != HLA_OK:
        raise HLAError(code, where)


def hla2_state_floats(d: int, dv: int) -> int:
    return int(lib().hla2_state_floats(d, dv))


def hla3_state_floats(d: int, dv: int) -> int:
    return int(lib().hla3_state_floats(d, dv))


def hla2_workspace_bytes(B, H, n, d, dv, chunk, dtype) -> int:
    code = dtype if isinstance(dtype, int) else (HLA_BF16 if dtype == torch.bfloat16 else HLA_F32)
    return int(lib().hla2_workspace_bytes(B, H, n, d, dv, chunk, code))


def hla3_workspace_bytes(B, H, n, d, dv, chunk, dtype) -> int:
    code = dtype if isinstance(dtype, int) else (HLA_BF16 if dtype == torch.bfloat16 else HLA_F32)
    return int(lib().hla3_workspace_bytes(B, H, n, d, dv, chunk, code))


def alloc_workspace(nbytes: int, device) -> torch.Tensor:
    """Caller-owned scratch for the forward calls (256-byte aligned by the allocator)."""
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)


def _on(stream, index):
    """(handle, side): the stream to run on, the caller's or GPU `index`'s current one; `side` is that stream as
    an object where it is not the current one, else None."""
    current = torch._C._cuda_getCurrentRawStream(index)  # current_stream(index).cuda_stream without the object
    if stream is None:
        return current, None
    handle = stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)
    if getattr(stream, "device_index", index) != index:
        raise ValueError("the stream is cuda:%d's, the tensors are on cuda:%d" % (stream.device_index, index))
    if handle == current:
        return handle, None
    if not isinstance(stream, torch.cuda.Stream):
        # (0 and 1 both name the default stream)
        stream = torch.cuda.ExternalStream(handle, index) if handle > 1 else torch.cuda.default_stream(index)
    return handle, stream


def _index(t):
    """The GPU a tensor is on."""
    index = t.get_device()
    return index if index >= 0 else torch.cuda.current_device()


def _entry(name, index):
    """The entry point, made with GPU `index`, where its tensors and its stream are, as the current one."""
    fn = getattr(lib(), name)
    if torch._C._cuda_getDevice() == index:
        return fn

    def there(*args):
        with torch.cuda.device(index):
            return fn(*args)
    return there


def _empty(shape, dtype, device, side):
    """A new output tensor.  Where the call runs on another stream than the current one it is that stream's memory
    (what is the current stream's may still be in use there), and is kept for the current one, where the caller may
    read it, when it is released."""
    if side is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(side):
        t = torch.empty(shape, dtype=dtype, device=device)
    t.record_stream(torch.cuda.current_stream(device))
    return t


def _workspace(nbytes, device, side):
    """alloc_workspace for the stream the call runs on: it is released when the call returns, and then goes to work
    that comes later on that stream, not on the current one."""
    if side is None:
        return alloc_workspace(nbytes, device)
    with torch.cuda.stream(side):
        return alloc_workspace(nbytes, device)


def _forward(fn_name, ws_fn, q, k, v, out, masked, normalized, eps, chunk, state_in, state_out, workspace, stream):
    if q.dim() != 4:
        raise ValueError("q, k, v must be [B, H, n, d]")
    B, H, n, d = q.shape
    dv = v.shape[-1]
    if k.shape != q.shape or v.shape[:3] != q.shape[:3]:
        raise ValueError("shape mismatch: q %s k %s v %s" % (tuple(q.shape), tuple(k.shape), tuple(v.shape)))
    for t in (q, k, v):
        if not t.is_cuda or not t.is_contiguous() or t.dtype != q.dtype:
            raise ValueError("q, k, v must be contiguous CUDA tensors of one dtype")
    index = _index(q)
    handle, side = _on(stream, index)
    if out is None:
        out = _empty((B, H, n, dv), q.dtype, q.device, side)
    dt = _dtype_code(q)
    if workspace is None:
        workspace = _workspace(ws_fn(B, H, n, d, dv, chunk, dt), q.device, side)
    _check(_entry(fn_name, index)(
        _ptr(q), _ptr(k), _ptr(v), _ptr(out), dt, B, H, n, d, dv, int(masked), int(normalized),
        float(eps), int(chunk), _ptr(state_in), _ptr(state_out), _ptr(workspace),
        workspace.numel() * workspace.element_size(), handle), fn_name)
    return out


def hla2_forward(q, k, v, out=None, *, masked=True, normalized=False, eps=1e-6, chunk=128, state_in=None,
                 state_out=None, workspace=None, stream=None):
    """Second-order HLA forward (include/hla.h: hla2_forward). Returns ``out``."""
    return _forward("hla2_forward", hla2_workspace_bytes, q, k, v, out, masked, normalized, eps, chunk, state_in,
                    state_out, workspace, stream)


def hla3_forward(q, k, v, out=None, *, masked=True, normalized=False, eps=1e-6, chunk=32, state_in=None,
                 state_out=None, workspace=None, stream=None):
    """Third-order HLA forward (include/hla.h: hla3_forward). Returns ``out``."""
    return _forward("hla3_forward", hla3_workspace_bytes, q, k, v, out, masked, normalized, eps, chunk, state_in,
                    state_out, workspace, stream)


def hla2_forward_noalloc(q, k, v, out=None, *, masked=True, normalized=False, eps=1e-6, chunk=128, state_in=None,
                         stream=None):
    """hla2_forward without a workspace, for callers that cannot allocate device
    memory; the library's own 16 MiB device array serves as scratch (include/hla.h:
    hla2_forward_noalloc).  Returns ``out``."""
    B, H, n, d = q.shape
    dv = v.shape[-1]
    index = _index(q)
    handle, side = _on(stream, index)
    if out is None:
        out = _empty((B, H, n, dv), q.dtype, q.device, side)
    _check(_entry("hla2_forward_noalloc", index)(
        _ptr(q), _ptr(k), _ptr(v), _ptr(out), _dtype_code(q), B, H, n, d, dv,
        int(masked), int(normalized), float(eps), int(chunk), _ptr(state_in), handle), "hla2_forward_noalloc")
    return out


def hla2_forward_path(B, H, n, d, dv, *, masked=True, normalized=False, chunk=128, dtype=torch.bfloat16,
                      has_state_in=False, has_state_out=False):
    """(path, launches) that hla2_forward takes: path 1 = fused tcgen05 kernel, 0 = generic, -1 = unsupported."""
    code = dtype if isinstance(dtype, int) else (HLA_BF16 if dtype == torch.bfloat16 else HLA_F32)
    n_launch = ctypes.c_int(0)
    path = lib().hla2_forward_path(B, H, n, d, dv, int(masked), int(normalized), int(chunk), code,
                                   int(has_state_in), int(has_state_out), ctypes.byref(n_launch))
    return int(path), int(n_launch.value)


def hla3_forward_path(B, H, n, d, dv, *, masked=True, normalized=False, chunk=32, dtype=torch.float32,
                      has_state_in=False, has_state_out=False):
    """(path, launches) that hla3_forward takes: path 2 = tensor-core kernels, 1 = chunk-parallel fp32
    kernels, 0 = serial kernel, -1 = unsupported."""
    code = dtype if isinstance(dtype, int) else (HLA_BF16 if dtype == torch.bfloat16 else HLA_F32)
    n_launch = ctypes.c_int(0)
    path = lib().hla3_forward_path(B, H, n, d, dv, int(masked), int(normalized), int(chunk), code,
                                   int(has_state_in), int(has_state_out), ctypes.byref(n_launch))
    return int(path), int(n_launch.value)


def hla2_step(q, k, v, state, out=None, *, masked=True, normalized=False, eps=1e-6, stream=None):
    """One decode step for every head (include/hla.h: hla2_step); ``state`` is updated in place.

    q, k: [B, H, d]; v: [B, H, dv]; state: fp32 [B, H, hla2_state_floats(d, dv)].
    """
    B, H, d = q.shape
    dv = v.shape[-1]
    index = _index(q)
    handle, side = _on(stream, index)
    if out is None:
        out = _empty((B, H, dv), q.dtype, q.device, side)
    if state.dtype != torch.float32 or not state.is_contiguous():
        raise ValueError("state must be contiguous float32")
    _check(_entry("hla2_step", index)(
        _ptr(q), _ptr(k), _ptr(v), _ptr(out), _dtype_code(q), B, H, d, dv, int(masked),
        int(normalized), float(eps), _ptr(state), handle), "hla2_step")
    return out


def hla2_backward_workspace_bytes(B, H, n, d, dv, chunk, dtype) -> int:
    code = dtype if isinstance(dtype, int) else (HLA_BF16 if dtype == torch.bfloat16 else HLA_F32)
    return int(lib().hla2_backward_workspace_bytes(B, H, n, d, dv, chunk, code))


def hla2_backward(q, k, v, dout, *, normalized=False, eps=1e-6, chunk=64, workspace=None, stream=None):
    """Gradients (dq, dk, dv) of sum(dout * out) for the masked second-order forward
    (include/hla.h: hla2_backward)."""
    B, H, n, d = q.shape
    dv = v.shape[-1]
    for t in (q, k, v, dout):
        if not t.is_cuda or not t.is_contiguous() or t.dtype != q.dtype:
            raise ValueError("q, k, v, dout must be contiguous CUDA tensors of one dtype")
    dt = _dtype_code(q)
    index = _index(q)
    handle, side = _on(stream, index)
    gq, gk, gv = (_empty(t.shape, t.dtype, t.device, side) for t in (q, k, v))
    if workspace is None:
        workspace = _workspace(hla2_backward_workspace_bytes(B, H, n, d, dv, chunk, dt), q.device, side)
    _check(_entry("hla2_backward", index)(
        _ptr(q), _ptr(k), _ptr(v), _ptr(dout), _ptr(gq), _ptr(gk), _ptr(gv), dt, B, H, n, d,
        dv, int(normalized), float(eps), int(chunk), _ptr(workspace), workspace.numel() * workspace.element_size(),
        handle), "hla2_backward")
    return gq, gk, gv


def ahla_state_floats(d: int, dv: int) -> int:
    return int(lib().ahla_state_floats(d, dv))


def ahla_workspace_bytes(B, H, n, d, dv, chunk, dtype) -> int:
    code = dtype if isinstance(dtype, int) else (HLA_BF16 if dtype == torch.bfloat16 else HLA_F32)
    return int(lib().ahla_workspace_bytes(B, H, n, d, dv, chunk, code))


def ahla_forward(q, k, v, out=None, *, normalized=False, eps=1e-6, chunk=64, state_in=None, state_out=None,
                 workspace=None, stream=None):
    """AHLA forward (include/hla.h: ahla_forward). Returns ``out``."""
    if q.dim() != 4:
        raise ValueError("q, k, v must be [B, H, n, d]")
    B, H, n, d = q.shape
    dv = v.shape[-1]
    for t in (q, k, v):
        if not t.is_cuda or not t.is_contiguous() or t.dtype != q.dtype:
            raise ValueError("q, k, v must be contiguous CUDA tensors of one dtype")
    index = _index(q)
    handle, side = _on(stream, index)
    if out is None:
        out = _empty((B, H, n, dv), q.dtype, q.device, side)
    dt = _dtype_code(q)
    if workspace is None:
        workspace = _workspace(ahla_workspace_bytes(B, H, n, d, dv, chunk, dt), q.device, side)
    _check(_entry("ahla_forward", index)(
        _ptr(q), _ptr(k), _ptr(v), _ptr(out), dt, B, H, n, d, dv, int(normalized), float(eps),
        int(chunk), _ptr(state_in), _ptr(state_out), _ptr(workspace), workspace.numel() * workspace.element_size(),
        handle), "ahla_forward")
    return out


def hla2_backward_path(B, H, n, d, dv, *, normalized=False, chunk=64, dtype=torch.bfloat16) -> int:
    """1 if hla2_backward runs on the tensor cores for these arguments, 0 on the fp32 kernels, -1 unsupported."""
    code = dtype if isinstance(dtype, int) else (HLA_BF16 if dtype == torch.bfloat16 else HLA_F32)
    return int(lib().hla2_backward_path(B, H, n, d, dv, int(normalized), int(chunk), code))


def ahla_forward_path(B, H, n, d, dv, *, normalized=False, chunk=64, dtype=torch.bfloat16, has_state_in=False,
                      has_state_out=False) -> int:
    """1 if ahla_forward runs on the tensor cores for these arguments, 0 on the fp32 kernels, -1 unsupported."""
    code = dtype if isinstance(dtype, int) else (HLA_BF16 if dtype == torch.bfloat16 else HLA_F32)
    return int(lib().ahla_forward_path(B, H, n, d, dv, int(normalized), int(chunk), code, int(has_state_in),
                                       int(has_state_out)))


def ahla_step(q, k, v, state, out=None, *, normalized=False, eps=1e-6, stream=None):
    """One AHLA decode step for every head (include/hla.h: ahla_step); ``state`` is updated in place."""
    B, H, d = q.shape
    dv = v.shape[-1]
    index = _index(q)
    handle, side = _on(stream, index)
    if out is None:
        out = _empty((B, H, dv), q.dtype, q.device, side)
    if state.dtype != torch.float32 or not state.is_contiguous():
        raise ValueError("state must be contiguous float32")
    _check(_entry("ahla_step", index)(
        _ptr(q), _ptr(k), _ptr(v), _ptr(out), _dtype_code(q), B, H, d, dv, int(normalized),
        float(eps), _ptr(state), handle), "ahla_step")
    return out


def hla2_sde_state_floats(d: int, dv: int) -> int:
    return int(lib().hla2_sde_state_floats(d, dv))


def hla2_state_to_sde(state, d: int, dv: int, sde=None, *, stream=None):
    """(S, C, m, G, h) tuples [B, H, hla2_state_floats(d, dv)] -> (S, D, e) states
    [B, H, hla2_sde_state_floats(d, dv)] (include/hla.h: hla2_state_to_sde)."""
    B, H = state.shape[:2]
    index = _index(state)
    handle, side = _on(stream, index)
    if sde is None:
        sde = _empty((B, H, hla2_sde_state_floats(d, dv)), torch.float32, state.device, side)
    _check(_entry("hla2_state_to_sde", index)(
        _ptr(state), _ptr(sde), B, H, d, dv, handle), "hla2_state_to_sde")
    return sde


def hla2_step_sde(q, k, v, sde, out=None, *, normalized=False, eps=1e-6, stream=None):
    """One decode step of the masked operator on (S, D, e) states, updated in place
    (include/hla.h: hla2_step_sde).  q, k: [B, H, d]; v: [B, H, dv]."""
    B, H, d = q.shape
    dv = v.shape[-1]
    index = _index(q)
    handle, side = _on(stream, index)
    if out is None:
        out = _empty((B, H, dv), q.dtype, q.device, side)
    if sde.dtype != torch.float32 or not sde.is_contiguous():
        raise ValueError("state must be contiguous float32")
    _check(_entry("hla2_step_sde", index)(
        _ptr(q), _ptr(k), _ptr(v), _ptr(out), _dtype_code(q), B, H, d, dv, int(normalized),
        float(eps), _ptr(sde), handle), "hla2_step_sde")
    return out


def hla_poll_error_noalloc(stream=None) -> int:
    """Synchronise and read the device-side error flag of the library's own scratch array, used by
    hla2_forward_noalloc (include/hla.h: hla_poll_error_noalloc)."""
    return int(lib().hla_poll_error_noalloc(_stream(stream)))


def hla_poll_error(workspace, stream=None) -> int:
    """Synchronise and read the device-side error flag of a workspace (include/hla.h: hla_poll_error)."""
    return int(lib().hla_poll_error(_ptr(workspace), _stream(stream)))


# ------------------------------------------------------------------------------------------------
# the operators around the mixers: short convolution, selective scan, q/k norm with rotation
# ------------------------------------------------------------------------------------------------

_TYPE_CODES = {torch.bfloat16: HLA_BF16, torch.float32: HLA_F32}


def _type_code(dtype) -> int:
    code = _TYPE_CODES.get(dtype)
    if code is not None:
        return code
    if isinstance(dtype, int):
        return dtype
    raise TypeError("tokens must be bfloat16 or float32, got %s" % dtype)


def _same_order(got, want):
    """Whether contiguous tensors of two shapes hold the same elements in the same order as far as shapes can tell:
    one of them is the other with neighbouring dimensions taken together."""
    def steps(shape):  # elements from one index of a dimension to the next, and of all
        seen, step = {1}, 1
        for size in reversed(shape):
            step *= size
            seen.add(step)
        return step, seen
    (count, a), (other, b) = steps(got), steps(want)
    return count == other and (count == 0 or a <= b or b <= a)


def _flat(name, t, count, dtype, index):
    """Address of a contiguous tensor of one dimension and `count` elements on GPU `index` (None stays None)."""
    if t is None:
        return None
    if t.numel() != count or t.dtype is not dtype or t.get_device() != index or not t.is_contiguous():
        raise ValueError("%s must be a contiguous %s tensor of %d elements on cuda:%d, got %s %s on %s"
                         % (name, dtype, count, index, t.dtype, tuple(t.shape), t.device))
    return t.data_ptr()


def _shaped(name, t, shape, dtype, index):
    """Address of a contiguous tensor of a shape, or of one that holds it in the same order, on GPU `index` (None
    stays None)."""
    if t is None:
        return None
    if t.shape != shape and not _same_order(t.shape, shape) or (
            t.dtype is not dtype or t.get_device() != index or not t.is_contiguous()):
        raise ValueError("%s must be a contiguous %s tensor %s on cuda:%d, got %s %s on %s"
                         % (name, dtype, tuple(shape), index, t.dtype, tuple(t.shape), t.device))
    return t.data_ptr()


def _rows(name, t, shape, inner, dtype, index, own=False):
    """Row stride (elements) of a token tensor on GPU `index`: `shape` with rows of strides `inner`.  own: of the
    tensor that shape, dtype and index were taken from."""
    if own or (t.dtype is dtype and t.get_device() == index and t.shape == shape):
        st, lead = t.stride(), len(shape) - len(inner)
        if st[lead:] == inner:
            rows = shape[lead - 1]
            if rows > 1:
                if lead == 1 or shape[0] == 1 or st[0] == rows * st[1]:
                    return st[lead - 1]
            elif lead == 2 and rows == 1 and shape[0] > 1:
                return st[0]
            else:
                return inner[0] * shape[lead]
    else:
        lead = len(shape) - len(inner)
    return _row_stride(name, t, lead, shape, dtype, torch.device("cuda", index))


def _row_stride(name, t, lead, shape, dtype, device):
    """Row stride (elements) of a token tensor of `lead` leading dimensions whose rows are contiguous and
    equally spaced; raises where they are not."""
    if t.shape != shape or t.dtype != dtype or t.device != device:
        raise ValueError("%s must be a %s tensor %s on %s, got %s %s on %s"
                         % (name, dtype, tuple(shape), device, t.dtype, tuple(t.shape), t.device))
    st, width = t.stride(), 1
    for j in range(len(shape) - 1, lead - 1, -1):
        if st[j] != width and shape[j] > 1:
            raise ValueError("%s: the elements of a row must be contiguous, got strides %s" % (name, st))
        width *= shape[j]
    if lead == 1:
        return st[0] if shape[0] > 1 else width
    if shape[1] > 1:
        row = st[1]
        if shape[0] > 1 and st[0] != shape[1] * row:
            raise ValueError("%s: rows must be equally spaced over batch and tokens, got strides %s" % (name, st))
        return row
    return st[0] if shape[0] > 1 else width


def _gpu(t):
    """Index of a tensor's GPU."""
    index = t.get_device()
    if index < 0:
        raise ValueError("tensors must be CUDA tensors, got one on %s" % t.device)
    return index


def _scratch(workspace, need, index, side, *sizes):
    """(address, bytes, tensor) of the caller's workspace, or of a new one of need(*sizes) bytes."""
    if workspace is None:
        workspace = _workspace(need(*sizes), torch.device("cuda", index), side)
    elif workspace.get_device() != index or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous tensor on cuda:%d" % index)
    return workspace.data_ptr(), workspace.numel() * workspace.element_size(), workspace


def _conv_sizes(x, weight, dims):
    if x.dim() != dims or weight.dim() != 2:
        raise ValueError("x must be %s and weight [C, width], got %s and %s"
                         % ("[B, n, C]" if dims == 3 else "[B, C]", tuple(x.shape), tuple(weight.shape)))
    return x.shape, weight.shape[1], _type_code(x.dtype), x.dtype, _gpu(x)


def hla_conv_forward(x, weight, bias=None, out=None, *, silu=True, lengths=None, state_in=None, state_out=None,
                     stream=None):
    """Short causal depthwise convolution over a prompt (include/hla.h: hla_conv_forward).  Returns ``out``.

    x: [B, n, C], rows may be slices of wider rows; weight: [C, width]; bias: [C]; lengths: int32 [B];
    states: [B, width - 1, C] (state_out may be state_in).
    """
    shape, W, dt, T, i = _conv_sizes(x, weight, 3)
    handle, side = _on(stream, i)
    B, n, C = shape
    if out is None:
        out = _empty(shape, T, x.device, side)
    kept = (B, W - 1, C)
    _check(_entry("hla_conv_forward", i)(
        x.data_ptr(), _flat("weight", weight, C * W, T, i), _flat("bias", bias, C, T, i),
        out.data_ptr(), dt, B, n, C, W,
        _rows("x", x, shape, (1,), T, i, True), _rows("out", out, shape, (1,), T, i), 1 if silu else 0,
        _flat("lengths", lengths, B, torch.int32, i), _shaped("state_in", state_in, kept, T, i),
        _shaped("state_out", state_out, kept, T, i), handle), "hla_conv_forward")
    return out


def hla_conv_step(x, weight, state, bias=None, out=None, *, silu=True, stream=None):
    """One token a sequence of hla_conv_forward (include/hla.h: hla_conv_step); ``state`` [B, width - 1, C] is
    updated in place.  x: [B, C]; ``out`` may be ``x``."""
    shape, W, dt, T, i = _conv_sizes(x, weight, 2)
    handle, side = _on(stream, i)
    B, C = shape
    if out is None:
        out = _empty(shape, T, x.device, side)
    _check(_entry("hla_conv_step", i)(
        x.data_ptr(), _flat("weight", weight, C * W, T, i), _flat("bias", bias, C, T, i),
        out.data_ptr(), dt, B, C, W,
        _rows("x", x, shape, (1,), T, i, True), _rows("out", out, shape, (1,), T, i), 1 if silu else 0,
        _shaped("state", state, (B, W - 1, C), T, i), handle), "hla_conv_step")
    return out


def hla_conv_backward_workspace_bytes(B, n, C, width, dtype) -> int:
    return int(lib().hla_conv_backward_workspace_bytes(B, n, C, width, _type_code(dtype)))


def hla_conv_backward(x, weight, dout, bias=None, dx=None, *, silu=True, lengths=None, workspace=None, stream=None):
    """Gradients (dx, dweight, dbias) of sum(dout * out) for hla_conv_forward from a zero state
    (include/hla.h: hla_conv_backward); the weights' are fp32, dbias is None where bias is."""
    shape, W, dt, T, i = _conv_sizes(x, weight, 3)
    handle, side = _on(stream, i)
    B, n, C = shape
    if dx is None:
        dx = _empty(shape, T, x.device, side)
    dw = _empty((C, W), torch.float32, x.device, side)
    db = None if bias is None else _empty((C,), torch.float32, x.device, side)
    ws, ws_bytes, _keep = _scratch(workspace, hla_conv_backward_workspace_bytes, i, side, B, n, C, W, dt)
    _check(_entry("hla_conv_backward", i)(
        x.data_ptr(), _flat("weight", weight, C * W, T, i), _flat("bias", bias, C, T, i),
        dout.data_ptr(), dx.data_ptr(),
        dw.data_ptr(), None if db is None else db.data_ptr(), dt, B, n, C, W, _rows("x", x, shape, (1,), T, i, True),
        _rows("dout", dout, shape, (1,), T, i), _rows("dx", dx, shape, (1,), T, i), 1 if silu else 0,
        _flat("lengths", lengths, B, torch.int32, i), ws, ws_bytes, handle), "hla_conv_backward")
    return dx, dw, db


def hla_ssm_workspace_bytes(B, n, H, P, G, N, dtype) -> int:
    return int(lib().hla_ssm_workspace_bytes(B, n, H, P, G, N, _type_code(dtype)))


def hla_ssm_forward(x, delta, a, b, c, out=None, *, skip=None, delta_bias=None, softplus=True, lengths=None,
                    state_in=None, state_out=None, workspace=None, stream=None):
    """Selective state space scan over a prompt (include/hla.h: hla_ssm_forward).  Returns ``out``.

    x: [B, n, H, P]; delta: [B, n, H]; b, c: [B, n, G, N] (rows of all four may be slices of wider rows);
    a, skip, delta_bias: fp32 [H]; lengths: int32 [B]; states: fp32 [B, H, N, P] (state_out may be state_in).
    """
    if x.dim() != 4 or b.dim() != 4:
        raise ValueError("x must be [B, n, H, P] and b [B, n, G, N], got %s and %s" % (tuple(x.shape), tuple(b.shape)))
    T, i, shape = x.dtype, _gpu(x), x.shape
    handle, side = _on(stream, i)
    B, n, H, P = shape
    G, N = b.shape[2:]
    dt, f32 = _type_code(T), torch.float32
    if out is None:
        out = _empty(shape, T, x.device, side)
    bc, inner, bc_inner, kept = (B, n, G, N), (P, 1), (N, 1), (B, H, N, P)
    ws, ws_bytes, _keep = _scratch(workspace, hla_ssm_workspace_bytes, i, side, B, n, H, P, G, N, dt)
    _check(_entry("hla_ssm_forward", i)(
        x.data_ptr(), delta.data_ptr(), _flat("a", a, H, f32, i), b.data_ptr(), c.data_ptr(),
        _flat("skip", skip, H, f32, i), _flat("delta_bias", delta_bias, H, f32, i), out.data_ptr(),
        dt, B, n, H, P, G, N, _rows("x", x, shape, inner, T, i, True), _rows("delta", delta, (B, n, H), (1,), T, i),
        _rows("b", b, bc, bc_inner, T, i), _rows("c", c, bc, bc_inner, T, i), _rows("out", out, shape, inner, T, i),
        1 if softplus else 0, _flat("lengths", lengths, B, torch.int32, i),
        _shaped("state_in", state_in, kept, f32, i), _shaped("state_out", state_out, kept, f32, i), ws, ws_bytes,
        handle), "hla_ssm_forward")
    return out


def hla_ssm_forward_path(B, n, H, P, G, N, *, dtype=torch.bfloat16, aligned_rows=True):
    """(path, launches) that hla_ssm_forward takes: path 1 = tensor-core kernels, 0 = fp32 kernels, -1 = unsupported."""
    launches = ctypes.c_int(0)
    path = lib().hla_ssm_forward_path(B, n, H, P, G, N, _type_code(dtype), int(aligned_rows), ctypes.byref(launches))
    return int(path), int(launches.value)


def hla_ssm_step(x, delta, a, b, c, state, out=None, *, skip=None, delta_bias=None, softplus=True, stream=None):
    """One token a sequence of hla_ssm_forward (include/hla.h: hla_ssm_step); ``state`` fp32 [B, H, N, P] is
    updated in place.  x: [B, H, P]; delta: [B, H]; b, c: [B, G, N]; ``out`` may be ``x``."""
    if x.dim() != 3 or b.dim() != 3:
        raise ValueError("x must be [B, H, P] and b [B, G, N], got %s and %s" % (tuple(x.shape), tuple(b.shape)))
    T, i, shape, bc = x.dtype, _gpu(x), x.shape, b.shape
    handle, side = _on(stream, i)
    B, H, P = shape
    G, N = bc[1], bc[2]
    dt, f32 = _type_code(T), torch.float32
    if out is None:
        out = _empty(shape, T, x.device, side)
    bc, inner, bc_inner = (B, G, N), (P, 1), (N, 1)
    _check(_entry("hla_ssm_step", i)(
        x.data_ptr(), delta.data_ptr(), _flat("a", a, H, f32, i), b.data_ptr(), c.data_ptr(),
        _flat("skip", skip, H, f32, i), _flat("delta_bias", delta_bias, H, f32, i), out.data_ptr(),
        dt, B, H, P, G, N, _rows("x", x, shape, inner, T, i, True), _rows("delta", delta, (B, H), (1,), T, i),
        _rows("b", b, bc, bc_inner, T, i), _rows("c", c, bc, bc_inner, T, i), _rows("out", out, shape, inner, T, i),
        1 if softplus else 0, _shaped("state", state, (B, H, N, P), f32, i), handle), "hla_ssm_step")
    return out


def _qk_sizes(q, k, cos, sin):
    if q.dim() != 4 or k.dim() != 4:
        raise ValueError("q must be [B, n, H, d] and k [B, n, Hk, d], got %s and %s" % (tuple(q.shape), tuple(k.shape)))
    rot, top = 0, 0
    if cos is not None:
        if cos.dim() != 2 or sin is None:
            raise ValueError("cos and sin must both be [rows, rot / 2]")
        top, half = cos.shape
        rot = 2 * half
    return q.dtype, _gpu(q), q.shape, k.shape[2], rot, top


def hla_qk_norm_forward(q, k, wq=None, wk=None, cos=None, sin=None, q_out=None, k_out=None, *, positions=None, pos0=0,
                        eps=1e-6, interleaved=False, stream=None):
    """Norm of every query and key head and rotation by position, into the mixers' layout
    (include/hla.h: hla_qk_norm_forward).  Returns (q_out, k_out), both [B, H, n, d].

    q: [B, n, H, d]; k: [B, n, Hk, d] (rows may be slices of wider rows); wq, wk: [d]; cos, sin: fp32
    [rows, rot / 2]; positions: int32 [B, n], or None for pos0, pos0 + 1, ...
    """
    T, i, shape, Hk, rot, top = _qk_sizes(q, k, cos, sin)
    handle, side = _on(stream, i)
    B, n, H, d = shape
    if q_out is None:
        q_out = _empty((B, H, n, d), T, q.device, side)
    if k_out is None:
        k_out = _empty((B, H, n, d), T, q.device, side)
    inner, table, heads = (d, 1), (top, rot // 2), (B, H, n, d)
    _check(_entry("hla_qk_norm_forward", i)(
        q.data_ptr(), k.data_ptr(), _flat("wq", wq, d, T, i), _flat("wk", wk, d, T, i),
        _flat("cos", cos, top * rot // 2, torch.float32, i), _shaped("sin", sin, table, torch.float32, i),
        _shaped("positions", positions, (B, n), torch.int32, i), _shaped("q_out", q_out, heads, T, i),
        _shaped("k_out", k_out, heads, T, i), _type_code(T), B, n, H, Hk, d, rot, 1 if interleaved else 0,
        _rows("q", q, shape, inner, T, i, True), _rows("k", k, (B, n, Hk, d), inner, T, i), pos0, top, eps,
        handle), "hla_qk_norm_forward")
    return q_out, k_out


def hla_qk_norm_backward_workspace_bytes(B, n, H, Hk, d, dtype) -> int:
    return int(lib().hla_qk_norm_backward_workspace_bytes(B, n, H, Hk, d, _type_code(dtype)))


def hla_qk_norm_backward(q, k, wq, wk, cos, sin, dq_out, dk_out, dq=None, dk=None, *, positions=None, pos0=0, eps=1e-6,
                         interleaved=False, workspace=None, stream=None):
    """Gradients (dq, dk, dwq, dwk) of sum(dq_out * q_out) + sum(dk_out * k_out) for hla_qk_norm_forward
    (include/hla.h: hla_qk_norm_backward); dwq, dwk are fp32 [d], None where the weight is."""
    T, i, shape, Hk, rot, top = _qk_sizes(q, k, cos, sin)
    handle, side = _on(stream, i)
    B, n, H, d = shape
    k_shape = (B, n, Hk, d)
    if dq is None:
        dq = _empty(shape, T, q.device, side)
    if dk is None:
        dk = _empty(k_shape, T, q.device, side)
    dwq = None if wq is None else _empty((d,), torch.float32, q.device, side)
    dwk = None if wk is None else _empty((d,), torch.float32, q.device, side)
    dt, inner, table, heads = _type_code(T), (d, 1), (top, rot // 2), (B, H, n, d)
    ws, ws_bytes, _keep = _scratch(workspace, hla_qk_norm_backward_workspace_bytes, i, side, B, n, H, Hk, d, dt)
    _check(_entry("hla_qk_norm_backward", i)(
        q.data_ptr(), k.data_ptr(), _flat("wq", wq, d, T, i), _flat("wk", wk, d, T, i),
        _flat("cos", cos, top * rot // 2, torch.float32, i), _shaped("sin", sin, table, torch.float32, i),
        _shaped("positions", positions, (B, n), torch.int32, i), _shaped("dq_out", dq_out, heads, T, i),
        _shaped("dk_out", dk_out, heads, T, i), dq.data_ptr(), dk.data_ptr(), None if dwq is None else dwq.data_ptr(),
        None if dwk is None else dwk.data_ptr(), dt, B, n, H, Hk, d, rot, 1 if interleaved else 0,
        _rows("q", q, shape, inner, T, i, True), _rows("k", k, k_shape, inner, T, i),
        _rows("dq", dq, shape, inner, T, i), _rows("dk", dk, k_shape, inner, T, i), pos0, top, eps, ws, ws_bytes,
        handle), "hla_qk_norm_backward")
    return dq, dk, dwq, dwk
