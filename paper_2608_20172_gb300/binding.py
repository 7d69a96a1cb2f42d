"""Thin ctypes binding of librelation (include/relation.h) for torch CUDA tensors.

Argument marshalling only: every step of the operator runs in the library's CUDA
kernels.  Tensors are [B, T, H, d_h] (any strides with d_h contiguous, the same for
all tensors of a call); logZ is a dense fp32 [B, H, T].  Calls are enqueued on the
current torch CUDA stream unless ``stream`` is given.

Loading fails loudly (``RelationLibraryMissing``) when the compiled library is absent:
there is no CPU fallback.
"""
from __future__ import annotations

import ctypes
import importlib.machinery
import importlib.util
import os
import threading
import warnings
from typing import NamedTuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "_build", "librelation.so")
CALLS_PATH = os.path.join(_HERE, "_build", "relation_calls.so")

# relation_status
OK, ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_ALIGNMENT, ERR_WORKSPACE, ERR_CUDA, ERR_TIMEOUT, \
    ERR_CAPACITY = range(8)
# relation_dtype
F32, BF16 = 0, 1
# relation_kernel
KERNELS = {"auto": 0, "simt": 1, "tcgen05": 2}

EXPORTED = ("relation_fwd", "relation_fwd_ex", "relation_bwd", "relation_bwd_ex",
            "relation_bwd_workspace_size", "relation_status_string", "relation_version",
            "relation_selftest_wait_timeout", "relation_launch_count", "relation_last_cuda_error",
            "relation_bwd_stages", "relation_bwd_static", "relation_fwd_flow",
            "relation_decode", "relation_decode_workspace_size", "relation_fwd_state",
            "relation_state_merge", "relation_state_finish", "relation_linear_fwd",
            "relation_linear_fwd_ex", "relation_linear_fwd_ws",
            "relation_linear_fwd_workspace_size",
            "relation_linear_bwd", "relation_linear_bwd_workspace_size",
            "relation_linear_bwd_ex", "relation_linear_bwd_ex_workspace_size", "relation_layer_prep",
            "relation_layer_grad", "relation_layer_grad_workspace_size", "relation_page_plan",
            "relation_cache_append", "relation_paged_decode",
            "relation_paged_decode_workspace_size", "relation_sample")


class RelationLibraryMissing(RuntimeError):
    pass


class RelationError(RuntimeError):
    def __init__(self, code: int, where: str):
        msg = f"{where}: {status_string(code)} ({code})"
        if code == ERR_CUDA:
            msg += f": {load().relation_last_cuda_error().decode()}"
        super().__init__(msg)
        self.code = code


class Shape(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int), ("T", ctypes.c_int), ("H", ctypes.c_int),
                ("d_h", ctypes.c_int), ("sB", ctypes.c_longlong), ("sT", ctypes.c_longlong),
                ("sH", ctypes.c_longlong)]


class Pages(ctypes.Structure):
    _fields_ = [("n_pages", ctypes.c_int), ("page_size", ctypes.c_int), ("H", ctypes.c_int),
                ("d_h", ctypes.c_int), ("sP", ctypes.c_longlong), ("sR", ctypes.c_longlong),
                ("sH", ctypes.c_longlong)]


_lock = threading.Lock()
_lib = None


def load(path: str | None = None):
    """Load librelation.so (default: the in-tree build) and declare its signatures."""
    global _lib
    if path is None and _lib is not None:
        return _lib
    with _lock:
        if _lib is not None and path is None:
            return _lib
        p = path or LIB_PATH
        if not os.path.exists(p):
            raise RelationLibraryMissing(
                f"{p} not found: build it with paper_2608_20172_gb300.build.build()")
        lib = ctypes.CDLL(p)
        vp, ip = ctypes.c_void_p, ctypes.c_void_p
        f, i, sz = ctypes.c_float, ctypes.c_int, ctypes.c_size_t
        lib.relation_fwd.argtypes = [vp, vp, vp, vp, vp, f, f, Shape, i, ip, vp]
        lib.relation_fwd_ex.argtypes = [vp, vp, vp, vp, vp, f, f, Shape, i, i, ip, vp]
        lib.relation_fwd_flow.argtypes = [vp, vp, vp, vp, vp, vp, f, f, Shape, i, i, ip, vp]
        ll = ctypes.c_longlong
        lib.relation_decode.argtypes = [vp, vp, vp, vp, vp, vp, f, f, Shape, ll, ll, i, vp,
                                        ctypes.c_size_t, ip, vp]
        lib.relation_decode_workspace_size.argtypes = [Shape, i]
        lib.relation_fwd_state.argtypes = [vp, vp, vp, vp, vp, vp, Shape, Shape, i, i, ip, vp]
        lib.relation_state_merge.argtypes = [vp, vp, vp, vp, vp, vp, Shape, vp]
        lib.relation_state_finish.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, f, f, ll, Shape,
                                              i, vp]
        lib.relation_linear_fwd.argtypes = [vp, vp, vp, vp, vp, f, Shape, i, ip, vp]
        lib.relation_linear_fwd_ex.argtypes = [vp, vp, vp, vp, vp, f, Shape, i, i, ip, vp]
        lib.relation_linear_fwd_ws.argtypes = [vp, vp, vp, vp, vp, f, Shape, i, vp, sz, ip, vp]
        lib.relation_linear_fwd_workspace_size.argtypes = [Shape, i]
        lib.relation_linear_fwd_workspace_size.restype = sz
        lib.relation_linear_bwd.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, f, Shape, i, vp,
                                            ctypes.c_size_t, ip, vp]
        lib.relation_linear_bwd_workspace_size.argtypes = [Shape, i]
        lib.relation_linear_bwd_ex.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, f, Shape, i, i,
                                               vp, sz, ip, vp]
        lib.relation_linear_bwd_ex_workspace_size.argtypes = [Shape, i, i]
        lib.relation_linear_bwd_ex_workspace_size.restype = sz
        lib.relation_layer_prep.argtypes = [vp, vp, vp, vp, i, f, vp, vp, vp, Shape, i, vp]
        lib.relation_layer_grad.argtypes = [vp, vp, vp, vp, vp, i, f, vp, vp, vp, vp, Shape, i,
                                            vp, sz, vp]
        lib.relation_layer_grad_workspace_size.argtypes = [Shape, i]
        lib.relation_layer_grad_workspace_size.restype = sz
        lib.relation_page_plan.argtypes = [vp, vp, i, i, vp, i, ll, vp, i, vp, vp, vp, vp, vp, vp, i,
                                           ip, vp]
        lib.relation_cache_append.argtypes = [vp, vp, vp, vp, i, f, vp, vp, vp, i, ll, ll, vp, vp,
                                              Pages, i, ip, vp]
        lib.relation_paged_decode.argtypes = [vp, vp, vp, vp, i, ll, vp, vp, vp, f, f, i, i, Pages, ll,
                                              ll, i, vp, sz, ip, vp]
        lib.relation_paged_decode_workspace_size.argtypes = [i, Pages, i]
        lib.relation_paged_decode_workspace_size.restype = sz
        lib.relation_sample.argtypes = [vp, i, i, ll, i, vp, vp, vp, vp, vp, vp, vp, vp, ip, vp]
        lib.relation_linear_bwd_workspace_size.restype = ctypes.c_size_t
        lib.relation_decode_workspace_size.restype = ctypes.c_size_t
        lib.relation_bwd.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, f, f, Shape, i, vp,
                                     sz, ip, vp]
        lib.relation_bwd_ex.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, f, f, Shape, i,
                                        vp, sz, i, ip, vp]
        lib.relation_bwd_stages.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, f, f, Shape,
                                            i, vp, sz, i, ctypes.c_uint, ip, vp]
        lib.relation_bwd_stages.restype = ctypes.c_int
        lib.relation_bwd_static.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, f, f, Shape,
                                            i, i, ip, vp]
        lib.relation_bwd_static.restype = ctypes.c_int
        lib.relation_bwd_workspace_size.argtypes = [Shape, i]
        lib.relation_bwd_workspace_size.restype = sz
        lib.relation_status_string.argtypes = [i]
        lib.relation_status_string.restype = ctypes.c_char_p
        lib.relation_version.argtypes = []
        lib.relation_selftest_wait_timeout.argtypes = [ip, i, vp]
        lib.relation_launch_count.argtypes = [i, i, i, i]
        lib.relation_last_cuda_error.argtypes = []
        lib.relation_last_cuda_error.restype = ctypes.c_char_p
        for n in ("relation_fwd", "relation_fwd_ex", "relation_bwd", "relation_bwd_ex",
                  "relation_version", "relation_selftest_wait_timeout", "relation_launch_count"):
            getattr(lib, n).restype = ctypes.c_int
        if path is None:
            _lib = lib
        return lib


def status_string(code: int) -> str:
    return load().relation_status_string(int(code)).decode()


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return F32
    if t.dtype == torch.bfloat16:
        return BF16
    raise TypeError(f"unsupported dtype {t.dtype}")


def shape_of(t: torch.Tensor) -> Shape:
    """relation_shape of a [B, T, H, d_h] tensor with d_h contiguous."""
    st = t.stride()
    if len(st) != 4:
        raise ValueError("expected a [B, T, H, d_h] tensor")
    if st[3] != 1:
        raise ValueError("d_h must be contiguous")
    return Shape(*t.shape, *st[:3])


def _same_layout(ref: torch.Tensor, *others: torch.Tensor):
    shape, stride, dtype, device = ref.shape, ref.stride(), ref.dtype, ref.device
    for o in others:
        if o.shape != shape or o.stride() != stride or o.dtype != dtype:
            raise ValueError("all tensors of a call need the same shape, strides and dtype")
        if not o.is_cuda or o.device != device:
            raise ValueError("all tensors must live on the same CUDA device")


# torch.cuda.current_stream().cuda_stream without the Stream object, where torch has it
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream) -> int:
    if stream is None:
        if _raw_stream is None:
            return torch.cuda.current_stream().cuda_stream
        return _raw_stream(torch.cuda.current_device())
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _owned(stream, device, make, result=True):
    """make()'s tensor in the memory of the stream that the call runs on.  Memory of the caller's
    stream would go back to the allocator while the call's kernels are still queued on `stream`
    (scratch does when the call returns), and its last use on the caller's stream need not be over
    when they begin.  A result is used on the caller's stream too, and waits for it when it is freed."""
    given = None if stream is None else _stream(stream)
    if given is None or given == _stream(None):
        return make()
    if not isinstance(stream, torch.cuda.Stream):
        # (the default stream: 0, or cudaStreamLegacy, 1; ExternalStream takes 0 for none given)
        stream = torch.cuda.ExternalStream(given, device=device) if given > 1 else \
            torch.cuda.default_stream(device)
    here = torch.cuda.current_stream(device)
    with torch.cuda.stream(stream):
        t = make()
    if result:
        t.record_stream(here)
    return t


def _like(t: torch.Tensor, stream=None) -> torch.Tensor:
    """An output with t's shape, dtype, device and strides, of the call's stream.  The C ABI writes
    an output with its input's element strides, which torch.empty_like does not keep for a view
    that is not dense (e.g. a slice of a padded tensor); for a contiguous one it does."""
    if stream is not None:
        return _owned(stream, t.device, lambda: _like(t))
    if type(t) is torch.Tensor and t.is_contiguous():
        return torch.empty_like(t)
    return torch.empty_strided(t.size(), t.stride(), dtype=t.dtype, device=t.device)


def _new(size, dtype, device, stream=None) -> torch.Tensor:
    """A dense output of the call's stream."""
    if stream is None:
        return torch.empty(size, dtype=dtype, device=device)
    return _owned(stream, device, lambda: torch.empty(size, dtype=dtype, device=device))


def _scratch(nbytes: int, device, stream=None) -> torch.Tensor:
    """Device bytes that only the call's kernels use."""
    if stream is None:
        return torch.empty(nbytes, dtype=torch.uint8, device=device)
    return _owned(stream, device, lambda: torch.empty(nbytes, dtype=torch.uint8, device=device),
                  result=False)


def _queue(stream, device: int) -> int:
    """The stream of a call whose operands are on cuda:`device`: given, or the current one.  The
    library launches on the current device."""
    if device != torch.cuda.current_device():
        raise ValueError(f"the operands are on cuda:{device}, which is not the current device")
    return _stream(stream)


def _ptr(t):
    return None if t is None else t.data_ptr()


def _status(t, device: int):
    """dev_status's pointer: an int32 that the kernels of a call on cuda:`device` may write (on that
    device, or in pinned host memory)."""
    if t is None:
        return None
    if t.dtype is not torch.int32 or t.numel() < 1 or not (t.get_device() == device or
                                                           (t.device.type == "cpu" and t.is_pinned())):
        raise ValueError("dev_status must be an int32 tensor on the operands' CUDA device")
    return t.data_ptr()


def workspace_size(q: torch.Tensor) -> int:
    return int(load().relation_bwd_workspace_size(shape_of(q), _dtype_code(q)))


def fwd(q, k, v, lam: float, tau_s: float = 2.0, *, kernel: str = "auto", out=None, logz=None,
        dev_status=None, stream=None):
    """Forward.  Returns (Y, logZ)."""
    _same_layout(q, k, v)
    B, T, H, _ = q.shape
    if out is None:
        out = _like(q, stream)
    else:
        _same_layout(q, out)
    if logz is None:
        logz = _new((B, H, T), torch.float32, q.device, stream)
    rc = load().relation_fwd_ex(_ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(logz), float(lam),
                                float(tau_s), shape_of(q), _dtype_code(q), KERNELS[kernel],
                                _status(dev_status, q.get_device()), _queue(stream, q.get_device()))
    if rc != OK:
        raise RelationError(rc, "relation_fwd")
    return out, logz


def fwd_flow(q, k, v, lam: float, tau_s: float = 2.0, *, kernel: str = "auto", out=None,
             logz=None, self_flow=None, dev_status=None, stream=None):
    """Forward with the Self flow F_ii = 1 - g_i of every row as a side output.
    Returns (Y, logZ, F_self) with F_self [B, H, T] fp32."""
    _same_layout(q, k, v)
    B, T, H, _ = q.shape
    if out is None:
        out = _like(q, stream)
    else:
        _same_layout(q, out)
    if logz is None:
        logz = _new((B, H, T), torch.float32, q.device, stream)
    if self_flow is None:
        self_flow = _new((B, H, T), torch.float32, q.device, stream)
    rc = load().relation_fwd_flow(_ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(logz),
                                  _ptr(self_flow), float(lam), float(tau_s), shape_of(q),
                                  _dtype_code(q), KERNELS[kernel], _status(dev_status, q.get_device()),
                                  _queue(stream, q.get_device()))
    if rc != OK:
        raise RelationError(rc, "relation_fwd_flow")
    return out, logz, self_flow


def linear_fwd(p1, p2, v, alpha, tau_s: float = 2.0, *, kernel: str = "auto", out=None,
               dev_status=None, stream=None):
    """Linear Relation forward.  p1, p2, v [B, T, H, d] (fp32 or bf16), alpha [B, T, H, d]
    fp32 with p1's strides.  ``kernel``: "simt" (the recurrence), "tcgen05" (the chunked
    tensor-core form) or "auto".  Returns Y."""
    _same_layout(p1, p2, v)
    if alpha.dtype != torch.float32 or tuple(alpha.shape) != tuple(p1.shape) or \
            tuple(alpha.stride()) != tuple(p1.stride()):
        raise ValueError("alpha must be fp32 with p1's shape and strides")
    if out is None:
        out = _like(p1, stream)
    else:
        _same_layout(p1, out)
    rc = load().relation_linear_fwd_ex(_ptr(p1), _ptr(p2), _ptr(v), _ptr(alpha), _ptr(out),
                                       float(tau_s), shape_of(p1), _dtype_code(p1),
                                       KERNELS[kernel], _status(dev_status, p1.get_device()),
                                       _queue(stream, p1.get_device()))
    if rc != OK:
        raise RelationError(rc, "relation_linear_fwd_ex")
    return out


def _check_summary(state, B, H, T, d, device):
    """(m, l, z): dense fp32 [B, H, T], [B, H, T], [B, H, T, d] on `device`."""
    m, l, z = state
    for t, shp in ((m, (B, H, T)), (l, (B, H, T)), (z, (B, H, T, d))):
        if tuple(t.shape) != shp or t.dtype != torch.float32 or not t.is_contiguous() or \
                t.device != device:
            raise ValueError("an Exchange summary is dense fp32 (m, l [B, H, T], z [B, H, T, d]) "
                             "on the operands' device")


def fwd_state(q, k, v, causal: bool, *, out=None, dev_status=None, stream=None):
    """Exchange summary of every row of q ([B, Tq, H, d]) over the keys of k, v ([B, Tk, H,
    d]): causal = the queries' own tokens (keys before each row), else every key precedes
    every query.  Returns (m, l, z): m, l [B, H, Tq] and z [B, H, Tq, d], fp32."""
    _same_layout(k, v)
    if causal:
        _same_layout(q, k, v)
    B, Tq, H, d = q.shape
    if out is None:
        out = (_new((B, H, Tq), torch.float32, q.device, stream),
               _new((B, H, Tq), torch.float32, q.device, stream),
               _new((B, H, Tq, d), torch.float32, q.device, stream))
    m, l, z = out
    _check_summary(out, B, H, Tq, d, q.device)
    rc = load().relation_fwd_state(_ptr(q), _ptr(k), _ptr(v), _ptr(m), _ptr(l), _ptr(z),
                                   shape_of(q), shape_of(k), int(bool(causal)), _dtype_code(q),
                                   _status(dev_status, k.get_device()), _queue(stream, k.get_device()))
    if rc != OK:
        raise RelationError(rc, "relation_fwd_state")
    return m, l, z


def state_merge(state, other, *, stream=None):
    """Merge the summary ``other`` into ``state`` (both (m, l, z) as fwd_state returns them,
    same rows) in place; returns ``state``."""
    m, l, z = state
    m2, l2, z2 = other
    B, H, T, d = z.shape
    _check_summary(state, B, H, T, d, z.device)
    _check_summary(other, B, H, T, d, z.device)
    rc = load().relation_state_merge(_ptr(m), _ptr(l), _ptr(z), _ptr(m2), _ptr(l2), _ptr(z2),
                                     Shape(B, T, H, d, T * H * d, H * d, d),
                                     _queue(stream, z.get_device()))
    if rc != OK:
        raise RelationError(rc, "relation_state_merge")
    return state


def state_finish(q, k, v, state, lam: float, tau_s: float = 2.0, pos0: int = 0, *, out=None,
                 logz=None, self_flow=None, stream=None):
    """Y and logZ of the rows of q, k, v from their merged summary ``state``; row r is at
    zero-based position pos0 + r of the sequence.  Returns (Y, logZ)."""
    _same_layout(q, k, v)
    m, l, z = state
    B, T, H, d = q.shape
    if out is None:
        out = _like(q, stream)
    else:
        _same_layout(q, out)
    logz = _new((B, H, T), torch.float32, q.device, stream) if logz is None else logz
    _check_summary(state, B, H, T, d, q.device)
    if tuple(logz.shape) != (B, H, T) or logz.dtype != torch.float32 or not logz.is_contiguous():
        raise ValueError("logz must be a dense fp32 [B, H, T] tensor")
    rc = load().relation_state_finish(_ptr(q), _ptr(k), _ptr(v), _ptr(m), _ptr(l), _ptr(z),
                                      _ptr(out), _ptr(logz), _ptr(self_flow), float(lam),
                                      float(tau_s), int(pos0), shape_of(q), _dtype_code(q),
                                      _queue(stream, q.get_device()))
    if rc != OK:
        raise RelationError(rc, "relation_state_finish")
    return out, logz


def linear_fwd_workspace_size(p1) -> int:
    return int(load().relation_linear_fwd_workspace_size(shape_of(p1), _dtype_code(p1)))


def linear_fwd_ws(p1, p2, v, alpha, tau_s: float = 2.0, *, workspace=None, out=None,
                  dev_status=None, stream=None):
    """Linear Relation forward through relation_linear_fwd_ws (the chunk-parallel form for
    long sequences with few heads).  ``workspace``: a uint8 CUDA tensor of at least
    linear_fwd_workspace_size(p1) bytes (allocated here when None).  Returns Y."""
    _same_layout(p1, p2, v)
    if alpha.dtype != torch.float32 or tuple(alpha.shape) != tuple(p1.shape) or \
            tuple(alpha.stride()) != tuple(p1.stride()):
        raise ValueError("alpha must be fp32 with p1's shape and strides")
    if out is None:
        out = _like(p1, stream)
    else:
        _same_layout(p1, out)
    if workspace is None:
        workspace = _scratch(max(linear_fwd_workspace_size(p1), 16), p1.device, stream)
    rc = load().relation_linear_fwd_ws(_ptr(p1), _ptr(p2), _ptr(v), _ptr(alpha), _ptr(out),
                                       float(tau_s), shape_of(p1), _dtype_code(p1),
                                       _ptr(workspace), workspace.numel(),
                                       _status(dev_status, p1.get_device()),
                                       _queue(stream, p1.get_device()))
    if rc != OK:
        raise RelationError(rc, "relation_linear_fwd_ws")
    return out


def linear_bwd_workspace_size(p1, kernel: str = "auto") -> int:
    """Bytes of device scratch linear_bwd needs for tensors shaped like p1 (0: the kernel
    family does not serve this request)."""
    return int(load().relation_linear_bwd_ex_workspace_size(shape_of(p1), _dtype_code(p1),
                                                            KERNELS[kernel]))


def linear_bwd(p1, p2, v, alpha, dy, tau_s: float = 2.0, *, kernel: str = "auto",
               workspace=None, dev_status=None, stream=None):
    """Linear Relation backward.  Returns (dp1, dp2, dv, dalpha) with dalpha fp32.
    ``kernel``: "auto", "simt" (reverse mode through the token recurrence) or "tcgen05"
    (through the 128-token blocks of the chunked forward; bf16, d_h 64)."""
    _same_layout(p1, p2, v, dy)
    if alpha.dtype != torch.float32 or tuple(alpha.shape) != tuple(p1.shape) or \
            tuple(alpha.stride()) != tuple(p1.stride()):
        raise ValueError("alpha must be fp32 with p1's shape and strides")
    dp1, dp2, dv = _like(p1, stream), _like(p1, stream), _like(p1, stream)
    dalpha = _like(alpha, stream)
    if workspace is None:
        workspace = _scratch(max(linear_bwd_workspace_size(p1, kernel), 16), p1.device, stream)
    rc = load().relation_linear_bwd_ex(_ptr(p1), _ptr(p2), _ptr(v), _ptr(alpha), _ptr(dy),
                                       _ptr(dp1), _ptr(dp2), _ptr(dv), _ptr(dalpha),
                                       float(tau_s), shape_of(p1), _dtype_code(p1),
                                       KERNELS[kernel], _ptr(workspace),
                                       workspace.numel() * workspace.element_size(),
                                       _status(dev_status, p1.get_device()),
                                       _queue(stream, p1.get_device()))
    if rc != OK:
        raise RelationError(rc, "relation_linear_bwd_ex")
    return dp1, dp2, dv, dalpha


def _layer_args(theta, pairing, rope_base, x, stream):
    if theta.dtype != torch.float32 or theta.device != x.device or theta.numel() != x.shape[2] // 2:
        raise ValueError("theta must be fp32 [H/2] on the inputs' device")
    if pairing not in (0, 1):
        raise ValueError("pairing must be 0 (pairs (0,1), (2,3), ...) or 1 ((1,2), ..., (H-1,0))")
    if not theta.is_contiguous():
        theta = _owned(stream, x.device, theta.contiguous, result=False)
    return theta, int(pairing), float(rope_base)


def layer_prep(p1, p2, info, theta, pairing: int = 0, rope_base: float = 1.0e4, *, out=None,
               stream=None):
    """The layer's transforms before the operator: returns (q, k, v) = (RoPE(p1),
    RoPE(p2), Givens(info)) for [B, T, H, d] inputs of one layout, theta fp32 [H/2]."""
    _same_layout(p1, p2, info)
    theta, pairing, rope_base = _layer_args(theta, pairing, rope_base, p1, stream)
    if out is None:
        q, k, v = _like(p1, stream), _like(p1, stream), _like(p1, stream)
    else:
        q, k, v = out
        _same_layout(p1, q, k, v)
    rc = load().relation_layer_prep(_ptr(p1), _ptr(p2), _ptr(info), _ptr(theta), pairing,
                                    rope_base, _ptr(q), _ptr(k), _ptr(v), shape_of(p1),
                                    _dtype_code(p1), _queue(stream, p1.get_device()))
    if rc != OK:
        raise RelationError(rc, "relation_layer_prep")
    return q, k, v


def layer_grad_workspace_size(x) -> int:
    """Device bytes relation_layer_grad needs for a [B, T, H, d] tensor of this dtype."""
    return int(load().relation_layer_grad_workspace_size(shape_of(x), _dtype_code(x)))


def layer_grad(dq, dk, dv, info, theta, pairing: int = 0, rope_base: float = 1.0e4, *,
               workspace=None, stream=None):
    """Gradient of layer_prep: returns (dp1, dp2, dinfo, dtheta)."""
    _same_layout(dq, dk, dv, info)
    theta, pairing, rope_base = _layer_args(theta, pairing, rope_base, dq, stream)
    dp1, dp2, dinfo = _like(dq, stream), _like(dq, stream), _like(dq, stream)
    dtheta = _like(theta, stream)
    if workspace is None:
        workspace = _scratch(max(layer_grad_workspace_size(dq), 16), dq.device, stream)
    rc = load().relation_layer_grad(_ptr(dq), _ptr(dk), _ptr(dv), _ptr(info), _ptr(theta),
                                    pairing, rope_base, _ptr(dp1), _ptr(dp2), _ptr(dinfo),
                                    _ptr(dtheta), shape_of(dq), _dtype_code(dq), _ptr(workspace),
                                    workspace.numel() * workspace.element_size(),
                                    _queue(stream, dq.get_device()))
    if rc != OK:
        raise RelationError(rc, "relation_layer_grad")
    return dp1, dp2, dinfo, dtheta


def decode_workspace_size(k_cache) -> int:
    """Device bytes relation_decode needs for a [B, T, H, d] cache of this dtype."""
    return int(load().relation_decode_workspace_size(shape_of(k_cache), _dtype_code(k_cache)))


def decode(q, k_cache, v_cache, lengths, lam: float, tau_s: float = 2.0, *, out=None, logz=None,
           workspace=None, dev_status=None, stream=None):
    """One new token per sequence against a [B, T, H, d] key/value cache whose row
    lengths[b] - 1 is that token.  q is [B, H, d]; lengths is a device int32 [B].
    Returns (Y [B, H, d], logZ [B, H])."""
    _same_layout(k_cache, v_cache)
    B, T, H, d = k_cache.shape
    if tuple(q.shape) != (B, H, d) or q.stride(2) != 1 or q.dtype != k_cache.dtype:
        raise ValueError("q must be [B, H, d] with d contiguous, of the cache's dtype")
    if lengths.dtype != torch.int32 or lengths.numel() != B or not lengths.is_contiguous():
        raise ValueError("lengths must be a contiguous int32 tensor of B entries")
    out = _like(q, stream) if out is None else out
    if out.stride() != q.stride():
        raise ValueError("out must have q's layout")
    if logz is None:
        logz = _new((B, H), torch.float32, q.device, stream)
    if workspace is None:
        workspace = _scratch(decode_workspace_size(k_cache), q.device, stream)
    rc = load().relation_decode(_ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(lengths), _ptr(out),
                                _ptr(logz), float(lam), float(tau_s), shape_of(k_cache),
                                q.stride(0), q.stride(1), _dtype_code(q), _ptr(workspace),
                                workspace.numel() * workspace.element_size(),
                                _status(dev_status, k_cache.get_device()),
                                _queue(stream, k_cache.get_device()))
    if rc != OK:
        raise RelationError(rc, "relation_decode")
    return out, logz


# The calls of a serving step are short, so that the host's time counts.  The common call (outputs to be
# allocated, the current stream) goes through csrc/torch_calls.cpp, which checks, allocates and calls
# the library in native code (host time of page_plan, cache_append, paged_decode and sample: 8, 5, 9 and
# 6 us a call, 19, 16, 21 and 14 in Python) and answers None to whatever it does not take; then, and
# where there is none to use, the code here does the same and says what is wrong.
_I32, _I64, _F32 = torch.int32, torch.int64, torch.float32
_calls = None


class _NoCalls:
    """Stands for relation_calls.so where there is none to use: takes nothing."""

    @staticmethod
    def page_plan(*_):
        return None

    cache_append = paged_decode = sample = page_plan


def _load_calls(lib):
    """relation_calls.so, bound to the library's functions; _NoCalls where it is not built, and with
    a warning where it does not load or is not that of these sources and this torch."""
    from . import build

    if not os.path.exists(CALLS_PATH):
        return _NoCalls
    try:
        if not build.calls_current(CALLS_PATH):
            raise ImportError("built from other sources or for another torch")
        loader = importlib.machinery.ExtensionFileLoader("relation_calls", CALLS_PATH)
        m = importlib.util.module_from_spec(importlib.util.spec_from_loader("relation_calls", loader))
    except ImportError as e:
        warnings.warn(f"relation_calls.so is not used ({e}): the serving calls run through Python; "
                      "paper_2608_20172_gb300.build.build() builds it", RuntimeWarning, stacklevel=4)
        return _NoCalls
    m.bind(*(ctypes.cast(f, ctypes.c_void_p).value for f in (
        lib.relation_page_plan, lib.relation_cache_append, lib.relation_paged_decode,
        lib.relation_paged_decode_workspace_size, lib.relation_sample)))
    return m


def _native():
    """The serving calls in native code."""
    global _calls
    lib = load()
    with _lock:
        if _calls is None:
            _calls = _load_calls(lib)
    return _calls


class PagePlan(NamedTuple):
    """What page_plan returns; the block table and the free pages are updated in place."""
    slots: torch.Tensor       # int64 [n_tokens]: page * page_size + row, -1 for padding
    positions: torch.Tensor   # int32 [n_tokens]: zero-based position, -1 for padding
    starts: torch.Tensor      # int32 [B + 1]: request b's tokens are starts[b] .. starts[b + 1] - 1
    lengths: torch.Tensor     # int32 [B]: rows in the cache after the step
    free_state: torch.Tensor  # int32 [2]: head and count of the ring of free pages after it


def _need(name, t, device, dtype, count):
    """Raise unless t is a contiguous CUDA tensor of `count` entries of this dtype on the device."""
    if t.dtype is not dtype or not t.is_contiguous() or t.numel() != count or \
            t.get_device() != device or device < 0:
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of {count} entries on the "
                         "operands' CUDA device")


def _is_table(t, B, device):
    return t.dtype is _I32 and t.dim() == 2 and t.shape[0] == B and t.stride(1) == 1 and \
        t.get_device() == device


def page_plan(lengths, counts, block_table, free_pages, free_state, page_size: int, n_tokens: int,
              *, out: PagePlan | None = None, dev_status=None, stream=None) -> PagePlan:
    """Pages, slots and positions of one step's new tokens: lengths and counts int32 [B] (count
    < 0: the request has ended), block_table int32 [B, cols] (rows may be strided) and the ring
    free_pages int32 [n_pages], both updated in place, free_state int32 [2] = (head, count).
    ``n_tokens`` is the size of the step's token buffer.  See relation_page_plan."""
    if out is None and stream is None:
        r = (_calls or _native()).page_plan(lengths, counts, block_table, free_pages, free_state,
                                            page_size, n_tokens, dev_status)
        if r is not None:
            return PagePlan._make(r)
    dev, B, n, n_pages = lengths.get_device(), lengths.numel(), int(n_tokens), free_pages.numel()
    _need("lengths", lengths, dev, _I32, B)
    _need("counts", counts, dev, _I32, B)
    _need("free_pages", free_pages, dev, _I32, n_pages)
    _need("free_state", free_state, dev, _I32, 2)
    if not _is_table(block_table, B, dev):
        raise ValueError("block_table must be an int32 [B, cols] tensor with contiguous rows on "
                         "the operands' device")
    if out is None:  # (five small allocations take less than one and its views)
        on = lengths.device
        slots = _new(n, _I64, on, stream)
        positions = _new(n, _I32, on, stream)
        starts = _new(B + 1, _I32, on, stream)
        new = _new(B, _I32, on, stream)
        state = _new(2, _I32, on, stream)
        out = PagePlan(slots, positions, starts, new, state)
    else:
        slots, positions, starts, new, state = out
        _need("out.slots", slots, dev, _I64, n)
        _need("out.positions", positions, dev, _I32, n)
        _need("out.starts", starts, dev, _I32, B + 1)
        _need("out.lengths", new, dev, _I32, B)
        _need("out.free_state", state, dev, _I32, 2)
    rc = load().relation_page_plan(lengths.data_ptr(), counts.data_ptr(), B, int(page_size),
                                   block_table.data_ptr(), block_table.shape[1],
                                   block_table.stride(0), free_pages.data_ptr(), n_pages,
                                   free_state.data_ptr(), state.data_ptr(), new.data_ptr(),
                                   starts.data_ptr(), slots.data_ptr(), positions.data_ptr(), n,
                                   _status(dev_status, dev), _queue(stream, dev))
    if rc != OK:
        raise RelationError(rc, "relation_page_plan")
    return out


def pages_of(k_pages, v_pages) -> Pages:
    """relation_pages of a pair of [n_pages, page_size, H, d] tensors with d contiguous."""
    shape, st = k_pages.shape, k_pages.stride()
    if v_pages is not k_pages and (v_pages.shape != shape or v_pages.stride() != st or
                                   v_pages.dtype is not k_pages.dtype or
                                   v_pages.get_device() != k_pages.get_device()):
        raise ValueError("the keys' and the values' pages need the same shape, strides, dtype and "
                         "device")
    if len(st) != 4 or st[3] != 1 or k_pages.get_device() < 0:
        raise ValueError("pages must be CUDA [n_pages, page_size, H, d] tensors with d contiguous")
    return Pages(*shape, *st[:3])


def cache_append(p1, p2, info, theta, positions, slots, k_pages, v_pages, pairing: int = 0,
                 rope_base: float = 1.0e4, *, out=None, dev_status=None, stream=None):
    """The layer's transforms of N new tokens at their positions, written into the pages:
    k_pages[slot] = RoPE(p2), v_pages[slot] = Givens(info); returns q = RoPE(p1) (None where p1 is
    None).  p1, p2, info [N, H, d] of one layout, theta fp32 [H/2] or None (no mixing), positions
    int32 [N] (unused with rope_base 0: no rotation), slots int64 [N], negative for padding."""
    if out is None and stream is None:
        r = (_calls or _native()).cache_append(p1, p2, info, theta, positions, slots, k_pages, v_pages,
                                               pairing, rope_base, dev_status)
        if r is not None:
            return r
    pages = pages_of(k_pages, v_pages)
    dev, dtype, shape, st = k_pages.get_device(), k_pages.dtype, p2.shape, p2.stride()
    if p1 is None:
        out = None
    elif out is None:
        out = _like(p1, stream)
    for t in (p2, info) if p1 is None else (p2, info, p1, out):
        if t.dtype is not dtype or t.get_device() != dev or t.shape != shape or t.stride() != st:
            raise ValueError("p1, p2, info and out need the same shape and strides and the pages' "
                             "dtype and device")
    if len(shape) != 3 or st[2] != 1 or shape[1] != pages.H or shape[2] != pages.d_h:
        raise ValueError("tokens must be [N, H, d] with d contiguous, of the pages' H and d")
    N = shape[0]
    _need("slots", slots, dev, _I64, N)
    if positions is not None:
        _need("positions", positions, dev, _I32, N)
    if theta is not None:
        _need("theta", theta, dev, _F32, shape[1] // 2)
    rc = load().relation_cache_append(_ptr(p1), p2.data_ptr(), info.data_ptr(), _ptr(theta),
                                      int(pairing), float(rope_base), _ptr(positions),
                                      slots.data_ptr(), _ptr(out), N, st[0], st[1],
                                      k_pages.data_ptr(), v_pages.data_ptr(), pages,
                                      _dtype_code(p2), _status(dev_status, dev), _queue(stream, dev))
    if rc != OK:
        raise RelationError(rc, "relation_cache_append")
    return out


def paged_decode_workspace_size(q, k_pages) -> int:
    """Device bytes paged_decode needs for queries [B, H, d] over these pages."""
    return int(load().relation_paged_decode_workspace_size(q.shape[1], pages_of(k_pages, k_pages),
                                                           _dtype_code(k_pages)))


def paged_decode(q, k_pages, v_pages, block_table, lengths, lam: float, tau_s: float = 2.0, *,
                 out=None, logz=None, workspace=None, dev_status=None, stream=None):
    """One new token per request over [n_pages, page_size, Hk, d] pages: q [B, H, d] with H a
    multiple of Hk, block_table int32 [B, cols] (rows may be strided), lengths int32 [B] counting
    the new token (0: idle).  Returns (Y [B, H, d], logZ [B, H])."""
    if out is None and logz is None and workspace is None and stream is None:
        r = (_calls or _native()).paged_decode(q, k_pages, v_pages, block_table, lengths, lam, tau_s,
                                               dev_status)
        if r is not None:
            return r
    pages = pages_of(k_pages, v_pages)
    dev, shape, st = k_pages.get_device(), q.shape, q.stride()
    if len(shape) != 3 or shape[2] != pages.d_h or st[2] != 1 or \
            q.dtype is not k_pages.dtype or q.get_device() != dev:
        raise ValueError("q must be [B, H, d] with d contiguous, of the pages' d, dtype and device")
    B, H, _ = shape
    _need("lengths", lengths, dev, _I32, B)
    if not _is_table(block_table, B, dev):
        raise ValueError("block_table must be an int32 [B, cols] tensor with contiguous rows on "
                         "the pages' device")
    if out is None:
        out = _like(q, stream)
    elif out.shape != shape or out.stride() != st or out.dtype is not q.dtype or \
            out.get_device() != dev:
        raise ValueError("out must have q's layout")
    if logz is None:
        logz = _new((B, H), _F32, q.device, stream)
    else:
        _need("logz", logz, dev, _F32, B * H)
    lib, dt = load(), _dtype_code(q)
    if workspace is None:
        workspace = _scratch(lib.relation_paged_decode_workspace_size(H, pages, dt), q.device, stream)
    rc = lib.relation_paged_decode(q.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(),
                                   block_table.data_ptr(), block_table.shape[1],
                                   block_table.stride(0), lengths.data_ptr(), out.data_ptr(),
                                   logz.data_ptr(), float(lam), float(tau_s), B, H, pages, st[0],
                                   st[1], dt, workspace.data_ptr(),
                                   workspace.numel() * workspace.element_size(),
                                   _status(dev_status, dev), _queue(stream, dev))
    if rc != OK:
        raise RelationError(rc, "relation_paged_decode")
    return out, logz


def sample(logits, u, *, temperature=None, top_k=None, top_p=None, min_p=None, out=None,
           dev_status=None, stream=None):
    """The next token of every row of logits [R, V] (fp32 or bf16, rows may be strided) from
    uniform numbers u fp32 [R]; temperature, top_p, min_p fp32 [R] and top_k int32 [R], each
    optional.  Returns (token int32 [R], logprob fp32 [R], logz fp32 [R]); see relation_sample."""
    if out is None and stream is None:
        r = (_calls or _native()).sample(logits, u, temperature, top_k, top_p, min_p, dev_status)
        if r is not None:
            return r
    dev, dt, st = logits.get_device(), _dtype_code(logits), logits.stride()
    if len(st) != 2 or st[1] != 1 or dev < 0:
        raise ValueError("logits must be a CUDA [R, V] tensor with contiguous rows")
    R, V = logits.shape
    _need("u", u, dev, _F32, R)
    if temperature is not None:
        _need("temperature", temperature, dev, _F32, R)
    if top_k is not None:
        _need("top_k", top_k, dev, _I32, R)
    if top_p is not None:
        _need("top_p", top_p, dev, _F32, R)
    if min_p is not None:
        _need("min_p", min_p, dev, _F32, R)
    if out is None:
        out = (_new(R, _I32, u.device, stream), _like(u, stream), _like(u, stream))
        token, logprob, logz = out
    else:
        token, logprob, logz = out
        _need("token", token, dev, _I32, R)
        _need("logprob", logprob, dev, _F32, R)
        _need("logz", logz, dev, _F32, R)
    rc = load().relation_sample(logits.data_ptr(), R, V, st[0], dt, u.data_ptr(),
                                _ptr(temperature), _ptr(top_k), _ptr(top_p), _ptr(min_p),
                                token.data_ptr(), logprob.data_ptr(), logz.data_ptr(),
                                _status(dev_status, dev), _queue(stream, dev))
    if rc != OK:
        raise RelationError(rc, "relation_sample")
    return out


BWD_PREPARE, BWD_TILES, BWD_FINALIZE, BWD_ALL = 1, 2, 4, 7


def bwd(q, k, v, o, dout, logz, lam: float, tau_s: float = 2.0, *, kernel: str = "auto",
        workspace=None, dq=None, dk=None, dv=None, dlambda=None, dev_status=None, stream=None,
        stages: int = BWD_ALL):
    """Backward.  Returns (dQ, dK, dV, dlambda) with dlambda a 1-element fp32 device tensor.
    ``stages`` selects a subset of the three backward stages (see relation_bwd_stages)."""
    _same_layout(q, k, v, o, dout)
    given = [t for t in (dq, dk, dv) if t is not None]
    if given:
        _same_layout(q, *given)
    dq = _like(q, stream) if dq is None else dq
    dk = _like(q, stream) if dk is None else dk
    dv = _like(q, stream) if dv is None else dv
    if dlambda is None:
        dlambda = _new(1, torch.float32, q.device, stream)
    if workspace is None:
        workspace = _scratch(workspace_size(q), q.device, stream)
    rc = load().relation_bwd_stages(_ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(dout), _ptr(logz),
                                    _ptr(dq), _ptr(dk), _ptr(dv), _ptr(dlambda), float(lam),
                                    float(tau_s), shape_of(q), _dtype_code(q),
                                    _ptr(workspace), workspace.numel() * workspace.element_size(),
                                    KERNELS[kernel], int(stages), _status(dev_status, q.get_device()),
                                    _queue(stream, q.get_device()))
    if rc != OK:
        raise RelationError(rc, "relation_bwd")
    return dq, dk, dv, dlambda


def launches_per_call(kernel: str, dtype: str, d: int, which: str) -> int:
    """Kernel launches one fwd / bwd call makes (0 when unsupported)."""
    dt = F32 if dtype in ("fp32", "f32", torch.float32) else BF16
    return int(load().relation_launch_count(dt, int(d), KERNELS[kernel], int(which == "bwd")))


STATIC_SCRATCH_BYTES = 64 << 20  # RELATION_STATIC_SCRATCH_BYTES


def bwd_no_alloc(q, k, v, o, dout, logz, lam: float, tau_s: float = 2.0, *,
                 kernel: str = "auto", dq, dk, dv, dlambda, dev_status=None, stream=None):
    """Backward through relation_bwd_static: the library's fixed scratch array replaces the
    workspace, for callers that must not allocate device memory.  All outputs are
    caller-provided (this function allocates nothing either)."""
    _same_layout(q, k, v, o, dout, dq, dk, dv)
    rc = load().relation_bwd_static(_ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(dout), _ptr(logz),
                                    _ptr(dq), _ptr(dk), _ptr(dv), _ptr(dlambda), float(lam),
                                    float(tau_s), shape_of(q), _dtype_code(q), KERNELS[kernel],
                                    _status(dev_status, q.get_device()), _queue(stream, q.get_device()))
    if rc != OK:
        raise RelationError(rc, "relation_bwd_static")
    return dq, dk, dv, dlambda


def selftest_wait_timeout(dev_status: torch.Tensor, timeout_us: int = 1000, stream=None) -> int:
    """Launch the bounded-wait self-test; returns the launch status."""
    return int(load().relation_selftest_wait_timeout(
        _status(dev_status, torch.cuda.current_device()), int(timeout_us), _stream(stream)))


class RelationFunction(torch.autograd.Function):
    """Autograd wrapper: Y = Relation(q, k, v; lambda).  lambda is a 1-element tensor
    (its gradient is returned); tau_S is a constant."""

    @staticmethod
    def forward(ctx, q, k, v, lam, tau_s=2.0, kernel="auto"):
        y, logz = fwd(q, k, v, float(lam), tau_s, kernel=kernel)
        ctx.save_for_backward(q, k, v, y, logz)
        ctx.lam, ctx.tau_s, ctx.kernel = float(lam), tau_s, kernel
        return y

    @staticmethod
    def backward(ctx, dy):
        q, k, v, y, logz = ctx.saved_tensors
        if dy.stride() != q.stride() or dy.dtype != q.dtype:
            dy = _like(q).copy_(dy)
        dq, dk, dv, dl = bwd(q, k, v, y, dy, logz, ctx.lam, ctx.tau_s, kernel=ctx.kernel)
        return dq, dk, dv, dl.reshape(()).to(torch.float32), None, None
