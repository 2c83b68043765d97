"""Python binding of ``libloca.so`` (argument marshalling only).

Every function here has the name of the C entry point it calls (``include/loca.h``), checks
the tensors it is given (device, dtype, shape, contiguity), passes their device pointers and
the current torch stream, and raises :class:`LocaError` on a non-OK status.  All arithmetic
of the hot path runs in the library's CUDA kernels; PyTorch only provides device memory and
streams.  There is no CPU fallback: importing works without a GPU, calling needs one.

Without ``stream`` a call goes to the current torch stream, else to that one; scratch memory that a call
allocates itself belongs to the stream it goes to.  What the caller hands over follows torch's rules:
work on another stream has to come after the work that made it, and its memory has to live until then.
"""

from __future__ import annotations

import ctypes
import functools
import os

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libloca.so")
LIB_DEBUG_PATH = os.path.join(_PKG, "libloca_debug.so")  # built with -DLOCA_DEBUG (bounds checks)

LOCA_F32 = 0
LOCA_BF16 = 1
ACTIVATIONS = {"silu": 0, "gelu": 1}  # LOCA_ACT_SILU, LOCA_ACT_GELU (the tanh form)

STATUS_NAMES = {
    0: "LOCA_OK", 1: "LOCA_ERR_INVALID_ARG", 2: "LOCA_ERR_SHAPE", 3: "LOCA_ERR_ALIGNMENT",
    4: "LOCA_ERR_UNSUPPORTED_DTYPE", 5: "LOCA_ERR_CUDA", 6: "LOCA_ERR_TIMEOUT",
    7: "LOCA_ERR_WORKSPACE", 8: "LOCA_ERR_UNSUPPORTED", 9: "LOCA_ERR_NUMERIC", 10: "LOCA_ERR_BOUNDS",
}

# (name, restype, argtypes) of every exported entry point
_P = ctypes.c_void_p
_I32 = ctypes.c_int32
_I64 = ctypes.c_int64
_SZ = ctypes.c_size_t
_F = ctypes.c_float
SIGNATURES = [
    ("loca_version", ctypes.c_int, []),
    ("loca_last_error_string", ctypes.c_char_p, []),
    ("loca_device_status", ctypes.c_int, [ctypes.POINTER(_I32), _P]),
    ("loca_debug_build", ctypes.c_int, []),
    ("loca_set_wait_limit", ctypes.c_int, [ctypes.c_uint64]),
    ("loca_error", ctypes.c_int, [_P, ctypes.c_int, _I64, _I64, _I64, _P, _I32, _P, _P, ctypes.c_int, _P, _P, _P]),
    ("loca_targets_workspace_size", ctypes.c_int, [_I64, _I32, _I64, ctypes.POINTER(_SZ)]),
    ("loca_targets", ctypes.c_int, [_P, _I64, _I32, _P, _P, _I32, _I32, _I64, _P, ctypes.c_int, _P, _P, _SZ, _P]),
    ("loca_accumulate_workspace_size", ctypes.c_int, [_I32, _I64, _I64, ctypes.c_int, ctypes.POINTER(_SZ)]),
    ("loca_accumulate", ctypes.c_int,
     [_P, _P, ctypes.c_int, _I32, _I64, _I64, _P, _F, ctypes.c_int, _P, _P, _P, _P, _SZ, _P]),
    ("loca_accumulate_noalloc", ctypes.c_int,
     [_P, _P, ctypes.c_int, _I32, _I64, _I64, _P, _F, ctypes.c_int, _P, _P, _P, _P]),
    ("loca_accumulate_streamed", ctypes.c_int,
     [_P, _P, _P, ctypes.c_int, _I32, _I64, _I64, _I32, _P, _F, ctypes.c_int, _P, _P, _P, _P, _SZ, _P]),
    ("loca_alignment_workspace_size", ctypes.c_int, [_I64, _I32, _I64, _I32, _I32, ctypes.POINTER(_SZ)]),
    ("loca_alignment", ctypes.c_int, [_P, _P, _I64, _I32, _I64, _I32, _P, _P, _I32, _P, _P, _SZ, _P]),
    ("loca_kspace_workspace_size", ctypes.c_int, [_I32, _I64, _I64, _I32, _I32, _I32, ctypes.POINTER(_SZ)]),
    ("loca_kspace_accumulate", ctypes.c_int,
     [_P, ctypes.c_int, _I32, _I64, _I64, _P, _I32, _P, _I32, _P, _P, _I32, _F, ctypes.c_int, _P, _P, _P, _P, _P,
      _SZ, _P]),
    ("loca_kspace_solve", ctypes.c_int,
     [_P, _P, _P, _P, _P, _P, ctypes.POINTER(_F), _I32, _I32, _I64, _I32, _I32, _I32, _P, _P, _P, _P]),
    ("loca_host_alloc", ctypes.c_int, [_SZ, ctypes.POINTER(ctypes.c_void_p)]),
    ("loca_host_free", ctypes.c_int, [_P]),
    ("loca_batch_step_workspace_size", ctypes.c_int, [_I32, ctypes.POINTER(_SZ)]),
    ("loca_batch_step", ctypes.c_int, [_P, ctypes.c_int, _I32, _I64, _I64, _P, _F, ctypes.c_int, _P, _P, _P, _SZ, _P]),
    ("loca_gram_cross_workspace_size", ctypes.c_int, [ctypes.POINTER(_SZ)]),
    ("loca_gram_cross", ctypes.c_int,
     [_P, _P, ctypes.c_int, _I32, _I64, _I64, _P, ctypes.c_int, _P, _P, _P, _SZ, _P]),
    ("loca_targets_sq_workspace_size", ctypes.c_int, [_I64, _I32, ctypes.POINTER(_SZ)]),
    ("loca_targets_sq", ctypes.c_int, [_P, _I64, _I32, _P, _P, _I32, _I32, _I64, _P, _P, _SZ, _P]),
    ("loca_gram_cross_fused_workspace_size", ctypes.c_int, [_I32, _I64, _I32, ctypes.POINTER(_SZ)]),
    ("loca_gram_cross_fused", ctypes.c_int,
     [_P, ctypes.c_int, _I32, _I64, _I64, _P, _I32, _P, _P, _I32, _P, ctypes.c_int, _P, _P, _P, _SZ, _P]),
    ("loca_ridge_solve_workspace_size", ctypes.c_int, [_I32, _I64, _I32, ctypes.POINTER(_SZ)]),
    ("loca_ridge_solve", ctypes.c_int,
     [_P, _P, _P, _P, _P, _P, ctypes.POINTER(_F), _I32, _I32, _I64, _I32, _P, _P, _P, _P, _P, _SZ, _P]),
    ("loca_step_from_gram", ctypes.c_int, [_P, _I32, _I64, _P, _F, _P, _P, _P]),
    ("loca_calib_fit_workspace_size", ctypes.c_int, [_I64, _I32, _I64, _I32, _I32, ctypes.POINTER(_SZ)]),
    ("loca_calib_fit", ctypes.c_int,
     [_P, _P, _I64, _I32, _I64, _I32, _F, _I32, _P, _P, _P, _P, _SZ, _P]),
    ("loca_calib_fit_rsvd_workspace_size", ctypes.c_int, [_I64, _I32, _I64, _I32, _I32, _I32, ctypes.POINTER(_SZ)]),
    ("loca_calib_fit_rsvd", ctypes.c_int,
     [_P, _P, _I64, _I32, _I64, _I32, _F, _I32, _I32, _I32, _P, _P, _P, _P, _P, _SZ, _P]),
    ("loca_head_loss_workspace_size", ctypes.c_int, [_I64, _I64, _I64, _I32, ctypes.POINTER(_SZ)]),
    ("loca_head_loss", ctypes.c_int,
     [_P, _I64, _I64, _I64, _P, _I64, _P, _P, _P, _I32, _P, _P, _P, _P, _SZ, _P]),
    ("loca_head_loss_backward_workspace_size", ctypes.c_int,
     [_I64, _I64, _I64, ctypes.c_int, ctypes.c_int, ctypes.POINTER(_SZ)]),
    ("loca_head_loss_backward", ctypes.c_int,
     [_P, _I64, _I64, _I64, _P, _I64, _P, _P, _P, _P, _F, _P, _I64, _P, _P, _SZ, _P]),
    ("loca_head_distill_workspace_size", ctypes.c_int, [_I64, _I64, _I64, _I32, ctypes.POINTER(_SZ)]),
    ("loca_head_distill", ctypes.c_int,
     [_P, _I64, _I64, _I64, _P, _I64, _P, _P, _I32, _F, _P, _P, _P, _P, _SZ, _P]),
    ("loca_head_distill_backward_workspace_size", ctypes.c_int,
     [_I64, _I64, _I64, _I32, ctypes.c_int, ctypes.c_int, ctypes.POINTER(_SZ)]),
    ("loca_head_distill_backward", ctypes.c_int,
     [_P, _I64, _I64, _I64, _P, _I64, _P, _P, _I32, _F, _P, _P, _P, _F, _P, _I64, _P, _P, _SZ, _P]),
    ("loca_adapter_packed_size", ctypes.c_int, [_I32, _I64, _I64, _I32, ctypes.POINTER(_SZ)]),
    ("loca_adapter_pack", ctypes.c_int, [_P, _P, ctypes.c_int, _I32, _I64, _I64, _I32, _P, _P, _P]),
    ("loca_adapter_plan_size", ctypes.c_int, [_I64, _I32, ctypes.POINTER(_SZ)]),
    ("loca_adapter_plan", ctypes.c_int, [_P, _I64, _I32, _P, _P]),
    ("loca_adapter_workspace_size", ctypes.c_int,
     [_I64, _I64, _I64, _I32, _I32, ctypes.c_int, ctypes.POINTER(_SZ)]),
    ("loca_adapter_apply", ctypes.c_int,
     [_P, _I64, _I64, _I64, _P, _I64, _P, _I32, _I32, _P, _P, _I64, _P, _SZ, _P]),
    ("loca_adapter_backward", ctypes.c_int,
     [_P, _I64, _P, _I64, _I64, _I64, _P, _I64, _P, _I32, _I32, _P, _P, _I64, _P, _P, ctypes.c_int, _P, _SZ, _P]),
    ("loca_q4_packed_size", ctypes.c_int, [_I64, _I64, _I32, ctypes.c_int, ctypes.c_int, ctypes.POINTER(_SZ)]),
    ("loca_q4_pack", ctypes.c_int, [_P, _P, ctypes.c_int, _P, _I64, _I64, _I32, _P, _P]),
    ("loca_q4_workspace_size", ctypes.c_int, [_I64, _I64, _I64, _I32, _I32, ctypes.POINTER(_SZ)]),
    ("loca_q4_apply", ctypes.c_int,
     [_P, _I64, _I64, _I64, _P, _I64, _I32, ctypes.c_int, ctypes.c_int, _P, _I32, _I32, _P, _P, _I64, _P, _SZ, _P]),
    ("loca_gated_workspace_size", ctypes.c_int, [_I64, _I64, _I64, ctypes.POINTER(_SZ)]),
    ("loca_gated", ctypes.c_int,
     [_P, _I64, _I64, _I64, _P, _P, _I64, ctypes.c_int, _P, _I64, _P, _SZ, _P]),
    ("loca_gated_backward_workspace_size", ctypes.c_int,
     [_I64, _I64, _I64, ctypes.c_int, ctypes.c_int, ctypes.POINTER(_SZ)]),
    ("loca_gated_backward", ctypes.c_int,
     [_P, _I64, _I64, _I64, _P, _P, _I64, ctypes.c_int, _P, _I64, _P, _I64, _P, _P, _P, _SZ, _P]),
    ("loca_grad_clip_workspace_size", ctypes.c_int, [_I32, ctypes.POINTER(_SZ)]),
    ("loca_grad_clip", ctypes.c_int, [_P, _P, _P, _P, _I32, _F, _P, _P, _SZ, _P]),
]


class LocaError(RuntimeError):
    def __init__(self, status: int, where: str, message: str):
        self.status = status
        super().__init__(f"{where}: {STATUS_NAMES.get(status, status)}: {message}")


_lib = None
_loaded = {}


def _load(path: str) -> ctypes.CDLL:
    if path not in _loaded:
        if not os.path.exists(path):
            raise RuntimeError(f"{path} is not built: run __graft_entry__.build() (nvcc, sm_103a)")
        h = ctypes.CDLL(path)
        for name, res, args in SIGNATURES:
            fn = getattr(h, name)
            fn.restype = res
            fn.argtypes = args
        _loaded[path] = h
    return _loaded[path]


def lib() -> ctypes.CDLL:
    """The library every function here calls: ``libloca.so`` (built in-tree by
    ``_build.build()``) unless :func:`use_debug_library` switched it; fails loudly if missing."""
    global _lib
    if _lib is None:
        _lib = _load(LIB_PATH)
    return _lib


def use_debug_library(on: bool = True) -> ctypes.CDLL:
    """Route every function of this module to ``libloca_debug.so`` (``_build.build(debug=True)``:
    the same entry points with index bounds checks reported as LOCA_ERR_BOUNDS by
    :func:`loca_device_status`), or back to ``libloca.so``.  Each library keeps its own device
    status word; returns the library now in use."""
    global _lib
    _lib = _load(LIB_DEBUG_PATH if on else LIB_PATH)
    return _lib


def loca_debug_build() -> bool:
    """True when the library in use is the LOCA_DEBUG build."""
    return bool(lib().loca_debug_build())


def _check(rc: int, where: str):
    if rc != 0:
        msg = lib().loca_last_error_string().decode(errors="replace")
        raise LocaError(rc, where, msg)


def _ptr(t):
    return None if t is None else t.data_ptr()


# handle of the current stream without building a Stream object (3 us of a call that takes 6)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


# the current device of a process that has CUDA tensors (a third of torch.cuda.current_device()'s 0.26 us)
_get_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _stream(stream):
    if stream is None:
        if _raw_stream is not None:
            return ctypes.c_void_p(_raw_stream(torch.cuda.current_device()))
        stream = torch.cuda.current_stream()
    return ctypes.c_void_p(stream.cuda_stream)


def _dev(t, name, dtype=None, ndim=None):
    if t is None:
        return
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA tensor")
    if dtype is not None and t.dtype not in (dtype if isinstance(dtype, tuple) else (dtype,)):
        raise TypeError(f"{name} has dtype {t.dtype}, expected {dtype}")
    if ndim is not None and t.dim() != ndim:
        raise ValueError(f"{name} must have {ndim} dimensions, got {tuple(t.shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")


def _code(dtype) -> int:
    if dtype == torch.float32:
        return LOCA_F32
    if dtype == torch.bfloat16:
        return LOCA_BF16
    raise TypeError(f"unsupported dtype {dtype}")


def _torch_stream(stream):
    """``stream`` (any object with a ``cuda_stream`` handle) as torch's own type."""
    return stream if isinstance(stream, torch.cuda.Stream) else torch.cuda.ExternalStream(stream.cuda_stream)


def _empty(nbytes: int, device, stream=None):
    """Device memory that belongs to the stream of the call that uses it (``None``: the current one):
    what is allocated on the current stream after the call cannot get it while that call runs."""
    if stream is None:
        return torch.empty(nbytes, dtype=torch.uint8, device=device)
    with torch.cuda.stream(_torch_stream(stream)):
        return torch.empty(nbytes, dtype=torch.uint8, device=device)


class _Owned:
    """Device memory of an object of this module (:func:`_empty`), which may go out of scope while calls that use it
    wait: the allocator is told of every stream of theirs but the one that the memory belongs to, once of each."""

    def __init__(self, buf, stream=None):
        self.buf, self.streams = buf, {_stream(stream).value}


def _use(stream, *kept):
    """Handle of the call's stream, on which it uses the memory of the objects ``kept`` (``None``: none)."""
    on = _stream(stream)
    for k in kept:
        if k is not None and on.value not in k._memory.streams:
            k._memory.buf.record_stream(torch.cuda.current_stream() if stream is None else _torch_stream(stream))
            k._memory.streams.add(on.value)
    return on


def _workspace(nbytes: int, device, given=None, stream=None):
    if nbytes == 0:
        return None
    if given is not None:
        if not isinstance(given, torch.Tensor) or not given.is_cuda or not given.is_contiguous():
            raise TypeError("workspace must be a contiguous CUDA tensor")
        if given.numel() * given.element_size() < nbytes:
            raise ValueError(f"workspace has {given.numel() * given.element_size()} bytes, need {nbytes}")
        return given
    return _empty(nbytes, device, stream)


def loca_version() -> int:
    return lib().loca_version()


def loca_device_status(stream=None) -> int:
    """Read and clear the device status word (LOCA_OK or a device-side code: LOCA_ERR_TIMEOUT,
    LOCA_ERR_NUMERIC, or in the debug build LOCA_ERR_BOUNDS, whose source line
    :func:`loca_last_error` then names)."""
    out = ctypes.c_int32(0)
    _check(lib().loca_device_status(ctypes.byref(out), _stream(stream)), "loca_device_status")
    return out.value


def loca_last_error() -> str:
    """Message of the last non-OK status of the calling thread (``loca_last_error_string``)."""
    return lib().loca_last_error_string().decode(errors="replace")


def loca_set_wait_limit(ns: int):
    """Test hook: how long a device wait of the tensor-core kernels may take before it
    gives up with LOCA_ERR_TIMEOUT (0 restores the default of 4 s)."""
    _check(lib().loca_set_wait_limit(int(ns)), "loca_set_wait_limit")


def loca_error(logits, label_cols, y, E, w=None, ce=None, normaliser=0, stream=None):
    """Top-layer error at the head: fills ``E`` (N x C float) and optionally ``ce`` (N)."""
    if not isinstance(logits, torch.Tensor) or not logits.is_cuda:
        raise TypeError("logits must be a CUDA tensor")
    if logits.dtype not in (torch.float32, torch.bfloat16):
        raise TypeError(f"logits has dtype {logits.dtype}, expected float32 or bfloat16")
    if logits.dim() != 2 or logits.stride(1) != 1 or logits.stride(0) < logits.shape[1]:
        raise ValueError("logits must be 2-D with unit column stride and row pitch >= V")
    _dev(label_cols, "label_cols", torch.int32, 1)
    _dev(y, "y", torch.int32, 1)
    _dev(E, "E", torch.float32, 2)
    _dev(w, "w", torch.float32, 1)
    _dev(ce, "ce", torch.float32, 1)
    N, V = logits.shape
    C = label_cols.numel()
    if E.shape != (N, C) or y.numel() != N:
        raise ValueError("E must be N x C and y must have N entries")
    rc = lib().loca_error(_ptr(logits), _code(logits.dtype), N, V, logits.stride(0), _ptr(label_cols), C,
                          _ptr(y), _ptr(w), int(normaliser), _ptr(E), _ptr(ce), _stream(stream))
    _check(rc, "loca_error")


def targets_workspace_size(N, L, d) -> int:
    out = ctypes.c_size_t(0)
    _check(lib().loca_targets_workspace_size(N, L, d, ctypes.byref(out)), "loca_targets_workspace_size")
    return out.value


def loca_targets(E, P, Q, T, tsq=None, workspace=None, stream=None):
    """Feedback targets ``T_l = (E P_l) Q_l`` into ``T`` (L x N x d, bf16 or f32) and
    ``tsq`` (L, float64, optional).  A workspace is always used (allocated if not given)."""
    _dev(E, "E", torch.float32, 2)
    _dev(P, "P", torch.float32, 3)
    _dev(Q, "Q", torch.float32, 3)
    _dev(T, "T", (torch.float32, torch.bfloat16), 3)
    _dev(tsq, "tsq", torch.float64, 1)
    N, C = E.shape
    L, C2, r = P.shape
    L2, r2, d = Q.shape
    if C2 != C or L2 != L or r2 != r or tuple(T.shape) != (L, N, d):
        raise ValueError("shape mismatch among E (N x C), P (L x C x r), Q (L x r x d), T (L x N x d)")
    nbytes = targets_workspace_size(N, L, d)
    ws = _workspace(nbytes, E.device, workspace, stream)
    rc = lib().loca_targets(_ptr(E), N, C, _ptr(P), _ptr(Q), L, r, d, _ptr(T), _code(T.dtype), _ptr(tsq),
                            _ptr(ws), nbytes, _stream(stream))
    _check(rc, "loca_targets")


def accumulate_workspace_size(L, N, d, dtype) -> int:
    out = ctypes.c_size_t(0)
    _check(lib().loca_accumulate_workspace_size(L, N, d, _code(dtype), ctypes.byref(out)),
           "loca_accumulate_workspace_size")
    return out.value


def loca_accumulate(X, T, tsq, eta, gram, cross, xsq_total, zero_first, workspace=None, stream=None):
    """Add one mini-batch to the Gram / cross statistics of every block."""
    _dev(X, "X", (torch.float32, torch.bfloat16), 3)
    _dev(T, "T", X.dtype, 3)
    _dev(tsq, "tsq", torch.float64, 1)
    _dev(gram, "gram", torch.float32, 3)
    _dev(cross, "cross", torch.float32, 3)
    _dev(xsq_total, "xsq_total", torch.float64, 1)
    L, N, d = X.shape
    if tuple(T.shape) != (L, N, d) or tuple(gram.shape) != (L, d, d) or tuple(cross.shape) != (L, d, d):
        raise ValueError("shape mismatch among X, T (L x N x d) and gram, cross (L x d x d)")
    nbytes = accumulate_workspace_size(L, N, d, X.dtype)
    ws = _workspace(nbytes, X.device, workspace, stream)
    rc = lib().loca_accumulate(_ptr(X), _ptr(T), _code(X.dtype), L, N, d, _ptr(tsq), float(eta), int(bool(zero_first)),
                               _ptr(gram), _ptr(cross), _ptr(xsq_total), _ptr(ws), nbytes, _stream(stream))
    _check(rc, "loca_accumulate")


def loca_accumulate_noalloc(X, T, tsq, eta, gram, cross, xsq_total, zero_first, stream=None):
    """loca_accumulate without a workspace, for callers that cannot allocate device memory when
    they call the library; its scratch is a fixed array inside the library (L <= 64 blocks).
    Calls that may overlap on the GPU share that array and must be serialised."""
    _dev(X, "X", (torch.float32, torch.bfloat16), 3)
    _dev(T, "T", X.dtype, 3)
    _dev(tsq, "tsq", torch.float64, 1)
    _dev(gram, "gram", torch.float32, 3)
    _dev(cross, "cross", torch.float32, 3)
    _dev(xsq_total, "xsq_total", torch.float64, 1)
    L, N, d = X.shape
    if tuple(T.shape) != (L, N, d) or tuple(gram.shape) != (L, d, d) or tuple(cross.shape) != (L, d, d):
        raise ValueError("shape mismatch among X, T (L x N x d) and gram, cross (L x d x d)")
    rc = lib().loca_accumulate_noalloc(_ptr(X), _ptr(T), _code(X.dtype), L, N, d, _ptr(tsq), float(eta),
                                       int(bool(zero_first)), _ptr(gram), _ptr(cross), _ptr(xsq_total),
                                       _stream(stream))
    _check(rc, "loca_accumulate_noalloc")


class _HostBlock:
    """Owns one loca_host_alloc buffer; freed when the last tensor viewing it is gone."""

    def __init__(self, nbytes):
        p = ctypes.c_void_p(0)
        _check(lib().loca_host_alloc(nbytes, ctypes.byref(p)), "loca_host_alloc")
        self.ptr = p.value

    def __del__(self):
        if getattr(self, "ptr", None):
            lib().loca_host_free(ctypes.c_void_p(self.ptr))
            self.ptr = None


def host_empty(shape, dtype):
    """A CPU tensor in loca_host_alloc memory (page-locked, 2 MiB pages, zero-filled): host
    inputs in it copy to the GPU at the full link rate."""
    shape = tuple(int(s) for s in shape)
    n = 1
    for s in shape:
        n *= s
    nbytes = n * torch.empty((), dtype=dtype).element_size()
    if nbytes == 0:
        return torch.empty(shape, dtype=dtype)
    owner = _HostBlock(nbytes)
    buf = (ctypes.c_uint8 * nbytes).from_address(owner.ptr)
    buf.owner = owner  # the tensor keeps `buf` alive, `buf` keeps the allocation
    return torch.frombuffer(buf, dtype=dtype).view(shape)


def loca_accumulate_streamed(X_host, staging, T, tsq, eta, gram, cross, xsq_total, zero_first, group=2,
                             workspace=None, stream=None):
    """loca_accumulate with X in host memory: X_host (L x N x d, CPU tensor, ideally pinned) is
    copied to the device `group` blocks at a time into `staging` (a device tensor with room for
    2 x group x N x d elements, used as two alternating slots) while the statistics of the
    previous group run on the stream."""
    if not isinstance(X_host, torch.Tensor) or X_host.is_cuda or X_host.dim() != 3 or not X_host.is_contiguous():
        raise TypeError("X_host must be a contiguous 3-D CPU tensor")
    _dev(staging, "staging", X_host.dtype)
    _dev(T, "T", X_host.dtype, 3)
    _dev(tsq, "tsq", torch.float64, 1)
    _dev(gram, "gram", torch.float32, 3)
    _dev(cross, "cross", torch.float32, 3)
    _dev(xsq_total, "xsq_total", torch.float64, 1)
    L, N, d = X_host.shape
    group = max(1, min(int(group), L))
    if tuple(T.shape) != (L, N, d) or tuple(gram.shape) != (L, d, d) or tuple(cross.shape) != (L, d, d):
        raise ValueError("shape mismatch among X_host, T (L x N x d) and gram, cross (L x d x d)")
    if staging.numel() < 2 * group * N * d:
        raise ValueError(f"staging has {staging.numel()} elements, need 2 x group x N x d = {2 * group * N * d}")
    nbytes = accumulate_workspace_size(L, N, d, X_host.dtype)
    ws = _workspace(nbytes, T.device, workspace, stream)
    rc = lib().loca_accumulate_streamed(ctypes.c_void_p(X_host.data_ptr()), _ptr(staging), _ptr(T),
                                        _code(X_host.dtype), L, N, d, group, _ptr(tsq), float(eta),
                                        int(bool(zero_first)), _ptr(gram), _ptr(cross), _ptr(xsq_total),
                                        _ptr(ws), nbytes, _stream(stream))
    _check(rc, "loca_accumulate_streamed")


def loca_alignment(E_probe, G_probe, P, Q, alpha, workspace=None, stream=None):
    """Per-block cosine between the feedback predictions E P_l Q_l and the probe gradients."""
    _dev(E_probe, "E_probe", torch.float32, 2)
    _dev(G_probe, "G_probe", torch.float32, 3)
    _dev(P, "P", torch.float32, 3)
    _dev(Q, "Q", torch.float32, 3)
    _dev(alpha, "alpha", torch.float64, 1)
    Np, m = E_probe.shape
    L, _, d = G_probe.shape
    r = P.shape[2]
    if (tuple(G_probe.shape) != (L, Np, d) or tuple(P.shape) != (L, m, r) or tuple(Q.shape) != (L, r, d)
            or alpha.numel() != L):
        raise ValueError("shape mismatch among E_probe, G_probe, P, Q, alpha")
    out = ctypes.c_size_t(0)
    _check(lib().loca_alignment_workspace_size(Np, m, d, L, r, ctypes.byref(out)), "loca_alignment_workspace_size")
    ws = _workspace(out.value, G_probe.device, workspace, stream)
    rc = lib().loca_alignment(_ptr(E_probe), _ptr(G_probe), Np, m, d, L, _ptr(P), _ptr(Q), r, _ptr(alpha), _ptr(ws),
                              out.value, _stream(stream))
    _check(rc, "loca_alignment")


def kspace_workspace_size(L, N, d, k, C, r) -> int:
    out = ctypes.c_size_t(0)
    _check(lib().loca_kspace_workspace_size(L, N, d, k, C, r, ctypes.byref(out)), "loca_kspace_workspace_size")
    return out.value


def loca_kspace_accumulate(X, A, E, P, Q, eta, G, SC, xsq_total, zero_first, alpha=None, workspace=None,
                           stream=None):
    """The paper's k-space statistics of one mini-batch: G_l (+)= (X_l A_l)^T (X_l A_l),
    SC_l (+)= alpha_l E^T (X_l A_l), xsq_total (+)= ||X_l||^2, with alpha_l = -eta RMS(X_l)/RMS(T_l)
    and T_l = E P_l Q_l never formed."""
    _dev(X, "X", torch.bfloat16, 3)
    _dev(A, "A", torch.float32, 3)
    _dev(E, "E", torch.float32, 2)
    _dev(P, "P", torch.float32, 3)
    _dev(Q, "Q", torch.float32, 3)
    _dev(G, "G", torch.float32, 3)
    _dev(SC, "SC", torch.float32, 3)
    _dev(xsq_total, "xsq_total", torch.float64, 1)
    _dev(alpha, "alpha", torch.float32, 1)
    L, N, d = X.shape
    k = A.shape[2]
    C, r = P.shape[1], P.shape[2]
    if (tuple(A.shape) != (L, d, k) or tuple(E.shape) != (N, C) or tuple(Q.shape) != (L, r, d)
            or tuple(G.shape) != (L, k, k) or tuple(SC.shape) != (L, C, k) or P.shape[0] != L):
        raise ValueError("shape mismatch among X, A, E, P, Q, G, SC")
    nbytes = kspace_workspace_size(L, N, d, k, C, r)
    ws = _workspace(nbytes, X.device, workspace, stream)
    rc = lib().loca_kspace_accumulate(_ptr(X), LOCA_BF16, L, N, d, _ptr(A), k, _ptr(E), C, _ptr(P), _ptr(Q), r,
                                      float(eta), int(bool(zero_first)), _ptr(G), _ptr(SC), _ptr(xsq_total),
                                      _ptr(alpha), _ptr(ws), nbytes, _stream(stream))
    _check(rc, "loca_kspace_accumulate")


def loca_kspace_solve(G, SC, P, Q, lambda_rel, B, info, xsq_total=None, B_prev=None, C_out=None, stream=None):
    """Ridge solves from the k-space statistics: B[j, l] (G_l + lambda_j I) = C_l with
    C_l = B_prev,l G_l + Q_l^T (P_l^T SC_l); lambda_j = lambda_rel[j] xsq_total[l] / d."""
    _dev(G, "G", torch.float32, 3)
    _dev(SC, "SC", torch.float32, 3)
    _dev(P, "P", torch.float32, 3)
    _dev(Q, "Q", torch.float32, 3)
    _dev(B, "B", torch.float32, 4)
    _dev(info, "info", torch.int32, 2)
    _dev(xsq_total, "xsq_total", torch.float64, 1)
    _dev(B_prev, "B_prev", torch.float32, 3)
    _dev(C_out, "C_out", torch.float32, 3)
    L, k, _ = G.shape
    C, r = P.shape[1], P.shape[2]
    d = Q.shape[2]
    lam = [float(v) for v in lambda_rel]
    nl = len(lam)
    if tuple(B.shape) != (nl, L, d, k) or tuple(info.shape) != (nl, L) or tuple(SC.shape) != (L, C, k):
        raise ValueError("shape mismatch among G, SC, Q, B, info")
    arr = (ctypes.c_float * nl)(*lam)
    rc = lib().loca_kspace_solve(_ptr(G), _ptr(SC), _ptr(xsq_total), _ptr(P), _ptr(Q), _ptr(B_prev), arr, nl, L, d,
                                 k, C, r, _ptr(B), _ptr(info), _ptr(C_out), _stream(stream))
    _check(rc, "loca_kspace_solve")


def batch_step_workspace_size(L) -> int:
    out = ctypes.c_size_t(0)
    _check(lib().loca_batch_step_workspace_size(L, ctypes.byref(out)), "loca_batch_step_workspace_size")
    return out.value


def loca_batch_step(X, tsq, eta, xsq_total, alpha, zero_first, workspace=None, stream=None):
    """Step of Eq. 10 for one mini-batch: ``alpha[l] = -eta ||X_l|| / sqrt(tsq[l])``; updates
    ``xsq_total``."""
    _dev(X, "X", (torch.float32, torch.bfloat16), 3)
    _dev(tsq, "tsq", torch.float64, 1)
    _dev(xsq_total, "xsq_total", torch.float64, 1)
    _dev(alpha, "alpha", torch.float32, 1)
    L, N, d = X.shape
    nbytes = batch_step_workspace_size(L)
    ws = _workspace(nbytes, X.device, workspace, stream)
    rc = lib().loca_batch_step(_ptr(X), _code(X.dtype), L, N, d, _ptr(tsq), float(eta), int(bool(zero_first)),
                               _ptr(xsq_total), _ptr(alpha), _ptr(ws), nbytes, _stream(stream))
    _check(rc, "loca_batch_step")


def gram_cross_workspace_size() -> int:
    out = ctypes.c_size_t(0)
    _check(lib().loca_gram_cross_workspace_size(ctypes.byref(out)), "loca_gram_cross_workspace_size")
    return out.value


def loca_gram_cross(X, T, alpha, gram, cross, zero_first, workspace=None, stream=None):
    """Statistics of Eq. 9 for one mini-batch with the step ``alpha`` of loca_batch_step."""
    _dev(X, "X", (torch.float32, torch.bfloat16), 3)
    _dev(T, "T", X.dtype, 3)
    _dev(alpha, "alpha", torch.float32, 1)
    _dev(gram, "gram", torch.float32, 3)
    _dev(cross, "cross", torch.float32, 3)
    L, N, d = X.shape
    if tuple(T.shape) != (L, N, d) or tuple(gram.shape) != (L, d, d) or tuple(cross.shape) != (L, d, d):
        raise ValueError("shape mismatch among X, T (L x N x d) and gram, cross (L x d x d)")
    nbytes = gram_cross_workspace_size()
    ws = _workspace(nbytes, X.device, workspace, stream)
    rc = lib().loca_gram_cross(_ptr(X), _ptr(T), _code(X.dtype), L, N, d, _ptr(alpha), int(bool(zero_first)),
                               _ptr(gram), _ptr(cross), _ptr(ws), nbytes, _stream(stream))
    _check(rc, "loca_gram_cross")


def targets_sq_workspace_size(N, C) -> int:
    out = ctypes.c_size_t(0)
    _check(lib().loca_targets_sq_workspace_size(N, C, ctypes.byref(out)), "loca_targets_sq_workspace_size")
    return out.value


def loca_targets_sq(E, P, Q, tsq, workspace=None, stream=None):
    """``tsq[l] = ||E P_l Q_l||_F^2`` (float64, L) without forming the targets."""
    _dev(E, "E", torch.float32, 2)
    _dev(P, "P", torch.float32, 3)
    _dev(Q, "Q", torch.float32, 3)
    _dev(tsq, "tsq", torch.float64, 1)
    N, C = E.shape
    L, C2, r = P.shape
    L2, r2, d = Q.shape
    if C2 != C or L2 != L or r2 != r or tuple(tsq.shape) != (L,):
        raise ValueError("shape mismatch among E (N x C), P (L x C x r), Q (L x r x d), tsq (L)")
    nbytes = targets_sq_workspace_size(N, C)
    ws = _workspace(nbytes, E.device, workspace, stream)
    rc = lib().loca_targets_sq(_ptr(E), N, C, _ptr(P), _ptr(Q), L, r, d, _ptr(tsq), _ptr(ws), nbytes, _stream(stream))
    _check(rc, "loca_targets_sq")


def gram_cross_fused_workspace_size(L, N, r) -> int:
    out = ctypes.c_size_t(0)
    _check(lib().loca_gram_cross_fused_workspace_size(L, N, r, ctypes.byref(out)),
           "loca_gram_cross_fused_workspace_size")
    return out.value


def loca_gram_cross_fused(X, E, P, Q, alpha, gram, cross, zero_first, workspace=None, stream=None):
    """loca_gram_cross with each block's targets ``T_l = (E P_l) Q_l`` generated inside the kernel."""
    _dev(X, "X", torch.bfloat16, 3)
    _dev(E, "E", torch.float32, 2)
    _dev(P, "P", torch.float32, 3)
    _dev(Q, "Q", torch.float32, 3)
    _dev(alpha, "alpha", torch.float32, 1)
    _dev(gram, "gram", torch.float32, 3)
    _dev(cross, "cross", torch.float32, 3)
    L, N, d = X.shape
    C, r = P.shape[1], P.shape[2]
    if (tuple(E.shape) != (N, C) or tuple(P.shape) != (L, C, r) or tuple(Q.shape) != (L, r, d)
            or tuple(gram.shape) != (L, d, d) or tuple(cross.shape) != (L, d, d)):
        raise ValueError("shape mismatch among X, E, P, Q, gram, cross")
    nbytes = gram_cross_fused_workspace_size(L, N, r)
    ws = _workspace(nbytes, X.device, workspace, stream)
    rc = lib().loca_gram_cross_fused(_ptr(X), LOCA_BF16, L, N, d, _ptr(E), C, _ptr(P), _ptr(Q), r, _ptr(alpha),
                                     int(bool(zero_first)), _ptr(gram), _ptr(cross), _ptr(ws), nbytes, _stream(stream))
    _check(rc, "loca_gram_cross_fused")


def ridge_solve_workspace_size(L, d, k) -> int:
    out = ctypes.c_size_t(0)
    _check(lib().loca_ridge_solve_workspace_size(L, d, k, ctypes.byref(out)), "loca_ridge_solve_workspace_size")
    return out.value


def loca_ridge_solve(gram, cross, A, lambda_rel, B, info, xsq_total=None, B_prev=None, G_out=None, C_out=None,
                     cross_scale=None, workspace=None, stream=None):
    """Closed-form adapters ``B[j, l] = C_l (G_l + lambda_j I)^-1`` for every block and candidate;
    ``cross_scale`` (L, optional) multiplies ``cross_l``."""
    _dev(gram, "gram", torch.float32, 3)
    _dev(cross, "cross", torch.float32, 3)
    _dev(cross_scale, "cross_scale", torch.float32, 1)
    _dev(A, "A", torch.float32, 3)
    _dev(B, "B", torch.float32, 4)
    _dev(info, "info", torch.int32, 2)
    _dev(xsq_total, "xsq_total", torch.float64, 1)
    _dev(B_prev, "B_prev", torch.float32, 3)
    _dev(G_out, "G_out", torch.float32, 3)
    _dev(C_out, "C_out", torch.float32, 3)
    L, d, k = A.shape
    lam = [float(v) for v in lambda_rel]
    nl = len(lam)
    if tuple(B.shape) != (nl, L, d, k) or tuple(info.shape) != (nl, L):
        raise ValueError("B must be nl x L x d x k and info nl x L")
    lam_arr = (ctypes.c_float * max(nl, 1))(*lam)
    nbytes = ridge_solve_workspace_size(L, d, k)
    ws = _workspace(nbytes, A.device, workspace, stream)
    if cross_scale is not None and tuple(cross_scale.shape) != (L,):
        raise ValueError("cross_scale must have L entries")
    rc = lib().loca_ridge_solve(_ptr(gram), _ptr(cross), _ptr(cross_scale), _ptr(xsq_total), _ptr(A), _ptr(B_prev),
                                lam_arr, nl, L, d, k, _ptr(B), _ptr(info), _ptr(G_out), _ptr(C_out), _ptr(ws), nbytes,
                                _stream(stream))
    _check(rc, "loca_ridge_solve")


def loca_step_from_gram(gram, tsq, eta, xsq_total, alpha, stream=None):
    """Step of Eq. 10 for a pass with one mini-batch from ``tr(gram_l) = ||X_l||^2``:
    ``alpha[l] = -eta sqrt(tr(gram_l) / tsq[l])``, ``xsq_total[l] = tr(gram_l)``."""
    _dev(gram, "gram", torch.float32, 3)
    _dev(tsq, "tsq", torch.float64, 1)
    _dev(xsq_total, "xsq_total", torch.float64, 1)
    _dev(alpha, "alpha", torch.float32, 1)
    L, d, d2 = gram.shape
    if d2 != d or tuple(tsq.shape) != (L,) or tuple(xsq_total.shape) != (L,) or tuple(alpha.shape) != (L,):
        raise ValueError("gram must be L x d x d; tsq, xsq_total, alpha must have L entries")
    rc = lib().loca_step_from_gram(_ptr(gram), L, d, _ptr(tsq), float(eta), _ptr(xsq_total), _ptr(alpha),
                                   _stream(stream))
    _check(rc, "loca_step_from_gram")


def calib_fit_workspace_size(Np, m, d, L, r) -> int:
    out = ctypes.c_size_t(0)
    _check(lib().loca_calib_fit_workspace_size(Np, m, d, L, r, ctypes.byref(out)), "loca_calib_fit_workspace_size")
    return out.value


def loca_calib_fit(E_probe, G_probe, beta, r, P, Q, sigma=None, workspace=None, stream=None):
    """Rank-r feedback factors ``P`` (L x m x r), ``Q`` (L x r x d) from probe pairs."""
    _dev(E_probe, "E_probe", torch.float32, 2)
    _dev(G_probe, "G_probe", torch.float32, 3)
    _dev(P, "P", torch.float32, 3)
    _dev(Q, "Q", torch.float32, 3)
    _dev(sigma, "sigma", torch.float32, 2)
    Np, m = E_probe.shape
    L, Np2, d = G_probe.shape
    if Np2 != Np or tuple(P.shape) != (L, m, r) or tuple(Q.shape) != (L, r, d):
        raise ValueError("shape mismatch among E_probe, G_probe, P, Q")
    nbytes = calib_fit_workspace_size(Np, m, d, L, r)
    ws = _workspace(nbytes, E_probe.device, workspace, stream)
    rc = lib().loca_calib_fit(_ptr(E_probe), _ptr(G_probe), Np, m, d, L, float(beta), r, _ptr(P), _ptr(Q),
                              _ptr(sigma), _ptr(ws), nbytes, _stream(stream))
    _check(rc, "loca_calib_fit")


def calib_fit_rsvd_workspace_size(Np, m, d, L, r, ell) -> int:
    out = ctypes.c_size_t(0)
    _check(lib().loca_calib_fit_rsvd_workspace_size(Np, m, d, L, r, ell, ctypes.byref(out)),
           "loca_calib_fit_rsvd_workspace_size")
    return out.value


def loca_calib_fit_rsvd(E_probe, G_probe, beta, r, Omega, q, P, Q, sigma=None, workspace=None, stream=None):
    """Rank-r feedback factors for wide error spaces by randomized subspace iteration:
    ``Omega`` (d x ell) is the Gaussian test matrix, ``q`` the number of power iterations."""
    _dev(E_probe, "E_probe", torch.float32, 2)
    _dev(G_probe, "G_probe", torch.float32, 3)
    _dev(Omega, "Omega", torch.float32, 2)
    _dev(P, "P", torch.float32, 3)
    _dev(Q, "Q", torch.float32, 3)
    _dev(sigma, "sigma", torch.float32, 2)
    Np, m = E_probe.shape
    L, Np2, d = G_probe.shape
    ell = Omega.shape[1]
    if (Np2 != Np or Omega.shape[0] != d or tuple(P.shape) != (L, m, r) or tuple(Q.shape) != (L, r, d)
            or (sigma is not None and tuple(sigma.shape) != (L, r))):
        raise ValueError("shape mismatch among E_probe, G_probe, Omega, P, Q, sigma")
    nbytes = calib_fit_rsvd_workspace_size(Np, m, d, L, r, ell)
    ws = _workspace(nbytes, E_probe.device, workspace, stream)
    rc = lib().loca_calib_fit_rsvd(_ptr(E_probe), _ptr(G_probe), Np, m, d, L, float(beta), r, ell, int(q),
                                   _ptr(Omega), _ptr(P), _ptr(Q), _ptr(sigma), _ptr(ws), nbytes, _stream(stream))
    _check(rc, "loca_calib_fit_rsvd")


def _rows2d(t, name, dtype, shape=None):
    """A 2-D CUDA tensor with unit column stride (rows may be spaced); returns its row pitch."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} has dtype {t.dtype}, expected {dtype}")
    size, stride = t.shape, t.stride()
    if len(size) != 2 or (shape is not None and size != shape):
        raise ValueError(f"{name} must have shape {tuple(shape) if shape else '2-D'}, got {tuple(size)}")
    rows, cols = size
    if cols > 1 and stride[1] != 1:
        raise ValueError(f"{name} must have unit column stride")
    pitch = stride[0] if rows > 1 else cols
    if pitch < cols:
        raise ValueError(f"{name} must have a row pitch of at least its columns")
    return pitch


@functools.lru_cache(maxsize=1024)
def _size_on(device, name, *args) -> int:
    out = ctypes.c_size_t(0)
    _check(getattr(lib(), name)(*args, ctypes.byref(out)), name)
    return out.value


def _size(name, *args) -> int:
    """A workspace size, asked for once: it depends on the arguments and on the current device."""
    return _size_on(torch.cuda.current_device() if torch.cuda.is_initialized() else None, name, *args)


def head_loss_workspace_size(N, V, d, C=0) -> int:
    return _size("loca_head_loss_workspace_size", N, V, d, C)


def loca_head_loss(H, W, y, loss, lse=None, w=None, label_cols=None, E=None, workspace=None, stream=None):
    """Cross entropy of hidden states ``H`` (N x d bf16, rows may be spaced) against the head ``W``
    (V x d bf16) at labels ``y`` (N int32; outside [0, V) = masked) without the logits in memory:
    fills ``loss`` and ``lse`` (N float) and, for ``label_cols`` (C int32), the label-column error
    ``E`` (N x C float) that :func:`loca_targets` takes."""
    ldh = _rows2d(H, "H", torch.bfloat16)
    N, d = H.shape
    _dev(W, "W", torch.bfloat16, 2)
    _dev(y, "y", torch.int32, 1)
    _dev(loss, "loss", torch.float32, 1)
    _dev(lse, "lse", torch.float32, 1)
    _dev(w, "w", torch.float32, 1)
    _dev(label_cols, "label_cols", torch.int32, 1)
    _dev(E, "E", torch.float32, 2)
    V = W.shape[0]
    if (W.shape[1] != d or y.numel() != N or loss.numel() != N or (lse is not None and lse.numel() != N)
            or (w is not None and w.numel() != N)):
        raise ValueError("W must be V x d; y, loss, lse and w must have N entries")
    C = 0 if label_cols is None else label_cols.numel()
    if E is not None and tuple(E.shape) != (N, C):
        raise ValueError("E must be N x C for the C entries of label_cols")
    nbytes = head_loss_workspace_size(N, V, d, C)
    ws = _workspace(nbytes, H.device, workspace, stream)
    rc = lib().loca_head_loss(_ptr(H), ldh, N, d, _ptr(W), V, _ptr(y), _ptr(w), _ptr(label_cols), C, _ptr(loss),
                              _ptr(lse), _ptr(E), _ptr(ws), nbytes, _stream(stream))
    _check(rc, "loca_head_loss")


def head_loss_backward_workspace_size(N, V, d, want_dH=True, want_dW=True) -> int:
    return _size("loca_head_loss_backward_workspace_size", N, V, d, int(bool(want_dH)), int(bool(want_dW)))


def loca_head_loss_backward(H, W, y, lse, dH=None, dW=None, w=None, dloss=None, grad_scale=1.0, workspace=None,
                            stream=None):
    """Gradients of ``grad_scale * sum_n dloss[n] * loss[n]`` of :func:`loca_head_loss` for the hidden
    states (``dH``, N x d bf16, rows may be spaced) and the head (``dW``, V x d bf16), in pieces of
    the vocabulary; ``lse`` is the forward call's."""
    ldh = _rows2d(H, "H", torch.bfloat16)
    N, d = H.shape
    _dev(W, "W", torch.bfloat16, 2)
    _dev(y, "y", torch.int32, 1)
    _dev(lse, "lse", torch.float32, 1)
    _dev(w, "w", torch.float32, 1)
    _dev(dloss, "dloss", torch.float32, 1)
    lddh = 0 if dH is None else _rows2d(dH, "dH", torch.bfloat16, (N, d))
    _dev(dW, "dW", torch.bfloat16, 2)
    V = W.shape[0]
    if (W.shape[1] != d or y.numel() != N or lse.numel() != N or (w is not None and w.numel() != N)
            or (dloss is not None and dloss.numel() != N) or (dW is not None and tuple(dW.shape) != (V, d))):
        raise ValueError("W and dW must be V x d; y, lse, w and dloss must have N entries")
    nbytes = head_loss_backward_workspace_size(N, V, d, dH is not None, dW is not None)
    ws = _workspace(nbytes, H.device, workspace, stream)
    rc = lib().loca_head_loss_backward(_ptr(H), ldh, N, d, _ptr(W), V, _ptr(y), _ptr(w), _ptr(lse), _ptr(dloss),
                                       float(grad_scale), _ptr(dH), lddh, _ptr(dW), _ptr(ws), nbytes, _stream(stream))
    _check(rc, "loca_head_loss_backward")


def _same_device(*tensors):
    """The call runs on the current device: refuses tensors of another one."""
    here = _get_device()
    for t in tensors:
        if t is not None and t.get_device() != here:
            raise ValueError(f"a tensor is on {t.device}, the current device is cuda:{here}")


def head_distill_workspace_size(N, V, d, K) -> int:
    return _size("loca_head_distill_workspace_size", N, V, d, K)


def _distill_args(H, W, idx, t, w, lse):
    ldh = _rows2d(H, "H", torch.bfloat16)
    N, d = H.shape
    _dev(W, "W", torch.bfloat16, 2)
    _dev(idx, "idx", torch.int32, 2)
    _dev(t, "t", torch.float32, 2)
    _dev(w, "w", torch.float32, 1)
    _dev(lse, "lse", torch.float32, 1)
    if (W.shape[1] != d or idx.shape[0] != N or t.shape != idx.shape or (w is not None and w.numel() != N)
            or (lse is not None and lse.numel() != N)):
        raise ValueError("W must be V x d, idx and t N x K; w and lse must have N entries")
    return ldh, N, d, W.shape[0], idx.shape[1]


def loca_head_distill(H, W, idx, t, loss, lse=None, w=None, tau=1.0, workspace=None, stream=None):
    """Distillation from a teacher's top logits ``t`` (N x K float) at the words ``idx`` (N x K int32; outside
    [0, V) = none) for hidden states ``H`` (N x d bf16, rows may be spaced) and the head ``W`` (V x d bf16), without
    the student's logits in memory: ``loss = w tau^2 KL(softmax(t / tau) || softmax(H W^T / tau))`` and ``lse`` of
    the scaled logits (N float each).  A position without a word is masked."""
    ldh, N, d, V, K = _distill_args(H, W, idx, t, w, lse)
    _dev(loss, "loss", torch.float32, 1)
    if loss.numel() != N:
        raise ValueError("loss must have N entries")
    _same_device(H, W, idx, t, w, loss, lse)
    nbytes = head_distill_workspace_size(N, V, d, K)
    ws = _workspace(nbytes, H.device, workspace, stream)
    rc = lib().loca_head_distill(_ptr(H), ldh, N, d, _ptr(W), V, _ptr(idx), _ptr(t), K, float(tau), _ptr(w), _ptr(loss),
                                 _ptr(lse), _ptr(ws), nbytes, _stream(stream))
    _check(rc, "loca_head_distill")


def head_distill_backward_workspace_size(N, V, d, K, want_dH=True, want_dW=True) -> int:
    return _size("loca_head_distill_backward_workspace_size", N, V, d, K, int(bool(want_dH)), int(bool(want_dW)))


def loca_head_distill_backward(H, W, idx, t, lse, dH=None, dW=None, w=None, dloss=None, tau=1.0, grad_scale=1.0,
                               workspace=None, stream=None):
    """Gradients of ``grad_scale * sum_n dloss[n] * loss[n]`` of :func:`loca_head_distill` for the hidden states
    (``dH``, N x d bf16, rows may be spaced) and the head (``dW``, V x d bf16); ``lse`` is the forward call's."""
    ldh, N, d, V, K = _distill_args(H, W, idx, t, w, lse)
    _dev(dloss, "dloss", torch.float32, 1)
    lddh = 0 if dH is None else _rows2d(dH, "dH", torch.bfloat16, (N, d))
    _dev(dW, "dW", torch.bfloat16, 2)
    if (dloss is not None and dloss.numel() != N) or (dW is not None and tuple(dW.shape) != (V, d)):
        raise ValueError("dW must be V x d and dloss must have N entries")
    _same_device(H, W, idx, t, lse, dH, dW, w, dloss)
    nbytes = head_distill_backward_workspace_size(N, V, d, K, dH is not None, dW is not None)
    ws = _workspace(nbytes, H.device, workspace, stream)
    rc = lib().loca_head_distill_backward(_ptr(H), ldh, N, d, _ptr(W), V, _ptr(idx), _ptr(t), K, float(tau), _ptr(w),
                                          _ptr(lse), _ptr(dloss), float(grad_scale), _ptr(dH), lddh, _ptr(dW), _ptr(ws),
                                          nbytes, _stream(stream))
    _check(rc, "loca_head_distill_backward")


class AdapterSet:
    """The device layout of ``n`` adapters of one projection: ``A`` (n x d_in x k) and ``B``
    (n x d_out x k), float32 or bfloat16, each with an optional ``scale`` (n float).  Call
    :meth:`pack` once for serving and after every update in training."""

    def __init__(self, n, d_in, d_out, k, device="cuda"):
        out = ctypes.c_size_t(0)
        _check(lib().loca_adapter_packed_size(n, d_in, d_out, k, ctypes.byref(out)), "loca_adapter_packed_size")
        self.n, self.d_in, self.d_out, self.k = int(n), int(d_in), int(d_out), int(k)
        self.packed = torch.zeros(out.value, dtype=torch.uint8, device=device)
        self._memory = _Owned(self.packed)
        if not torch.cuda.is_current_stream_capturing():
            torch.cuda.current_stream().synchronize()  # the zeros come before a pack on any stream

    def pack(self, A, B, scale=None, stream=None):
        _dev(A, "A", (torch.float32, torch.bfloat16), 3)
        _dev(B, "B", A.dtype, 3)
        _dev(scale, "scale", torch.float32, 1)
        if (tuple(A.shape) != (self.n, self.d_in, self.k) or tuple(B.shape) != (self.n, self.d_out, self.k)
                or (scale is not None and scale.numel() != self.n)):
            raise ValueError("A must be n x d_in x k, B n x d_out x k and scale have n entries")
        on = _use(stream, self)
        rc = lib().loca_adapter_pack(_ptr(A), _ptr(B), _code(A.dtype), self.n, self.d_in, self.d_out, self.k, _ptr(scale),
                                     _ptr(self.packed), on)
        _check(rc, "loca_adapter_pack")
        return self


class AdapterPlan:
    """The tokens of one step grouped by adapter: ``ids`` (N int32 in any order; outside [0, n) = no
    adapter).  One plan serves every projection of the step; :meth:`update` takes the next step's
    ids of the same length."""

    def __init__(self, ids, n, stream=None):
        _dev(ids, "ids", torch.int32, 1)
        self.N, self.n = ids.numel(), int(n)
        out = ctypes.c_size_t(0)
        _check(lib().loca_adapter_plan_size(self.N, self.n, ctypes.byref(out)), "loca_adapter_plan_size")
        self.buf = _empty(max(out.value, 256), ids.device, stream)
        self._memory = _Owned(self.buf, stream)
        self.update(ids, stream=stream)

    def update(self, ids, stream=None):
        _dev(ids, "ids", torch.int32, 1)
        if ids.numel() != self.N:
            raise ValueError(f"the plan is for {self.N} tokens, got {ids.numel()}")
        on = _use(stream, self)
        rc = lib().loca_adapter_plan(_ptr(ids), self.N, self.n, _ptr(self.buf), on)
        _check(rc, "loca_adapter_plan")
        return self


def adapter_workspace_size(N, d_in, d_out, k, n, backward=False) -> int:
    return _size("loca_adapter_workspace_size", N, d_in, d_out, k, n, int(bool(backward)))


def _adapter_args(X, W, adapters, plan, stream):
    ldx = _rows2d(X, "X", torch.bfloat16)
    _dev(W, "W", torch.bfloat16, 2)
    N, d_in = X.shape
    if d_in != adapters.d_in or tuple(W.shape) != (adapters.d_out, d_in):
        raise ValueError(f"the adapters are for a {adapters.d_out} x {adapters.d_in} projection, got X {tuple(X.shape)}, "
                         f"W {tuple(W.shape)}")
    if plan.N != N or plan.n != adapters.n:
        raise ValueError(f"the plan is for {plan.N} tokens and {plan.n} adapters, got {N} and {adapters.n}")
    return ldx, N, d_in, _use(stream, adapters, plan)


def loca_adapter_apply(X, W, adapters, plan, Y, workspace=None, stream=None):
    """``Y = X W^T + s_a (X A_a) B_a^T`` for tokens with an adapter each (or none): ``X`` N x d_in and
    ``Y`` N x d_out bf16 (rows may be spaced), ``W`` d_out x d_in bf16, ``adapters`` an
    :class:`AdapterSet`, ``plan`` an :class:`AdapterPlan` of the tokens' adapters."""
    ldx, N, d_in, on = _adapter_args(X, W, adapters, plan, stream)
    ldy = _rows2d(Y, "Y", torch.bfloat16, (N, adapters.d_out))
    nbytes = adapter_workspace_size(N, d_in, adapters.d_out, adapters.k, adapters.n)
    ws = _workspace(nbytes, X.device, workspace, stream)
    rc = lib().loca_adapter_apply(_ptr(X), ldx, N, d_in, _ptr(W), adapters.d_out, _ptr(adapters.packed), adapters.n,
                                  adapters.k, _ptr(plan.buf), _ptr(Y), ldy, _ptr(ws), nbytes, on)
    _check(rc, "loca_adapter_apply")


def loca_adapter_backward(X, dY, W, adapters, plan, dX=None, dA=None, dB=None, workspace=None, stream=None):
    """Gradients of :func:`loca_adapter_apply` for the frozen projection's input (``dX``, N x d_in
    bf16) and the adapters (``dA`` n x d_in x k, ``dB`` n x d_out x k, float32 or bfloat16); the
    adapters as last packed."""
    ldx, N, d_in, on = _adapter_args(X, W, adapters, plan, stream)
    lddy = _rows2d(dY, "dY", torch.bfloat16, (N, adapters.d_out))
    lddx = 0 if dX is None else _rows2d(dX, "dX", torch.bfloat16, (N, d_in))
    both = (torch.float32, torch.bfloat16)
    _dev(dA, "dA", both, 3)
    _dev(dB, "dB", both if dA is None else dA.dtype, 3)
    if ((dA is not None and tuple(dA.shape) != (adapters.n, d_in, adapters.k))
            or (dB is not None and tuple(dB.shape) != (adapters.n, adapters.d_out, adapters.k))):
        raise ValueError("dA must be n x d_in x k and dB n x d_out x k")
    kind = torch.float32 if dA is None and dB is None else (dB if dA is None else dA).dtype
    nbytes = adapter_workspace_size(N, d_in, adapters.d_out, adapters.k, adapters.n, backward=True)
    ws = _workspace(nbytes, X.device, workspace, stream)
    rc = lib().loca_adapter_backward(_ptr(X), ldx, _ptr(dY), lddy, N, d_in, _ptr(W), adapters.d_out,
                                     _ptr(adapters.packed), adapters.n, adapters.k, _ptr(plan.buf), _ptr(dX), lddx,
                                     _ptr(dA), _ptr(dB), _code(kind), _ptr(ws), nbytes, on)
    _check(rc, "loca_adapter_backward")


class Q4Weight:
    """The device layout of a frozen projection in 4 bits: ``codes`` (d_out x d_in / 2 uint8, the even column in
    the low four bits), ``scales`` (d_out x d_in / group, float32 or bfloat16; group 32, 64 or 128) and optional
    ``zeros`` (like scales, uint8 0 .. 15; default 8), ``W = scale (code - zero)``.  Packs at once; the arguments are
    not needed afterwards, also where the stream has not come to the packing yet."""

    def __init__(self, codes, scales, zeros=None, stream=None):
        _dev(codes, "codes", torch.uint8, 2)
        _dev(scales, "scales", (torch.float32, torch.bfloat16), 2)
        _dev(zeros, "zeros", torch.uint8, 2)
        if codes is None or scales is None:
            raise TypeError("codes and scales must be CUDA tensors")
        d_out, d_in = codes.shape[0], 2 * codes.shape[1]
        groups = scales.shape[1]
        if scales.shape[0] != d_out or groups < 1 or d_in % groups != 0:
            raise ValueError(f"scales must be {d_out} x (columns / group), got {tuple(scales.shape)} for {d_in} columns")
        if zeros is not None and zeros.shape != scales.shape:
            raise ValueError("zeros must have the shape of scales")
        _same_device(codes, scales, zeros)
        self.d_out, self.d_in, self.group = d_out, d_in, d_in // groups
        self.scale_code, self.with_zeros = _code(scales.dtype), zeros is not None
        out = ctypes.c_size_t(0)
        _check(lib().loca_q4_packed_size(d_out, d_in, self.group, self.scale_code, int(self.with_zeros), ctypes.byref(out)),
               "loca_q4_packed_size")
        self.packed = _empty(out.value, codes.device, stream)
        self._memory = _Owned(self.packed, stream)
        on = torch.cuda.current_stream() if stream is None else _torch_stream(stream)
        for t in (codes, scales, zeros):
            if t is not None:
                t.record_stream(on)
        rc = lib().loca_q4_pack(_ptr(codes), _ptr(scales), self.scale_code, _ptr(zeros), d_out, d_in, self.group,
                                _ptr(self.packed), _stream(stream))
        _check(rc, "loca_q4_pack")


def q4_workspace_size(N, d_in, d_out, k=0, n=0) -> int:
    return _size("loca_q4_workspace_size", N, d_in, d_out, k, n)


def loca_q4_apply(X, weight, Y, adapters=None, plan=None, workspace=None, stream=None):
    """``Y = X W^T + s_a (X A_a) B_a^T`` for a few tokens with a 4-bit ``weight`` (a :class:`Q4Weight`): ``X`` N x d_in
    and ``Y`` N x d_out bf16 (rows may be spaced); ``adapters`` (an :class:`AdapterSet`) and ``plan`` (an
    :class:`AdapterPlan` of the tokens' adapters), or neither.  More than a few tokens too: it reads the weight again
    for every 128 of them (64 with groups below 128)."""
    ldx = _rows2d(X, "X", torch.bfloat16)
    N, d_in = X.shape
    if d_in != weight.d_in:
        raise ValueError(f"the weight has {weight.d_in} columns, X {d_in}")
    ldy = _rows2d(Y, "Y", torch.bfloat16, (N, weight.d_out))
    if (adapters is None) != (plan is None):
        raise ValueError("adapters and plan come together")
    n = k = 0
    if adapters is not None:
        n, k = adapters.n, adapters.k
        if (adapters.d_in, adapters.d_out) != (d_in, weight.d_out):
            raise ValueError(f"the adapters are for a {adapters.d_out} x {adapters.d_in} projection")
        if plan.N != N or plan.n != n:
            raise ValueError(f"the plan is for {plan.N} tokens and {plan.n} adapters, got {N} and {n}")
    _same_device(X, Y, weight.packed, None if adapters is None else adapters.packed, None if plan is None else plan.buf)
    on = _use(stream, weight, adapters, plan)
    nbytes = q4_workspace_size(N, d_in, weight.d_out, k, n)
    ws = _workspace(nbytes, X.device, workspace, stream)
    rc = lib().loca_q4_apply(_ptr(X), ldx, N, d_in, _ptr(weight.packed), weight.d_out, weight.group, weight.scale_code,
                             int(weight.with_zeros), None if adapters is None else _ptr(adapters.packed), n, k,
                             None if plan is None else _ptr(plan.buf), _ptr(Y), ldy, _ptr(ws), nbytes, on)
    _check(rc, "loca_q4_apply")


def gated_workspace_size(N, d, f) -> int:
    return _size("loca_gated_workspace_size", N, d, f)


def _gated_args(X, Wg, Wu, act):
    ldx = _rows2d(X, "X", torch.bfloat16)
    _dev(Wg, "Wg", torch.bfloat16, 2)
    _dev(Wu, "Wu", torch.bfloat16, 2)
    N, d = X.shape
    if Wg.shape[1] != d or Wu.shape != Wg.shape:
        raise ValueError(f"Wg and Wu must be f x {d}, got {tuple(Wg.shape)} and {tuple(Wu.shape)}")
    if act not in ACTIVATIONS:
        raise ValueError(f"act must be one of {sorted(ACTIVATIONS)}, got {act!r}")
    return ldx, N, d, Wg.shape[0], ACTIVATIONS[act]


def loca_gated(X, Wg, Wu, H, act="silu", workspace=None, stream=None):
    """Gated feed-forward ``H = act(X Wg^T) * (X Wu^T)`` in one launch: ``X`` N x d and ``H`` N x f bf16 (rows
    may be spaced), ``Wg`` and ``Wu`` f x d bf16; ``act`` "silu" or "gelu" (the tanh form)."""
    ldx, N, d, f, code = _gated_args(X, Wg, Wu, act)
    ldh = _rows2d(H, "H", torch.bfloat16, (N, f))
    _same_device(X, Wg, Wu, H)
    nbytes = gated_workspace_size(N, d, f)
    ws = _workspace(nbytes, X.device, workspace, stream)
    rc = lib().loca_gated(_ptr(X), ldx, N, d, _ptr(Wg), _ptr(Wu), f, code, _ptr(H), ldh, _ptr(ws), nbytes,
                          _stream(stream))
    _check(rc, "loca_gated")


def gated_backward_workspace_size(N, d, f, want_dX=True, want_dW=True) -> int:
    return _size("loca_gated_backward_workspace_size", N, d, f, int(bool(want_dX)), int(bool(want_dW)))


def loca_gated_backward(X, Wg, Wu, dH, dX=None, dWg=None, dWu=None, act="silu", workspace=None, stream=None):
    """Gradients of :func:`loca_gated` from ``dH`` (N x f bf16, rows may be spaced): ``dX`` (N x d bf16, rows
    may be spaced), ``dWg`` and ``dWu`` (f x d bf16), each optional.  Keeps nothing of the forward call: the
    pre-activations are computed again."""
    ldx, N, d, f, code = _gated_args(X, Wg, Wu, act)
    lddh = _rows2d(dH, "dH", torch.bfloat16, (N, f))
    lddx = 0 if dX is None else _rows2d(dX, "dX", torch.bfloat16, (N, d))
    _dev(dWg, "dWg", torch.bfloat16, 2)
    _dev(dWu, "dWu", torch.bfloat16, 2)
    if any(g is not None and tuple(g.shape) != (f, d) for g in (dWg, dWu)):
        raise ValueError("dWg and dWu must be f x d")
    _same_device(X, Wg, Wu, dH, dX, dWg, dWu)
    nbytes = gated_backward_workspace_size(N, d, f, dX is not None, dWg is not None or dWu is not None)
    ws = _workspace(nbytes, X.device, workspace, stream)
    rc = lib().loca_gated_backward(_ptr(X), ldx, N, d, _ptr(Wg), _ptr(Wu), f, code, _ptr(dH), lddh, _ptr(dX), lddx,
                                   _ptr(dWg), _ptr(dWu), _ptr(ws), nbytes, _stream(stream))
    _check(rc, "loca_gated_backward")


class GradClip:
    """Global norm and clipping of one list of gradient tensors (float32 and bfloat16, any shapes,
    contiguous): in place, or into ``out`` (tensors of the same shapes and types).  Holds the list
    from step to step; :meth:`run` enqueues one step."""

    def __init__(self, grads, out=None):
        self.grads = list(grads)
        self.out = None if out is None else list(out)
        if self.out is not None and len(self.out) != len(self.grads):
            raise ValueError("out must have one tensor for each of grads")
        for i, t in enumerate(self.grads):
            _dev(t, f"grads[{i}]", (torch.float32, torch.bfloat16))
            if t is None:
                raise TypeError(f"grads[{i}] must be a CUDA tensor")
            if self.out is not None:
                if self.out[i] is None:
                    raise TypeError(f"out[{i}] must be a CUDA tensor")
                _dev(self.out[i], f"out[{i}]", t.dtype)
                if self.out[i].numel() != t.numel():
                    raise ValueError(f"out[{i}] has {self.out[i].numel()} elements, grads[{i}] {t.numel()}")
        n = len(self.grads)
        self._in = (ctypes.c_void_p * max(n, 1))(*[t.data_ptr() for t in self.grads])
        self._out = None if out is None else (ctypes.c_void_p * max(n, 1))(*[t.data_ptr() for t in self.out])
        self._numel = (ctypes.c_int64 * max(n, 1))(*[t.numel() for t in self.grads])
        self._dtype = (ctypes.c_int32 * max(n, 1))(*[_code(t.dtype) for t in self.grads])
        size = ctypes.c_size_t(0)
        _check(lib().loca_grad_clip_workspace_size(n, ctypes.byref(size)), "loca_grad_clip_workspace_size")
        self._bytes = size.value
        # scratch memory for each stream, so that steps on two streams do not share their sums
        self._ws = {_stream(None).value: _empty(self._bytes, self.grads[0].device if n else "cuda")}

    def run(self, max_norm, norm, stream=None):
        """Writes the global norm before clipping to ``norm`` (one float, device) and the gradients
        scaled by ``min(1, max_norm / norm)``; ``max_norm = inf`` gives the norm alone."""
        _dev(norm, "norm", torch.float32)
        if norm is None or norm.numel() != 1:
            raise ValueError("norm must be a CUDA tensor of one element")
        on = _stream(stream)
        ws = self._ws.get(on.value)
        if ws is None:
            ws = self._ws[on.value] = _empty(self._bytes, norm.device, stream)
        rc = lib().loca_grad_clip(self._in, self._out, self._numel, self._dtype, len(self.grads), float(max_norm),
                                  _ptr(norm), _ptr(ws), self._bytes, on)
        _check(rc, "loca_grad_clip")


class Pass:
    """Device buffers and workspaces for repeated Stage-II outer iterations of one shape.

    ``run()`` enqueues loca_error -> (loca_targets -> loca_accumulate per mini-batch) ->
    loca_ridge_solve on the current stream and allocates nothing.
    """

    def __init__(self, L, N, d, C, r, k, act_dtype, lambda_rel, eta, micro_batches=1, device="cuda",
                 t_dtype=None):
        self.L, self.N, self.d, self.C, self.r, self.k = L, N, d, C, r, k
        self.eta = float(eta)
        self.lambda_rel = [float(v) for v in lambda_rel]
        self.mb = int(micro_batches)
        self.nb = -(-N // self.mb)
        dev = torch.device(device)
        t_dtype = act_dtype if t_dtype is None else t_dtype
        f32 = dict(dtype=torch.float32, device=dev)
        self.E = torch.empty((N, C), **f32)
        self.ce = torch.empty((N,), **f32)
        self.T = torch.empty((L, self.nb, d), dtype=t_dtype, device=dev)
        self.tsq = torch.empty((L,), dtype=torch.float64, device=dev)
        self.gram = torch.empty((L, d, d), **f32)
        self.cross = torch.empty((L, d, d), **f32)
        self.xsq = torch.empty((L,), dtype=torch.float64, device=dev)
        nl = len(self.lambda_rel)
        self.B = torch.empty((nl, L, d, k), **f32)
        self.info = torch.empty((nl, L), dtype=torch.int32, device=dev)
        self.ws_t = _workspace(targets_workspace_size(self.nb, L, d), dev)
        self.ws_a = _workspace(accumulate_workspace_size(L, self.nb, d, act_dtype), dev)
        self.ws_s = _workspace(ridge_solve_workspace_size(L, d, k), dev)

    def run(self, logits, label_cols, y, X, P, Q, A, B_prev=None, normaliser=0, stream=None):
        """``X``: one ``L x N x d`` tensor, or a list of per-mini-batch ``L x N_m x d`` tensors
        (contiguous token ranges of ``ceil(N / micro_batches)`` tokens, in order)."""
        loca_error(logits, label_cols, y, self.E, ce=self.ce, normaliser=normaliser, stream=stream)
        batches = X if isinstance(X, (list, tuple)) else [X]
        if len(batches) != self.mb:
            raise ValueError(f"expected {self.mb} mini-batches of X, got {len(batches)}")
        n0 = 0
        for m, Xm in enumerate(batches):
            nm = Xm.shape[1]
            Tm = self.T.view(-1)[: self.L * nm * self.d].view(self.L, nm, self.d)
            loca_targets(self.E[n0:n0 + nm], P, Q, Tm, tsq=self.tsq, workspace=self.ws_t, stream=stream)
            loca_accumulate(Xm, Tm, self.tsq, self.eta, self.gram, self.cross, self.xsq, zero_first=(m == 0),
                            workspace=self.ws_a, stream=stream)
            n0 += nm
        if n0 != self.N:
            raise ValueError(f"mini-batches hold {n0} tokens, expected {self.N}")
        loca_ridge_solve(self.gram, self.cross, A, self.lambda_rel, self.B, self.info, xsq_total=self.xsq,
                         B_prev=B_prev, workspace=self.ws_s, stream=stream)
        return self.B
