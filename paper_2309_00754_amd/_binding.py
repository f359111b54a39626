"""ctypes binding of libhydra (the C ABI declared in include/hydra.h).

Argument marshalling only: every step of the path runs in the HIP kernels of
libhydra.  Tensors are PyTorch tensors on a ROCm device (PyTorch provides the
device memory and the stream); they are checked for dtype, shape, device and
contiguity, then their data pointers are passed through.  There is no CPU
fallback: a missing library raises ``HydraLibraryMissing``.

The accepted form of a call goes through ``_hydra_native`` (native/binding.cpp),
which makes the same checks and the same library call without ctypes; for
anything else it answers ``SLOW`` and the Python checks below decide, with
their messages.
"""
from __future__ import annotations

import ctypes
import os
import warnings
from typing import Optional

PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(PKG, "libhydra.so")
NATIVE_PATH = os.path.join(PKG, "_hydra_native.so")

HYDRA_OK = 0
HYDRA_ERR_NULL = -1
HYDRA_ERR_SHAPE = -2
HYDRA_ERR_ALIGN = -3
HYDRA_ERR_UNSUPPORTED = -4
HYDRA_ERR_WORKSPACE = -5
HYDRA_ERR_HIP = -6
HYDRA_MAX_RANK = 128
HYDRA_MAX_GROUP = 8
HYDRA_MAX_ADAPTERS = 4
HYDRA_SCORE_NOALLOC_MAX_BYTES = 48 << 20
HYDRA_BF16 = 0
HYDRA_F32 = 1
HYDRA_MAX_TOP = 32
HYDRA_MAX_GRADS = 4096
HYDRA_MAX_DRAFTS = 128
HYDRA_GROUP_WS_CONTROL_BYTES = 4352
HYDRA_GROUP_WS_BOUND_WORD = 8
HYDRA_GROUP_WS_T_BYTES = 65536
HYDRA_GROUP_WS_Y_BYTES = 2097152

# Every symbol include/hydra.h declares.
EXPORTED = (
    "hydra_lora_linear",
    "hydra_lora_linear_workspace_bytes",
    "hydra_lora_linear_ws",
    "hydra_lora_linear_group",
    "hydra_lora_linear_group_workspace_bytes",
    "hydra_lora_linear_group_ws",
    "hydra_lora_linear_multi",
    "hydra_lora_linear_multi_workspace_bytes",
    "hydra_lora_linear_multi_ws",
    "hydra_score_workspace_bytes",
    "hydra_score",
    "hydra_score_noalloc",
    "hydra_score_two_input",
    "hydra_score_logits",
    "hydra_value_head",
    "hydra_ppo_advantages",
    "hydra_ppo_loss",
    "hydra_transpose_bf16",
    "hydra_lora_linear_backward_workspace_bytes",
    "hydra_lora_linear_backward",
    "hydra_layer_norm",
    "hydra_layer_norm_backward_workspace_bytes",
    "hydra_layer_norm_backward",
    "hydra_token_logprobs_workspace_bytes",
    "hydra_token_logprobs",
    "hydra_token_logprobs_backward",
    "hydra_grad_norm_workspace_bytes",
    "hydra_grad_norm",
    "hydra_grad_clip",
    "hydra_fp8_quantize",
    "hydra_fp8_lora_linear_workspace_bytes",
    "hydra_fp8_lora_linear",
    "hydra_fp8_lora_linear_backward_workspace_bytes",
    "hydra_fp8_lora_linear_backward",
    "hydra_dropout",
    "hydra_verify_drafts_workspace_bytes",
    "hydra_verify_drafts",
    "hydra_status_string",
    "hydra_abi_version",
)


class HydraLibraryMissing(ImportError):
    pass


class HydraError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = int(status)
        super().__init__(f"{where}: {status_string(status)} ({status})")


_lib: Optional[ctypes.CDLL] = None

_vp = ctypes.c_void_p
_i64 = ctypes.c_int64
_f32 = ctypes.c_float


def lib() -> ctypes.CDLL:
    """Load libhydra.so (built in-tree by ``python -m paper_2309_00754_amd.build``)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise HydraLibraryMissing(
            f"{LIB_PATH} is not built; run `python -m paper_2309_00754_amd.build` (no CPU fallback exists)")
    L = ctypes.CDLL(LIB_PATH)
    L.hydra_lora_linear.argtypes = [_vp, _vp, _vp, _vp, _f32, _i64, _i64, _i64, _i64, _vp, _vp, _vp]
    L.hydra_lora_linear.restype = ctypes.c_int
    _pp = ctypes.POINTER(ctypes.c_void_p)
    L.hydra_lora_linear_group.argtypes = [_i64, _pp, _pp, _pp, _pp, ctypes.POINTER(ctypes.c_float), _i64, _i64, _i64,
                                          _i64, _pp, _pp, _vp]
    L.hydra_lora_linear_group.restype = ctypes.c_int
    L.hydra_lora_linear_group_workspace_bytes.argtypes = [_i64, _i64, _i64, _i64, ctypes.POINTER(ctypes.c_size_t)]
    L.hydra_lora_linear_group_workspace_bytes.restype = ctypes.c_int
    L.hydra_lora_linear_group_ws.argtypes = [_i64, _pp, _pp, _pp, _pp, ctypes.POINTER(ctypes.c_float), _i64, _i64,
                                             _i64, _i64, _pp, _pp, _vp, ctypes.c_size_t, _vp]
    L.hydra_lora_linear_group_ws.restype = ctypes.c_int
    L.hydra_lora_linear_workspace_bytes.argtypes = [_i64, _i64, _i64, ctypes.POINTER(ctypes.c_size_t)]
    L.hydra_lora_linear_workspace_bytes.restype = ctypes.c_int
    L.hydra_lora_linear_ws.argtypes = [_vp, _vp, _vp, _vp, _f32, _i64, _i64, _i64, _i64, _vp, _vp, _vp,
                                       ctypes.c_size_t, _vp]
    L.hydra_lora_linear_ws.restype = ctypes.c_int
    L.hydra_lora_linear_multi.argtypes = [_vp, _vp, _i64, _pp, _pp, _pp, ctypes.POINTER(ctypes.c_float), _i64, _i64,
                                          _i64, _i64, _vp, _pp, _vp]
    L.hydra_lora_linear_multi.restype = ctypes.c_int
    L.hydra_lora_linear_multi_workspace_bytes.argtypes = [_i64, _i64, _i64, ctypes.POINTER(ctypes.c_size_t)]
    L.hydra_lora_linear_multi_workspace_bytes.restype = ctypes.c_int
    L.hydra_lora_linear_multi_ws.argtypes = [_vp, _vp, _i64, _pp, _pp, _pp, ctypes.POINTER(ctypes.c_float), _i64, _i64,
                                             _i64, _i64, _vp, _pp, _vp, ctypes.c_size_t, _vp]
    L.hydra_lora_linear_multi_ws.restype = ctypes.c_int
    L.hydra_score_workspace_bytes.argtypes = [_i64, _i64, ctypes.POINTER(ctypes.c_size_t)]
    L.hydra_score_workspace_bytes.restype = ctypes.c_int
    L.hydra_score.argtypes = [_vp, _vp, _vp, _vp, _f32, _vp, _vp, _i64, _i64, _i64, _i64, _i64,
                              _vp, _vp, _vp, _vp, _vp, _vp, _vp, ctypes.c_size_t, _vp, _vp]
    L.hydra_score.restype = ctypes.c_int
    L.hydra_score_noalloc.argtypes = [_vp, _vp, _vp, _vp, _f32, _vp, _vp, _i64, _i64, _i64, _i64, _i64,
                                      _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp]
    L.hydra_score_noalloc.restype = ctypes.c_int
    L.hydra_score_two_input.argtypes = [_vp, _vp, _vp, _vp, _vp, _f32, _vp, _vp, _i64, _i64, _i64, _i64, _i64,
                                        _vp, _vp, _vp, _vp, _vp, _vp, _vp, ctypes.c_size_t, _vp, _vp]
    L.hydra_score_two_input.restype = ctypes.c_int
    L.hydra_score_logits.argtypes = [_vp, _vp, _vp, _i64, _i64, _vp, _vp, _vp, _vp, _vp, _vp, _vp]
    L.hydra_score_logits.restype = ctypes.c_int
    L.hydra_value_head.argtypes = [_vp, _vp, _i64, _i64, _vp, _vp]
    L.hydra_value_head.restype = ctypes.c_int
    L.hydra_ppo_advantages.argtypes = [_vp, _vp, _vp, _i64, _i64, _i64, _f32, _f32, _f32, _vp, _vp, _vp, _vp]
    L.hydra_ppo_advantages.restype = ctypes.c_int
    L.hydra_ppo_loss.argtypes = [_vp, _vp, _vp, _vp, _vp, _i64, _i64, _i64, _f32, _vp, _vp, _vp, _vp]
    L.hydra_ppo_loss.restype = ctypes.c_int
    L.hydra_transpose_bf16.argtypes = [_vp, _i64, _i64, _vp, _vp]
    L.hydra_transpose_bf16.restype = ctypes.c_int
    L.hydra_lora_linear_backward_workspace_bytes.argtypes = [_i64, _i64, _i64, _i64, ctypes.POINTER(ctypes.c_size_t)]
    L.hydra_lora_linear_backward_workspace_bytes.restype = ctypes.c_int
    L.hydra_lora_linear_backward.argtypes = [_vp, _vp, _vp, _vp, _f32, _vp, _i64, _i64, _i64, _i64, _vp, _vp, _vp,
                                             _vp, ctypes.c_size_t, _vp]
    L.hydra_lora_linear_backward.restype = ctypes.c_int
    _int, _size, _sizep = ctypes.c_int, ctypes.c_size_t, ctypes.POINTER(ctypes.c_size_t)
    _i32p, _i64p = ctypes.POINTER(ctypes.c_int32), ctypes.POINTER(ctypes.c_int64)
    _f64 = ctypes.c_double
    for name, args in (
            ("hydra_layer_norm", [_vp, _int, _vp, _vp, _int, _f32, _i64, _i64, _vp, _int, _vp, _vp, _vp]),
            ("hydra_layer_norm_backward_workspace_bytes", [_i64, _i64, _sizep]),
            ("hydra_layer_norm_backward", [_vp, _int, _vp, _int, _vp, _int, _vp, _vp, _i64, _i64, _vp, _int, _vp, _vp,
                                           _vp, _size, _vp]),
            ("hydra_token_logprobs_workspace_bytes", [_i64, _i64, _i64, _sizep]),
            ("hydra_token_logprobs", [_vp, _int, _i64, _vp, _i64, _i64, _i64, _vp, _vp, _vp, _vp, _vp, _vp, _size, _vp,
                                      _vp]),
            ("hydra_token_logprobs_backward", [_vp, _int, _i64, _vp, _vp, _vp, _vp, _vp, _i64, _i64, _vp, _int, _i64, _vp,
                                               _vp]),
            ("hydra_grad_norm_workspace_bytes", [_sizep]),
            ("hydra_grad_norm", [_i64, _pp, _i32p, _i64p, _vp, _vp, _size, _vp]),
            ("hydra_grad_clip", [_i64, _pp, _i32p, _i64p, _f32, _vp, _pp, _i32p, _vp, _size, _vp, _vp]),
            ("hydra_fp8_quantize", [_vp, _int, _i64, _i64, _i64, _vp, _vp, _vp, _vp, _vp]),
            ("hydra_fp8_lora_linear_workspace_bytes", [_i64, _i64, _i64, _i64, _sizep]),
            ("hydra_fp8_lora_linear", [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _f32, _i64, _i64, _i64, _i64, _vp, _vp, _int,
                                       _vp, _size, _vp]),
            ("hydra_fp8_lora_linear_backward_workspace_bytes", [_i64, _i64, _i64, _i64, _sizep]),
            ("hydra_fp8_lora_linear_backward", [_vp, _vp, _vp, _vp, _vp, _f32, _vp, _i64, _i64, _i64, _i64, _f64, _vp, _vp,
                                                _int, _vp, _vp, _vp, _size, _vp]),
            ("hydra_dropout", [_vp, _int, _vp, _int, _f64, _vp, _i64, _vp, _int, _vp]),
            ("hydra_verify_drafts_workspace_bytes", [_i64, _i64, _i64, _sizep]),
            ("hydra_verify_drafts", [_vp, _int, _i64, _vp, _int, _i64, _vp, _vp, _vp, _i64, _i64, _i64, _f64, _vp, _vp, _vp,
                                     _vp, _size, _vp, _vp])):
        getattr(L, name).argtypes = args
        getattr(L, name).restype = ctypes.c_int
    L.hydra_status_string.argtypes = [ctypes.c_int]
    L.hydra_status_string.restype = ctypes.c_char_p
    L.hydra_abi_version.argtypes = []
    L.hydra_abi_version.restype = ctypes.c_int
    _lib = L
    return L


_SLOW = -1000


class _NoNative:
    """Stands in for _hydra_native where it is not built: every call takes the Python path."""

    def __getattr__(self, name):
        return lambda *args: _SLOW


_nat = None


def _native():
    """_hydra_native, loaded with the first call (it needs torch's libraries in the process)."""
    global _nat
    if _nat is None:
        _torch()
        try:
            from . import _hydra_native as nat
        except ImportError as e:
            if os.path.exists(NATIVE_PATH):  # built, and yet not loaded: not to go unnoticed
                warnings.warn(f"{NATIVE_PATH} does not load, calls go through ctypes and take longer on the host: "
                              f"{e}", RuntimeWarning, stacklevel=3)
            nat = _NoNative()
        _nat = nat
    return _nat


def status_string(status: int) -> str:
    return lib().hydra_status_string(int(status)).decode()


def _check(status: int, where: str) -> None:
    if status != HYDRA_OK:
        raise HydraError(status, where)


# ------------------------------------------------------------------ tensor helpers

def _torch():
    import torch
    return torch


def _ptr(t) -> Optional[int]:
    return None if t is None else int(t.data_ptr())


def _stream_handle(stream) -> Optional[int]:
    """The hipStream_t of ``stream``, or of torch's current stream on the current device when None (read through
    torch's raw-stream query when it has one: building a Stream object costs a few microseconds per call)."""
    torch = _torch()
    if stream is None:
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        if raw is not None:
            return int(raw(torch.cuda.current_device()))
        stream = torch.cuda.current_stream()
    return int(stream.cuda_stream)


def _need(t, name, dtypes, shape=None):
    if t is None:
        return
    torch = _torch()
    # the accepted case in one condition (a few attribute reads: these checks run for every tensor of every call,
    # and at decode sizes the host time of a call is comparable to its kernel's); the messages only on failure
    if isinstance(t, torch.Tensor) and t.is_cuda and t.dtype in dtypes and t.is_contiguous() and (
            shape is None or t.shape == tuple(shape)):
        return
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.device.type != "cuda":
        raise ValueError(f"{name} must be on a ROCm device, got {t.device}")
    if t.dtype not in dtypes:
        raise TypeError(f"{name} has dtype {t.dtype}, expected one of {dtypes}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")


def _bf16_types():
    torch = _torch()
    return (torch.bfloat16, torch.int16, torch.uint16)


# ------------------------------------------------------------------ entry points

def hydra_lora_linear(x, W, A, B, s: float, y_off=None, y_on=None, stream=None) -> None:
    """y_off = x W^T and/or y_on = x W^T + s (x A^T) B^T (see include/hydra.h).

    x [M,K], W [N,K], A [r,K], B [N,r]: bf16 (or 16-bit integer tensors holding
    bf16 bits); y_off, y_on [M,N] float32 outputs (either may be None).
    """
    st = (_nat or _native()).lora_linear(x, W, A, B, s, y_off, y_on, None, stream, False)
    if st == _SLOW:
        return _hydra_lora_linear(x, W, A, B, s, y_off, y_on, stream)
    if st != HYDRA_OK:
        _check(st, "hydra_lora_linear")


def _hydra_lora_linear(x, W, A, B, s, y_off, y_on, stream) -> None:
    torch = _torch()
    bf = _bf16_types()
    M, K = x.shape
    N = W.shape[0]
    r = 0 if A is None else A.shape[0]
    _need(x, "x", bf)
    _need(W, "W", bf, (N, K))
    _need(A, "A", bf, (r, K))
    _need(B, "B", bf, (N, r))
    _need(y_off, "y_off", (torch.float32,), (M, N))
    _need(y_on, "y_on", (torch.float32,), (M, N))
    st = lib().hydra_lora_linear(_ptr(x), _ptr(W), _ptr(A), _ptr(B), float(s), M, N, K, r,
                                 _ptr(y_off), _ptr(y_on), _stream_handle(stream))
    _check(st, "hydra_lora_linear")


def hydra_lora_linear_workspace_bytes(M: int, N: int, r: int) -> int:
    out = ctypes.c_size_t(0)
    _check(lib().hydra_lora_linear_workspace_bytes(int(M), int(N), int(r), ctypes.byref(out)),
           "hydra_lora_linear_workspace_bytes")
    return int(out.value)


def hydra_lora_linear_ws(x, W, A, B, s: float, y_off=None, y_on=None, workspace=None, stream=None) -> None:
    """hydra_lora_linear with the pre-pass workspace (see include/hydra.h); allocates one if none is given."""
    st = (_nat or _native()).lora_linear(x, W, A, B, s, y_off, y_on, workspace, stream, True)
    if st == _SLOW:
        return _hydra_lora_linear_ws(x, W, A, B, s, y_off, y_on, workspace, stream)
    if st != HYDRA_OK:
        _check(st, "hydra_lora_linear_ws")


def _hydra_lora_linear_ws(x, W, A, B, s, y_off, y_on, workspace, stream) -> None:
    torch = _torch()
    bf = _bf16_types()
    M, K = x.shape
    N = W.shape[0]
    r = 0 if A is None else A.shape[0]
    _need(x, "x", bf)
    _need(W, "W", bf, (N, K))
    _need(A, "A", bf, (r, K))
    _need(B, "B", bf, (N, r))
    _need(y_off, "y_off", (torch.float32,), (M, N))
    _need(y_on, "y_on", (torch.float32,), (M, N))
    need = hydra_lora_linear_workspace_bytes(M, N, r)
    if workspace is None and need > 0:
        workspace = torch.empty(need, dtype=torch.uint8, device=x.device)
    _need(workspace, "workspace", (torch.uint8,))
    nbytes = 0 if workspace is None else workspace.numel()
    st = lib().hydra_lora_linear_ws(_ptr(x), _ptr(W), _ptr(A), _ptr(B), float(s), M, N, K, r, _ptr(y_off),
                                    _ptr(y_on), _ptr(workspace), nbytes, _stream_handle(stream))
    _check(st, "hydra_lora_linear_ws")


def _ptr_array(ts):
    arr = (ctypes.c_void_p * len(ts))()
    for i, t in enumerate(ts):
        arr[i] = _ptr(t)
    return arr


def hydra_lora_linear_group(xs, Ws, As, Bs, ss, y_offs=None, y_ons=None, stream=None) -> None:
    """G linears with shared M, N, K, r in one call (see include/hydra.h).

    xs, Ws, As, Bs, y_offs, y_ons: sequences of G tensors (entries may be None);
    ss: G scales.
    """
    st = (_nat or _native()).lora_linear_group(xs, Ws, As, Bs, ss, y_offs, y_ons, None, stream, False)
    if st == _SLOW:
        return _hydra_lora_linear_group(xs, Ws, As, Bs, ss, y_offs, y_ons, stream)
    if st != HYDRA_OK:
        _check(st, "hydra_lora_linear_group")


def _hydra_lora_linear_group(xs, Ws, As, Bs, ss, y_offs, y_ons, stream) -> None:
    torch = _torch()
    bf = _bf16_types()
    G = len(Ws)
    if not (len(xs) == len(As) == len(Bs) == len(ss) == G):
        raise ValueError("all per-member sequences must have the same length")
    y_offs = list(y_offs) if y_offs is not None else [None] * G
    y_ons = list(y_ons) if y_ons is not None else [None] * G
    M, K = xs[0].shape
    N = Ws[0].shape[0]
    r = next((a.shape[0] for a in As if a is not None), 0)
    for i in range(G):
        _need(xs[i], "x", bf, (M, K))
        _need(Ws[i], "W", bf, (N, K))
        _need(As[i], "A", bf, (r, K))
        _need(Bs[i], "B", bf, (N, r))
        _need(y_offs[i], "y_off", (torch.float32,), (M, N))
        _need(y_ons[i], "y_on", (torch.float32,), (M, N))
    svals = (ctypes.c_float * G)(*[float(v) for v in ss])
    st = lib().hydra_lora_linear_group(G, _ptr_array(xs), _ptr_array(Ws), _ptr_array(As), _ptr_array(Bs), svals,
                                       M, N, K, r, _ptr_array(y_offs), _ptr_array(y_ons), _stream_handle(stream))
    _check(st, "hydra_lora_linear_group")


def hydra_lora_linear_group_workspace_bytes(G: int, M: int, N: int, r: int) -> int:
    out = ctypes.c_size_t(0)
    _check(lib().hydra_lora_linear_group_workspace_bytes(int(G), int(M), int(N), int(r), ctypes.byref(out)),
           "hydra_lora_linear_group_workspace_bytes")
    return int(out.value)


def hydra_lora_linear_group_workspace(G: int, M: int, N: int, r: int, device):
    """A zero-filled workspace for hydra_lora_linear_group_ws (the calls leave its control words zero, so it is
    reused as it is)."""
    torch = _torch()
    return torch.zeros(hydra_lora_linear_group_workspace_bytes(G, M, N, r), dtype=torch.uint8, device=device)


def hydra_lora_linear_group_ws(xs, Ws, As, Bs, ss, y_offs=None, y_ons=None, workspace=None, stream=None) -> None:
    """hydra_lora_linear_group with a caller workspace: a decode step (M <= 8) in one launch (see include/hydra.h).

    workspace: a uint8 tensor from hydra_lora_linear_group_workspace (zero before its first use)."""
    st = (_nat or _native()).lora_linear_group(xs, Ws, As, Bs, ss, y_offs, y_ons, workspace, stream, True)
    if st == _SLOW:
        return _hydra_lora_linear_group_ws(xs, Ws, As, Bs, ss, y_offs, y_ons, workspace, stream)
    if st != HYDRA_OK:
        _check(st, "hydra_lora_linear_group_ws")


def _hydra_lora_linear_group_ws(xs, Ws, As, Bs, ss, y_offs, y_ons, workspace, stream) -> None:
    torch = _torch()
    bf = _bf16_types()
    G = len(Ws)
    if not (len(xs) == len(As) == len(Bs) == len(ss) == G):
        raise ValueError("all per-member sequences must have the same length")
    y_offs = list(y_offs) if y_offs is not None else [None] * G
    y_ons = list(y_ons) if y_ons is not None else [None] * G
    M, K = xs[0].shape
    N = Ws[0].shape[0]
    r = next((a.shape[0] for a in As if a is not None), 0)
    for i in range(G):
        _need(xs[i], "x", bf, (M, K))
        _need(Ws[i], "W", bf, (N, K))
        _need(As[i], "A", bf, (r, K))
        _need(Bs[i], "B", bf, (N, r))
        _need(y_offs[i], "y_off", (torch.float32,), (M, N))
        _need(y_ons[i], "y_on", (torch.float32,), (M, N))
    if workspace is None:
        raise ValueError("hydra_lora_linear_group_ws needs a workspace from hydra_lora_linear_group_workspace")
    _need(workspace, "workspace", (torch.uint8,))
    svals = (ctypes.c_float * G)(*[float(v) for v in ss])
    st = lib().hydra_lora_linear_group_ws(G, _ptr_array(xs), _ptr_array(Ws), _ptr_array(As), _ptr_array(Bs), svals,
                                          M, N, K, r, _ptr_array(y_offs), _ptr_array(y_ons), _ptr(workspace),
                                          workspace.numel(), _stream_handle(stream))
    _check(st, "hydra_lora_linear_group_ws")


def _multi_args(x_off, W, x_ons, As, Bs, ss, y_off, y_ons):
    torch = _torch()
    bf = _bf16_types()
    n_on = len(x_ons)
    As = list(As) if As is not None else [None] * n_on
    Bs = list(Bs) if Bs is not None else [None] * n_on
    y_ons = list(y_ons) if y_ons is not None else [None] * n_on
    if not (len(As) == len(Bs) == len(ss) == len(y_ons) == n_on):
        raise ValueError("all per-input sequences must have the same length")
    ref = x_off if x_off is not None else (x_ons[0] if n_on else None)
    if ref is None:
        raise ValueError("at least one input is needed")
    M, K = ref.shape
    N = W.shape[0]
    r = next((a.shape[0] for a in As if a is not None), 0)
    _need(W, "W", bf, (N, K))
    _need(x_off, "x_off", bf, (M, K))
    _need(y_off, "y_off", (torch.float32,), (M, N))
    for a in range(n_on):
        _need(x_ons[a], "x_on", bf, (M, K))
        _need(As[a], "A", bf, (r, K))
        _need(Bs[a], "B", bf, (N, r))
        _need(y_ons[a], "y_on", (torch.float32,), (M, N))
    svals = (ctypes.c_float * max(n_on, 1))(*[float(v) for v in ss])
    return (_ptr(x_off), _ptr(W), n_on, _ptr_array(x_ons), _ptr_array(As), _ptr_array(Bs), svals if n_on else None, M,
            N, K, r, _ptr(y_off), _ptr_array(y_ons))


def hydra_lora_linear_multi(x_off, W, x_ons, As, Bs, ss, y_off=None, y_ons=None, stream=None) -> None:
    """One W for a LoRA-off input and several LoRA-on inputs with their own adapters (see include/hydra.h).

    x_off, y_off: tensors or None (together); x_ons, As, Bs, y_ons: sequences of n_on tensors (As, Bs may be
    None or all-None when r == 0); ss: n_on scales.
    """
    st = (_nat or _native()).lora_linear_multi(x_off, W, x_ons, As, Bs, ss, y_off, y_ons, None, stream, False)
    if st == _SLOW:
        return _hydra_lora_linear_multi(x_off, W, x_ons, As, Bs, ss, y_off, y_ons, stream)
    if st != HYDRA_OK:
        _check(st, "hydra_lora_linear_multi")


def _hydra_lora_linear_multi(x_off, W, x_ons, As, Bs, ss, y_off, y_ons, stream) -> None:
    st = lib().hydra_lora_linear_multi(*_multi_args(x_off, W, x_ons, As, Bs, ss, y_off, y_ons), _stream_handle(stream))
    _check(st, "hydra_lora_linear_multi")


def hydra_lora_linear_multi_workspace_bytes(M: int, N: int, r: int) -> int:
    out = ctypes.c_size_t(0)
    _check(lib().hydra_lora_linear_multi_workspace_bytes(int(M), int(N), int(r), ctypes.byref(out)),
           "hydra_lora_linear_multi_workspace_bytes")
    return int(out.value)


def hydra_lora_linear_multi_ws(x_off, W, x_ons, As, Bs, ss, y_off=None, y_ons=None, workspace=None,
                               stream=None) -> None:
    """hydra_lora_linear_multi with a caller workspace (rank 128 at every M; see include/hydra.h).

    workspace: a uint8 tensor of at least hydra_lora_linear_multi_workspace_bytes(M, N, r) bytes."""
    st = (_nat or _native()).lora_linear_multi(x_off, W, x_ons, As, Bs, ss, y_off, y_ons, workspace, stream, True)
    if st == _SLOW:
        return _hydra_lora_linear_multi_ws(x_off, W, x_ons, As, Bs, ss, y_off, y_ons, workspace, stream)
    if st != HYDRA_OK:
        _check(st, "hydra_lora_linear_multi_ws")


def _hydra_lora_linear_multi_ws(x_off, W, x_ons, As, Bs, ss, y_off, y_ons, workspace, stream) -> None:
    torch = _torch()
    if workspace is None:
        raise ValueError("hydra_lora_linear_multi_ws needs a workspace")
    _need(workspace, "workspace", (torch.uint8,))
    st = lib().hydra_lora_linear_multi_ws(*_multi_args(x_off, W, x_ons, As, Bs, ss, y_off, y_ons), _ptr(workspace),
                                          workspace.numel(), _stream_handle(stream))
    _check(st, "hydra_lora_linear_multi_ws")


def hydra_score_workspace_bytes(M: int, V: int) -> int:
    out = ctypes.c_size_t(0)
    _check(lib().hydra_score_workspace_bytes(int(M), int(V), ctypes.byref(out)), "hydra_score_workspace_bytes")
    return int(out.value)


def hydra_score(h, W_lm, A, B, s: float, tokens, w_rm, n_seq: int, seq_len: int,
                lp_on, lp_off, kl, reward=None, lse_on=None, lse_off=None,
                workspace=None, err_flag=None, stream=None) -> None:
    """Fused CLM-head (LoRA on and off) log-prob / KL scoring plus the reward head."""
    st = (_nat or _native()).score(None, h, W_lm, A, B, s, tokens, w_rm, n_seq, seq_len, lp_on, lp_off, kl, reward,
                                   lse_on, lse_off, workspace, err_flag, stream, False)
    if st == _SLOW:
        return _hydra_score(h, W_lm, A, B, s, tokens, w_rm, n_seq, seq_len, lp_on, lp_off, kl, reward, lse_on,
                            lse_off, workspace, err_flag, stream)
    if st != HYDRA_OK:
        _check(st, "hydra_score")


def _hydra_score(h, W_lm, A, B, s, tokens, w_rm, n_seq, seq_len, lp_on, lp_off, kl, reward, lse_on, lse_off,
                 workspace, err_flag, stream) -> None:
    torch = _torch()
    bf = _bf16_types()
    M, K = h.shape
    V = W_lm.shape[0]
    r = 0 if A is None else A.shape[0]
    if M != n_seq * seq_len:
        raise ValueError("h rows must equal n_seq * seq_len")
    _need(h, "h", bf)
    _need(W_lm, "W_lm", bf, (V, K))
    _need(A, "A", bf, (r, K))
    _need(B, "B", bf, (V, r))
    _need(tokens, "tokens", (torch.int32,), (M,))
    _need(w_rm, "w_rm", bf, (K,))
    for name, t in (("lp_on", lp_on), ("lp_off", lp_off), ("kl", kl), ("lse_on", lse_on), ("lse_off", lse_off)):
        _need(t, name, (torch.float32,), (M,))
    _need(reward, "reward", (torch.float32,), (n_seq,))
    _need(err_flag, "err_flag", (torch.int32,), (1,))
    need = hydra_score_workspace_bytes(M, V)
    if workspace is None:
        workspace = torch.empty(need, dtype=torch.uint8, device=h.device)
    _need(workspace, "workspace", (torch.uint8,))
    st = lib().hydra_score(_ptr(h), _ptr(W_lm), _ptr(A), _ptr(B), float(s), _ptr(tokens), _ptr(w_rm),
                           int(n_seq), int(seq_len), K, V, r, _ptr(lp_on), _ptr(lp_off), _ptr(kl), _ptr(reward),
                           _ptr(lse_on), _ptr(lse_off), _ptr(workspace), workspace.numel(), _ptr(err_flag),
                           _stream_handle(stream))
    _check(st, "hydra_score")


def hydra_score_two_input(h_act, h_off, W_lm, A, B, s: float, tokens, w_rm, n_seq: int, seq_len: int,
                          lp_on, lp_off, kl, reward=None, lse_on=None, lse_off=None,
                          workspace=None, err_flag=None, stream=None) -> None:
    """Scoring with the actor pass's own hidden states (h_act, with the head's LoRA) and the LoRA-off pass's (h_off:
    reference log-probabilities and reward), one launch over both (see include/hydra.h)."""
    st = (_nat or _native()).score(h_act, h_off, W_lm, A, B, s, tokens, w_rm, n_seq, seq_len, lp_on, lp_off, kl,
                                   reward,
                                   lse_on, lse_off, workspace, err_flag, stream, False) if h_act is not None else _SLOW
    if st == _SLOW:
        return _hydra_score_two_input(h_act, h_off, W_lm, A, B, s, tokens, w_rm, n_seq, seq_len, lp_on, lp_off, kl,
                                      reward, lse_on, lse_off, workspace, err_flag, stream)
    if st != HYDRA_OK:
        _check(st, "hydra_score_two_input")


def _hydra_score_two_input(h_act, h_off, W_lm, A, B, s, tokens, w_rm, n_seq, seq_len, lp_on, lp_off, kl, reward,
                           lse_on, lse_off, workspace, err_flag, stream) -> None:
    torch = _torch()
    bf = _bf16_types()
    M, K = h_off.shape
    V = W_lm.shape[0]
    r = 0 if A is None else A.shape[0]
    if M != n_seq * seq_len:
        raise ValueError("h rows must equal n_seq * seq_len")
    _need(h_act, "h_act", bf, (M, K))
    _need(h_off, "h_off", bf, (M, K))
    _need(W_lm, "W_lm", bf, (V, K))
    _need(A, "A", bf, (r, K))
    _need(B, "B", bf, (V, r))
    _need(tokens, "tokens", (torch.int32,), (M,))
    _need(w_rm, "w_rm", bf, (K,))
    for name, t in (("lp_on", lp_on), ("lp_off", lp_off), ("kl", kl), ("lse_on", lse_on), ("lse_off", lse_off)):
        _need(t, name, (torch.float32,), (M,))
    _need(reward, "reward", (torch.float32,), (n_seq,))
    _need(err_flag, "err_flag", (torch.int32,), (1,))
    if workspace is None:
        workspace = torch.empty(hydra_score_workspace_bytes(M, V), dtype=torch.uint8, device=h_off.device)
    _need(workspace, "workspace", (torch.uint8,))
    st = lib().hydra_score_two_input(_ptr(h_act), _ptr(h_off), _ptr(W_lm), _ptr(A), _ptr(B), float(s), _ptr(tokens),
                                     _ptr(w_rm), int(n_seq), int(seq_len), K, V, r, _ptr(lp_on), _ptr(lp_off),
                                     _ptr(kl), _ptr(reward), _ptr(lse_on), _ptr(lse_off), _ptr(workspace),
                                     workspace.numel(), _ptr(err_flag), _stream_handle(stream))
    _check(st, "hydra_score_two_input")


def hydra_score_noalloc(h, W_lm, A, B, s: float, tokens, w_rm, n_seq: int, seq_len: int,
                        lp_on, lp_off, kl, reward=None, lse_on=None, lse_off=None, err_flag=None,
                        stream=None) -> None:
    """hydra_score with its workspace in the library's own device scratch (no allocation by the call)."""
    st = (_nat or _native()).score(None, h, W_lm, A, B, s, tokens, w_rm, n_seq, seq_len, lp_on, lp_off, kl, reward,
                                   lse_on, lse_off, None, err_flag, stream, True)
    if st == _SLOW:
        return _hydra_score_noalloc(h, W_lm, A, B, s, tokens, w_rm, n_seq, seq_len, lp_on, lp_off, kl, reward, lse_on,
                                    lse_off, err_flag, stream)
    if st != HYDRA_OK:
        _check(st, "hydra_score_noalloc")


def _hydra_score_noalloc(h, W_lm, A, B, s, tokens, w_rm, n_seq, seq_len, lp_on, lp_off, kl, reward, lse_on, lse_off,
                         err_flag, stream) -> None:
    torch = _torch()
    bf = _bf16_types()
    M, K = h.shape
    V = W_lm.shape[0]
    r = 0 if A is None else A.shape[0]
    if M != n_seq * seq_len:
        raise ValueError("h rows must equal n_seq * seq_len")
    _need(h, "h", bf)
    _need(W_lm, "W_lm", bf, (V, K))
    _need(A, "A", bf, (r, K))
    _need(B, "B", bf, (V, r))
    _need(tokens, "tokens", (torch.int32,), (M,))
    _need(w_rm, "w_rm", bf, (K,))
    for name, t in (("lp_on", lp_on), ("lp_off", lp_off), ("kl", kl), ("lse_on", lse_on), ("lse_off", lse_off)):
        _need(t, name, (torch.float32,), (M,))
    _need(reward, "reward", (torch.float32,), (n_seq,))
    _need(err_flag, "err_flag", (torch.int32,), (1,))
    st = lib().hydra_score_noalloc(_ptr(h), _ptr(W_lm), _ptr(A), _ptr(B), float(s), _ptr(tokens), _ptr(w_rm),
                                   int(n_seq), int(seq_len), K, V, r, _ptr(lp_on), _ptr(lp_off), _ptr(kl),
                                   _ptr(reward), _ptr(lse_on), _ptr(lse_off), _ptr(err_flag), _stream_handle(stream))
    _check(st, "hydra_score_noalloc")


def hydra_score_logits(logits_on, logits_off, tokens, lp_on, lp_off, kl,
                       lse_on=None, lse_off=None, err_flag=None, stream=None) -> None:
    """Sampled-token log-probabilities and KL from materialised fp32 logits."""
    st = (_nat or _native()).score_logits(logits_on, logits_off, tokens, lp_on, lp_off, kl, lse_on, lse_off, err_flag,
                                          stream)
    if st == _SLOW:
        return _hydra_score_logits(logits_on, logits_off, tokens, lp_on, lp_off, kl, lse_on, lse_off, err_flag,
                                   stream)
    if st != HYDRA_OK:
        _check(st, "hydra_score_logits")


def _hydra_score_logits(logits_on, logits_off, tokens, lp_on, lp_off, kl, lse_on, lse_off, err_flag, stream) -> None:
    torch = _torch()
    M, V = logits_on.shape
    _need(logits_on, "logits_on", (torch.float32,))
    _need(logits_off, "logits_off", (torch.float32,), (M, V))
    _need(tokens, "tokens", (torch.int32,), (M,))
    for name, t in (("lp_on", lp_on), ("lp_off", lp_off), ("kl", kl), ("lse_on", lse_on), ("lse_off", lse_off)):
        _need(t, name, (torch.float32,), (M,))
    _need(err_flag, "err_flag", (torch.int32,), (1,))
    st = lib().hydra_score_logits(_ptr(logits_on), _ptr(logits_off), _ptr(tokens), M, V, _ptr(lp_on), _ptr(lp_off),
                                  _ptr(kl), _ptr(lse_on), _ptr(lse_off), _ptr(err_flag), _stream_handle(stream))
    _check(st, "hydra_score_logits")


def hydra_value_head(h, w_v, values, stream=None) -> None:
    """values[m] = <h[m], w_v>: the critic's scalar head on every row (see include/hydra.h)."""
    st = (_nat or _native()).value_head(h, w_v, values, stream)
    if st == _SLOW:
        return _hydra_value_head(h, w_v, values, stream)
    if st != HYDRA_OK:
        _check(st, "hydra_value_head")


def _hydra_value_head(h, w_v, values, stream) -> None:
    torch = _torch()
    bf = _bf16_types()
    M, K = h.shape
    _need(h, "h", bf)
    _need(w_v, "w_v", bf, (K,))
    _need(values, "values", (torch.float32,), (M,))
    st = lib().hydra_value_head(_ptr(h), _ptr(w_v), M, K, _ptr(values), _stream_handle(stream))
    _check(st, "hydra_value_head")


def hydra_ppo_advantages(kl, reward, values, n_seq: int, seq_len: int, advantages, returns, rewards=None,
                         start: int = 0, beta: float = 0.02, gamma: float = 1.0, lam: float = 0.95,
                         stream=None) -> None:
    """Per-token PPO reward and GAE advantages / returns (see include/hydra.h)."""
    st = (_nat or _native()).ppo_advantages(kl, reward, values, n_seq, seq_len, start, beta, gamma, lam, rewards,
                                            advantages, returns, stream)
    if st == _SLOW:
        return _hydra_ppo_advantages(kl, reward, values, n_seq, seq_len, advantages, returns, rewards, start, beta,
                                     gamma, lam, stream)
    if st != HYDRA_OK:
        _check(st, "hydra_ppo_advantages")


def _hydra_ppo_advantages(kl, reward, values, n_seq, seq_len, advantages, returns, rewards, start, beta, gamma, lam,
                          stream) -> None:
    torch = _torch()
    M = int(n_seq) * int(seq_len)
    for name, t, n in (("kl", kl, M), ("reward", reward, n_seq), ("values", values, M), ("advantages", advantages, M),
                       ("returns", returns, M), ("rewards", rewards, M)):
        _need(t, name, (torch.float32,), (n,))
    st = lib().hydra_ppo_advantages(_ptr(kl), _ptr(reward), _ptr(values), int(n_seq), int(seq_len), int(start),
                                    float(beta), float(gamma), float(lam), _ptr(rewards), _ptr(advantages),
                                    _ptr(returns), _stream_handle(stream))
    _check(st, "hydra_ppo_advantages")


def hydra_ppo_loss(lp_new, lp_old, advantages, values, returns, n_seq: int, seq_len: int, losses, d_lp=None,
                   d_v=None, start: int = 0, eps: float = 0.2, stream=None) -> None:
    """PPO policy and value losses with their per-token gradients (see include/hydra.h)."""
    st = (_nat or _native()).ppo_loss(lp_new, lp_old, advantages, values, returns, n_seq, seq_len, start, eps, losses,
                                      d_lp, d_v, stream)
    if st == _SLOW:
        return _hydra_ppo_loss(lp_new, lp_old, advantages, values, returns, n_seq, seq_len, losses, d_lp, d_v, start,
                               eps, stream)
    if st != HYDRA_OK:
        _check(st, "hydra_ppo_loss")


def _hydra_ppo_loss(lp_new, lp_old, advantages, values, returns, n_seq, seq_len, losses, d_lp, d_v, start, eps,
                    stream) -> None:
    torch = _torch()
    M = int(n_seq) * int(seq_len)
    for t, name in ((lp_new, "lp_new"), (lp_old, "lp_old"), (advantages, "advantages"), (values, "values"),
                    (returns, "returns"), (d_lp, "d_lp"), (d_v, "d_v")):
        _need(t, name, (torch.float32,), (M,))
    _need(losses, "losses", (torch.float32,), (3,))
    st = lib().hydra_ppo_loss(_ptr(lp_new), _ptr(lp_old), _ptr(advantages), _ptr(values), _ptr(returns),
                              int(n_seq), int(seq_len), int(start), float(eps), _ptr(losses), _ptr(d_lp),
                              _ptr(d_v), _stream_handle(stream))
    _check(st, "hydra_ppo_loss")


def hydra_transpose_bf16(src, dst, stream=None) -> None:
    """dst [C,R] = src [R,C]^T for 16-bit tensors (see include/hydra.h)."""
    bf = _bf16_types()
    R, C = src.shape
    _need(src, "src", bf)
    _need(dst, "dst", bf, (C, R))
    _check(lib().hydra_transpose_bf16(_ptr(src), R, C, _ptr(dst), _stream_handle(stream)), "hydra_transpose_bf16")


def hydra_lora_linear_backward_workspace_bytes(M: int, N: int, K: int, r: int) -> int:
    out = ctypes.c_size_t(0)
    _check(lib().hydra_lora_linear_backward_workspace_bytes(int(M), int(N), int(K), int(r), ctypes.byref(out)),
           "hydra_lora_linear_backward_workspace_bytes")
    return int(out.value)


def hydra_lora_linear_backward(x, Wt, A, B, s: float, dy, dx=None, dA=None, dB=None, workspace=None,
                               stream=None) -> None:
    """dx, dA, dB of y = x W^T + s (x A^T) B^T with W frozen (see include/hydra.h).

    x [M,K], Wt [K,N] (W transposed, may be None when dx is not wanted), A [r,K],
    B [N,r], dy [M,N]: bf16 (or 16-bit integer tensors holding bf16 bits);
    dx [M,K], dA [r,K], dB [N,r] float32 outputs (each optional).  Allocates
    the workspace if none is given.
    """
    st = (_nat or _native()).lora_linear_backward(x, Wt, A, B, s, dy, dx, dA, dB, workspace, stream)
    if st == _SLOW:
        return _hydra_lora_linear_backward(x, Wt, A, B, s, dy, dx, dA, dB, workspace, stream)
    if st != HYDRA_OK:
        _check(st, "hydra_lora_linear_backward")


def _hydra_lora_linear_backward(x, Wt, A, B, s, dy, dx, dA, dB, workspace, stream) -> None:
    torch = _torch()
    bf = _bf16_types()
    M, N = dy.shape
    K = A.shape[1] if A is not None else (x.shape[1] if x is not None else Wt.shape[0])
    r = 0 if A is None else A.shape[0]
    _need(x, "x", bf, (M, K))
    _need(Wt, "Wt", bf, (K, N))
    _need(A, "A", bf, (r, K))
    _need(B, "B", bf, (N, r))
    _need(dy, "dy", bf)
    _need(dx, "dx", (torch.float32,), (M, K))
    _need(dA, "dA", (torch.float32,), (r, K))
    _need(dB, "dB", (torch.float32,), (N, r))
    need = hydra_lora_linear_backward_workspace_bytes(M, N, K, r)
    if workspace is None and need > 0:
        workspace = torch.empty(need, dtype=torch.uint8, device=dy.device)
    _need(workspace, "workspace", (torch.uint8,))
    nbytes = 0 if workspace is None else workspace.numel()
    st = lib().hydra_lora_linear_backward(_ptr(x), _ptr(Wt), _ptr(A), _ptr(B), float(s), _ptr(dy), M, N, K, r,
                                          _ptr(dx), _ptr(dA), _ptr(dB), _ptr(workspace), nbytes,
                                          _stream_handle(stream))
    _check(st, "hydra_lora_linear_backward")


# ------------------------------------------------------------------ the update step's further operators
#
# These calls go to the device that their tensors are on, whichever is current, on `stream` or on that device's
# current stream.  A workspace that a call allocates itself belongs to that stream.

def _any_types():
    return _bf16_types() + (_torch().float32,)


def _type(t) -> int:
    return HYDRA_BF16 if t is None or t.dtype != _torch().float32 else HYDRA_F32


def _launch(where, tensors, stream, call, workspace=None, need=0) -> None:
    """call(workspace pointer, its bytes, stream handle) on the tensors' device; allocates a workspace of `need` bytes
    if none is given."""
    torch = _torch()
    _need(workspace, "workspace", (torch.uint8,))
    devices = {t.device for t in (*tensors, workspace) if t is not None}
    if len(devices) != 1:
        raise ValueError(f"{where}: the tensors are on different devices: {sorted(map(str, devices))}")
    device, = devices
    if stream is not None and stream.device != device:
        raise ValueError(f"{where}: the stream belongs to {stream.device}, the tensors are on {device}")
    with torch.cuda.device(device):
        if workspace is None and need > 0:
            with torch.cuda.stream(stream):
                workspace = torch.empty(need, dtype=torch.uint8, device=device)
        st = call(_ptr(workspace), 0 if workspace is None else workspace.numel(), _stream_handle(stream))
    _check(st, where)


def hydra_layer_norm(x, weight, bias, y, mean=None, rstd=None, eps: float = 1e-5, stream=None) -> None:
    """y = (x - mean) rstd weight + bias over the rows of x (see include/hydra.h).

    x, y [M,K]: bf16 (or 16-bit integer tensors holding bf16 bits) or float32 (y may be x); weight, bias [K]: either
    type, both the same, each may be None; mean, rstd [M] float32 outputs for the backward (each optional).
    """
    st = (_nat or _native()).layer_norm(x, weight, bias, y, mean, rstd, eps, stream)
    if st == _SLOW:
        return _hydra_layer_norm(x, weight, bias, y, mean, rstd, eps, stream)
    if st != HYDRA_OK:
        _check(st, "hydra_layer_norm")


def _affine(weight, bias, K) -> None:
    _need(weight, "weight", _any_types(), (K,))
    _need(bias, "bias", _any_types(), (K,))
    if weight is not None and bias is not None and _type(weight) != _type(bias):
        raise TypeError(f"weight is {weight.dtype}, bias {bias.dtype}")


def _hydra_layer_norm(x, weight, bias, y, mean, rstd, eps, stream) -> None:
    torch = _torch()
    _need(x, "x", _any_types())
    M, K = x.shape
    _affine(weight, bias, K)
    _need(y, "y", _any_types(), (M, K))
    _need(mean, "mean", (torch.float32,), (M,))
    _need(rstd, "rstd", (torch.float32,), (M,))
    _launch("hydra_layer_norm", (x, weight, bias, y, mean, rstd), stream, lambda ws, n, st: lib().hydra_layer_norm(
        _ptr(x), _type(x), _ptr(weight), _ptr(bias), _type(bias if weight is None else weight), float(eps), M, K,
        _ptr(y), _type(y), _ptr(mean), _ptr(rstd), st))


def hydra_layer_norm_backward_workspace_bytes(M: int, K: int) -> int:
    out = ctypes.c_size_t(0)
    _check(lib().hydra_layer_norm_backward_workspace_bytes(int(M), int(K), ctypes.byref(out)),
           "hydra_layer_norm_backward_workspace_bytes")
    return int(out.value)


def hydra_layer_norm_backward(dy, x, weight, mean, rstd, dx=None, dweight=None, dbias=None, workspace=None,
                              stream=None) -> None:
    """dx, dweight, dbias of hydra_layer_norm (see include/hydra.h).

    dy, x, dx [M,K]: bf16 (or 16-bit integer tensors holding bf16 bits) or float32, each of its own type (dx may be dy
    or x); weight [K]: either type or None; mean, rstd [M] float32, the forward's; dweight, dbias [K] float32 outputs
    (each output optional).  Allocates the workspace if none is given.
    """
    st = (_nat or _native()).layer_norm_backward(dy, x, weight, mean, rstd, dx, dweight, dbias, workspace, stream)
    if st == _SLOW:
        return _hydra_layer_norm_backward(dy, x, weight, mean, rstd, dx, dweight, dbias, workspace, stream)
    if st != HYDRA_OK:
        _check(st, "hydra_layer_norm_backward")


def _hydra_layer_norm_backward(dy, x, weight, mean, rstd, dx, dweight, dbias, workspace, stream) -> None:
    torch = _torch()
    _need(x, "x", _any_types())
    M, K = x.shape
    _need(dy, "dy", _any_types(), (M, K))
    _affine(weight, None, K)
    _need(dx, "dx", _any_types(), (M, K))
    for name, t, n in (("mean", mean, M), ("rstd", rstd, M), ("dweight", dweight, K), ("dbias", dbias, K)):
        _need(t, name, (torch.float32,), (n,))
    need = hydra_layer_norm_backward_workspace_bytes(M, K)
    _launch("hydra_layer_norm_backward", (dy, x, weight, mean, rstd, dx, dweight, dbias), stream,
            lambda ws, n, st: lib().hydra_layer_norm_backward(
                _ptr(dy), _type(dy), _ptr(x), _type(x), _ptr(weight), _type(weight), _ptr(mean), _ptr(rstd), M, K,
                _ptr(dx), _type(dx), _ptr(dweight), _ptr(dbias), ws, n, st), workspace, need)


def hydra_token_logprobs_workspace_bytes(M: int, V: int, top: int = 0) -> int:
    out = ctypes.c_size_t(0)
    _check(lib().hydra_token_logprobs_workspace_bytes(int(M), int(V), int(top), ctypes.byref(out)),
           "hydra_token_logprobs_workspace_bytes")
    return int(out.value)


def _rows(t, name, shape=None) -> int:
    """Checks a matrix whose rows may stand apart (each row contiguous, a row's end before the next one's start);
    returns the distance of its rows in elements."""
    torch = _torch()
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.device.type != "cuda":
        raise ValueError(f"{name} must be on a ROCm device, got {t.device}")
    if t.dtype not in _any_types():
        raise TypeError(f"{name} has dtype {t.dtype}, expected one of {_any_types()}")
    if t.dim() != 2 or (shape is not None and tuple(t.shape) != tuple(shape)):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {'two dimensions' if shape is None else tuple(shape)}")
    M, V = t.shape
    ld = t.stride(0) if M > 1 else V
    if (V > 1 and t.stride(1) != 1) or ld < V:
        raise ValueError(f"{name} must have contiguous rows, got strides {t.stride()}")
    return ld


def hydra_token_logprobs(logits, tokens, lp, lse=None, entropy=None, top_ids=None, top_lp=None, workspace=None,
                         err_flag=None, stream=None) -> None:
    """Log-probabilities of given tokens under one set of logits, with the distribution's entropy and the most likely
    alternatives (see include/hydra.h).

    logits [M,V]: bf16 (or 16-bit integer tensors holding bf16 bits) or float32, rows contiguous and possibly apart
    (logits[:, :V] of a padded vocabulary); tokens [M] int32 and lp [M] float32 (both None: alternatives or statistics
    alone); lse, entropy [M] float32, top_ids [M,top] int32, top_lp [M,top] float32 outputs (each optional; top_lp
    needs top_ids).  Allocates the workspace if one is needed and none is given.
    """
    st = (_nat or _native()).token_logprobs(logits, tokens, lp, lse, entropy, top_ids, top_lp, workspace, err_flag,
                                            stream)
    if st == _SLOW:
        return _hydra_token_logprobs(logits, tokens, lp, lse, entropy, top_ids, top_lp, workspace, err_flag, stream)
    if st != HYDRA_OK:
        _check(st, "hydra_token_logprobs")


def _hydra_token_logprobs(logits, tokens, lp, lse, entropy, top_ids, top_lp, workspace, err_flag, stream) -> None:
    torch = _torch()
    ld = _rows(logits, "logits")
    M, V = logits.shape
    top = top_ids.shape[1] if isinstance(top_ids, torch.Tensor) and top_ids.dim() == 2 else 0
    _need(tokens, "tokens", (torch.int32,), (M,))
    for name, t in (("lp", lp), ("lse", lse), ("entropy", entropy)):
        _need(t, name, (torch.float32,), (M,))
    _need(top_ids, "top_ids", (torch.int32,), (M, top))
    _need(top_lp, "top_lp", (torch.float32,), (M, top))
    _need(err_flag, "err_flag", (torch.int32,), (1,))
    need = hydra_token_logprobs_workspace_bytes(M, V, top)
    _launch("hydra_token_logprobs", (logits, tokens, lp, lse, entropy, top_ids, top_lp, err_flag), stream,
            lambda ws, n, st: lib().hydra_token_logprobs(
                _ptr(logits), _type(logits), ld, _ptr(tokens), M, V, top, _ptr(lp), _ptr(lse), _ptr(entropy),
                _ptr(top_ids), _ptr(top_lp), ws, n, _ptr(err_flag), st), workspace, need)


def hydra_token_logprobs_backward(logits, tokens, lse, d_logits, d_lp=None, entropy=None, d_entropy=None,
                                  err_flag=None, stream=None) -> None:
    """Gradient of hydra_token_logprobs' lp and entropy with respect to the logits (see include/hydra.h).

    logits, d_logits [M,V]: bf16 (or 16-bit integer tensors holding bf16 bits) or float32, rows contiguous and possibly
    apart (d_logits may be logits); tokens [M] int32; lse, d_lp [M] float32; entropy, d_entropy [M] float32 (d_entropy
    needs entropy).  Rows whose d_lp and d_entropy are 0 get zeros.
    """
    st = (_nat or _native()).token_logprobs_backward(logits, tokens, lse, d_logits, d_lp, entropy, d_entropy, err_flag,
                                                     stream)
    if st == _SLOW:
        return _hydra_token_logprobs_backward(logits, tokens, lse, d_logits, d_lp, entropy, d_entropy, err_flag, stream)
    if st != HYDRA_OK:
        _check(st, "hydra_token_logprobs_backward")


def _hydra_token_logprobs_backward(logits, tokens, lse, d_logits, d_lp, entropy, d_entropy, err_flag, stream) -> None:
    torch = _torch()
    ld = _rows(logits, "logits")
    M, V = logits.shape
    ld_d = _rows(d_logits, "d_logits", (M, V))
    _need(tokens, "tokens", (torch.int32,), (M,))
    for name, t in (("lse", lse), ("d_lp", d_lp), ("entropy", entropy), ("d_entropy", d_entropy)):
        _need(t, name, (torch.float32,), (M,))
    _need(err_flag, "err_flag", (torch.int32,), (1,))
    _launch("hydra_token_logprobs_backward", (logits, tokens, lse, d_logits, d_lp, entropy, d_entropy, err_flag), stream,
            lambda ws, n, st: lib().hydra_token_logprobs_backward(
                _ptr(logits), _type(logits), ld, _ptr(tokens), _ptr(lse), _ptr(entropy), _ptr(d_lp), _ptr(d_entropy), M,
                V, _ptr(d_logits), _type(d_logits), ld_d, _ptr(err_flag), st))


def hydra_grad_norm_workspace_bytes() -> int:
    out = ctypes.c_size_t(0)
    _check(lib().hydra_grad_norm_workspace_bytes(ctypes.byref(out)), "hydra_grad_norm_workspace_bytes")
    return int(out.value)


def _grad_workspace(workspace, norm, stream):
    """The workspace given, or one on the current stream's device where the call goes there: hundreds of tensors take
    the Python checks a millisecond, the native ones tens of microseconds."""
    torch = _torch()
    if workspace is None and stream is None and isinstance(norm, torch.Tensor) and norm.is_cuda and \
            norm.get_device() == torch.cuda.current_device():
        return torch.empty(hydra_grad_norm_workspace_bytes(), dtype=torch.uint8, device=norm.device)
    return workspace


def hydra_grad_norm(grads, norm, workspace=None, stream=None) -> None:
    """norm [1] float32 = the norm over all the tensors of `grads` (see include/hydra.h).

    grads: a sequence of contiguous tensors of any shape, bf16 (or 16-bit integer tensors holding bf16 bits) or
    float32.  Allocates the workspace (hydra_grad_norm_workspace_bytes()) if none is given.
    """
    workspace = _grad_workspace(workspace, norm, stream)
    st = (_nat or _native()).grad_clip(grads, None, norm, None, workspace, None, stream)
    if st == _SLOW:
        return _hydra_grad("hydra_grad_norm", grads, None, norm, None, workspace, None, stream)
    if st != HYDRA_OK:
        _check(st, "hydra_grad_norm")


def hydra_grad_clip(grads, max_norm: float, norm, outs=None, workspace=None, err_flag=None, stream=None) -> None:
    """hydra_grad_norm, and the gradients scaled to a norm of at most max_norm: in place, or into `outs` (see
    include/hydra.h).

    outs: None, or a sequence of contiguous tensors of the gradients' shapes, bf16 or float32; err_flag [1] int32 gets
    1 OR-ed in when the norm is not finite (nothing is scaled then).
    """
    if max_norm is None:
        raise TypeError("max_norm must be a number")
    workspace = _grad_workspace(workspace, norm, stream)
    st = (_nat or _native()).grad_clip(grads, max_norm, norm, outs, workspace, err_flag, stream)
    if st == _SLOW:
        return _hydra_grad("hydra_grad_clip", grads, max_norm, norm, outs, workspace, err_flag, stream)
    if st != HYDRA_OK:
        _check(st, "hydra_grad_clip")


def _hydra_grad(where, grads, max_norm, norm, outs, workspace, err_flag, stream) -> None:
    torch = _torch()
    grads = list(grads)
    n = len(grads)
    for i, g in enumerate(grads):
        if g is None:
            raise TypeError(f"grads[{i}] must be a torch.Tensor")
        _need(g, f"grads[{i}]", _any_types())
    _need(norm, "norm", (torch.float32,), (1,))
    _need(err_flag, "err_flag", (torch.int32,), (1,))
    if outs is not None:
        outs = list(outs)
        if len(outs) != n:
            raise ValueError("outs must have one tensor for each gradient")
        for i, o in enumerate(outs):
            if o is None:
                raise TypeError(f"outs[{i}] must be a torch.Tensor")
            _need(o, f"outs[{i}]", _any_types(), grads[i].shape)
    types = (ctypes.c_int32 * n)(*[_type(g) for g in grads])
    numels = (ctypes.c_int64 * n)(*[g.numel() for g in grads])
    head = (n, _ptr_array(grads), types, numels)

    def call(ws, nbytes, st):
        if max_norm is None:
            return lib().hydra_grad_norm(*head, _ptr(norm), ws, nbytes, st)
        return lib().hydra_grad_clip(*head, float(max_norm), _ptr(norm), None if outs is None else _ptr_array(outs),
                                     None if outs is None else (ctypes.c_int32 * n)(*[_type(o) for o in outs]), ws,
                                     nbytes, _ptr(err_flag), st)

    _launch(where, (*grads, norm, *(outs or ()), err_flag), stream, call, workspace, hydra_grad_norm_workspace_bytes())


# ------------------------------------------------------------------ the base in 8 bits, dropout, drafted tokens
#
# As above, these calls go to the device that their tensors are on.

def _fp8_types():
    torch = _torch()
    return (torch.float8_e4m3fn, torch.uint8)


def _scale_types():
    torch = _torch()
    return (torch.uint8, torch.float8_e8m0fnu)


def _blocks(n, rows=128) -> int:
    return -(-n // rows)


def hydra_fp8_quantize(x, q, scale, block_rows: int = 1, qt=None, scale_t=None, stream=None) -> None:
    """e4m3 values and power-of-two scales of a matrix, 128 values of a row (block_rows 1) or 128 x 128 (block_rows 128)
    to a scale (see include/hydra.h).

    x [M,K]: bf16 (or 16-bit integer tensors holding bf16 bits) or float32; q [M,K]: float8_e4m3fn (or uint8); scale
    [M or ceil(M/128), ceil(K/128)]: uint8 (or float8_e8m0fnu); qt [K,M], scale_t [ceil(K/128), ceil(M/128)]: the
    transposed copy, with block_rows 128 (both optional, together).
    """
    st = (_nat or _native()).fp8_quantize(x, q, scale, block_rows, qt, scale_t, stream)
    if st == _SLOW:
        return _hydra_fp8_quantize(x, q, scale, block_rows, qt, scale_t, stream)
    if st != HYDRA_OK:
        _check(st, "hydra_fp8_quantize")


def _hydra_fp8_quantize(x, q, scale, block_rows, qt, scale_t, stream) -> None:
    _need(x, "x", _any_types())
    M, K = x.shape
    rows = int(block_rows)
    if rows not in (1, 128):
        raise ValueError(f"block_rows must be 1 or 128, got {block_rows}")
    _need(q, "q", _fp8_types(), (M, K))
    _need(scale, "scale", _scale_types(), (_blocks(M, rows), _blocks(K)))
    _need(qt, "qt", _fp8_types(), (K, M))
    _need(scale_t, "scale_t", _scale_types(), (_blocks(K), _blocks(M, rows)))
    _launch("hydra_fp8_quantize", (x, q, scale, qt, scale_t), stream, lambda ws, n, st: lib().hydra_fp8_quantize(
        _ptr(x), _type(x), M, K, rows, _ptr(q), _ptr(scale), _ptr(qt), _ptr(scale_t), st))


def hydra_fp8_lora_linear_workspace_bytes(M: int, N: int, K: int, r: int) -> int:
    out = ctypes.c_size_t(0)
    _check(lib().hydra_fp8_lora_linear_workspace_bytes(int(M), int(N), int(K), int(r), ctypes.byref(out)),
           "hydra_fp8_lora_linear_workspace_bytes")
    return int(out.value)


def hydra_fp8_lora_linear(x, Wq, w_scale, A, B, s: float, y_off=None, y_on=None, x_adapter=None, xq=None, x_scale=None,
                          workspace=None, stream=None) -> None:
    """y_off = x W^T and/or y_on = x W^T + s (x_adapter A^T) B^T over a weight in 8 bits (see include/hydra.h).

    x [M,K] bf16 (or 16-bit integer tensors holding bf16 bits; may be None where xq is given and x_adapter is not
    needed or given); Wq [N,K], w_scale [ceil(N/128), ceil(K/128)] from hydra_fp8_quantize with block_rows 128; A [r,K],
    B [N,r] bf16; y_off, y_on [M,N]: bf16 or float32, both the same (either may be None); x_adapter [M,K] bf16: the
    adapter's own input (None: x); xq [M,K], x_scale [M, ceil(K/128)]: x already quantized.  Allocates the workspace if
    none is given.
    """
    st = (_nat or _native()).fp8_lora_linear(x, Wq, w_scale, A, B, s, y_off, y_on, x_adapter, xq, x_scale, workspace,
                                             stream)
    if st == _SLOW:
        return _hydra_fp8_lora_linear(x, Wq, w_scale, A, B, s, y_off, y_on, x_adapter, xq, x_scale, workspace, stream)
    if st != HYDRA_OK:
        _check(st, "hydra_fp8_lora_linear")


def _hydra_fp8_lora_linear(x, Wq, w_scale, A, B, s, y_off, y_on, x_adapter, xq, x_scale, workspace, stream) -> None:
    bf = _bf16_types()
    if x is None and xq is None:
        raise ValueError("x or xq is needed")
    _need(Wq, "Wq", _fp8_types())
    N, K = Wq.shape
    M = (xq if x is None else x).shape[0]
    r = 0 if A is None else A.shape[0]
    _need(w_scale, "w_scale", _scale_types(), (_blocks(N), _blocks(K)))
    for name, t in (("x", x), ("x_adapter", x_adapter)):
        _need(t, name, bf, (M, K))
    _need(xq, "xq", _fp8_types(), (M, K))
    _need(x_scale, "x_scale", _scale_types(), (M, _blocks(K)))
    _need(A, "A", bf, (r, K))
    _need(B, "B", bf, (N, r))
    for name, t in (("y_off", y_off), ("y_on", y_on)):
        _need(t, name, _any_types(), (M, N))
    if y_off is not None and y_on is not None and _type(y_off) != _type(y_on):
        raise TypeError(f"y_off is {y_off.dtype}, y_on {y_on.dtype}")
    y_type = _type(y_on if y_off is None else y_off)
    _launch("hydra_fp8_lora_linear", (x, Wq, w_scale, A, B, y_off, y_on, x_adapter, xq, x_scale), stream,
            lambda ws, n, st: lib().hydra_fp8_lora_linear(
                _ptr(x), _ptr(x_adapter), _ptr(xq), _ptr(x_scale), _ptr(Wq), _ptr(w_scale), _ptr(A), _ptr(B), float(s), M,
                N, K, r, _ptr(y_off), _ptr(y_on), y_type, ws, n, st),
            workspace, hydra_fp8_lora_linear_workspace_bytes(M, N, K, r))


def hydra_fp8_lora_linear_backward_workspace_bytes(M: int, N: int, K: int, r: int) -> int:
    out = ctypes.c_size_t(0)
    _check(lib().hydra_fp8_lora_linear_backward_workspace_bytes(int(M), int(N), int(K), int(r), ctypes.byref(out)),
           "hydra_fp8_lora_linear_backward_workspace_bytes")
    return int(out.value)


def hydra_fp8_lora_linear_backward(x, Wqt, wt_scale, A, B, s: float, dy, dx=None, dA=None, dB=None, p: float = 0.0,
                                   rng=None, workspace=None, stream=None) -> None:
    """dx, dA, dB of hydra_fp8_lora_linear's y_on, with dropout of probability p on the adapter's input (see
    include/hydra.h).

    x [M,K] bf16: the adapter's input of the forward (after dropout); Wqt [K,N], wt_scale [ceil(K/128), ceil(N/128)]: qt
    and scale_t of hydra_fp8_quantize (needed for dx alone); A [r,K], B [N,r], dy [M,N] bf16; dx [M,K]: bf16 or float32,
    dA [r,K], dB [N,r] float32 outputs (each optional); rng [2] int64: the forward's seed and offset, on the device.
    Allocates the workspace if none is given.
    """
    st = (_nat or _native()).fp8_lora_linear_backward(x, Wqt, wt_scale, A, B, s, dy, dx, dA, dB, p, rng, workspace, stream)
    if st == _SLOW:
        return _hydra_fp8_lora_linear_backward(x, Wqt, wt_scale, A, B, s, dy, dx, dA, dB, p, rng, workspace, stream)
    if st != HYDRA_OK:
        _check(st, "hydra_fp8_lora_linear_backward")


def _hydra_fp8_lora_linear_backward(x, Wqt, wt_scale, A, B, s, dy, dx, dA, dB, p, rng, workspace, stream) -> None:
    torch = _torch()
    bf = _bf16_types()
    _need(dy, "dy", bf)
    M, N = dy.shape
    if A is None and x is None and Wqt is None:
        raise ValueError("A, x or Wqt is needed")
    K = A.shape[1] if A is not None else (x.shape[1] if x is not None else Wqt.shape[0])
    r = 0 if A is None else A.shape[0]
    _need(x, "x", bf, (M, K))
    _need(Wqt, "Wqt", _fp8_types(), (K, N))
    _need(wt_scale, "wt_scale", _scale_types(), (_blocks(K), _blocks(N)))
    _need(A, "A", bf, (r, K))
    _need(B, "B", bf, (N, r))
    _need(dx, "dx", _any_types(), (M, K))
    _need(dA, "dA", (torch.float32,), (r, K))
    _need(dB, "dB", (torch.float32,), (N, r))
    _need(rng, "rng", (torch.int64, torch.uint64), (2,))
    _launch("hydra_fp8_lora_linear_backward", (x, Wqt, wt_scale, A, B, dy, dx, dA, dB, rng), stream,
            lambda ws, n, st: lib().hydra_fp8_lora_linear_backward(
                _ptr(x), _ptr(Wqt), _ptr(wt_scale), _ptr(A), _ptr(B), float(s), _ptr(dy), M, N, K, r, float(p), _ptr(rng),
                _ptr(dx), _type(dx), _ptr(dA), _ptr(dB), ws, n, st),
            workspace, hydra_fp8_lora_linear_backward_workspace_bytes(M, N, K, r))


def hydra_dropout(x, y, p: float, rng, residual=None, stream=None) -> None:
    """y = residual + (x scaled where it is kept, else 0), the mask from seed and offset alone (see include/hydra.h).

    x, y and residual: contiguous tensors of one shape, bf16 (or 16-bit integer tensors holding bf16 bits) or float32, each
    of its own type (y may be x or residual); rng [2] int64 on the device: seed and offset.  The gradient with respect
    to x is the same call on dy.
    """
    st = (_nat or _native()).dropout(x, y, p, rng, residual, stream)
    if st == _SLOW:
        return _hydra_dropout(x, y, p, rng, residual, stream)
    if st != HYDRA_OK:
        _check(st, "hydra_dropout")


def _hydra_dropout(x, y, p, rng, residual, stream) -> None:
    torch = _torch()
    _need(x, "x", _any_types())
    if x is None or y is None:
        raise TypeError("x and y must be torch.Tensors")
    _need(y, "y", _any_types(), x.shape)
    _need(residual, "residual", _any_types(), x.shape)
    _need(rng, "rng", (torch.int64, torch.uint64), (2,))
    _launch("hydra_dropout", (x, y, rng, residual), stream, lambda ws, n, st: lib().hydra_dropout(
        _ptr(x), _type(x), _ptr(residual), _type(residual), float(p), _ptr(rng), x.numel(), _ptr(y), _type(y), st))


def hydra_verify_drafts_workspace_bytes(n: int, k: int, V: int) -> int:
    out = ctypes.c_size_t(0)
    _check(lib().hydra_verify_drafts_workspace_bytes(int(n), int(k), int(V), ctypes.byref(out)),
           "hydra_verify_drafts_workspace_bytes")
    return int(out.value)


def hydra_verify_drafts(target, draft, drafts, u, accepted, tokens, lp=None, lens=None, temperature: float = 1.0,
                        workspace=None, err_flag=None, stream=None) -> None:
    """Drafted tokens against the target's probabilities, and the next token, from given random numbers (see
    include/hydra.h).

    target [n*(k+1),V], draft [n*k,V] (None: drafts without a distribution): bf16 (or 16-bit integer tensors holding
    bf16 bits) or float32, each of its own type, rows contiguous and possibly apart; drafts [n,k] int32 (None for k = 0);
    u [n,k+1] float32; accepted [n], tokens [n,k+1] int32, lp [n,k+1] float32 (optional) outputs; lens [n] int32: how many
    drafts each sequence has (None: all).  Allocates the workspace if none is given.
    """
    st = (_nat or _native()).verify_drafts(target, draft, drafts, u, accepted, tokens, lp, lens, temperature, workspace,
                                           err_flag, stream)
    if st == _SLOW:
        return _hydra_verify_drafts(target, draft, drafts, u, accepted, tokens, lp, lens, temperature, workspace, err_flag,
                                    stream)
    if st != HYDRA_OK:
        _check(st, "hydra_verify_drafts")


def _hydra_verify_drafts(target, draft, drafts, u, accepted, tokens, lp, lens, temperature, workspace, err_flag,
                         stream) -> None:
    torch = _torch()
    _need(u, "u", (torch.float32,))
    if u is None or u.dim() != 2 or u.shape[1] < 1:
        raise ValueError("u must have the shape [n, k + 1]")
    n, k = u.shape[0], u.shape[1] - 1
    ld = _rows(target, "target")
    V = target.shape[1]
    _rows(target, "target", (n * (k + 1), V))
    ld_d = 0 if draft is None else _rows(draft, "draft", (n * k, V))
    _need(drafts, "drafts", (torch.int32,), (n, k))
    for name, t, shape in (("accepted", accepted, (n,)), ("tokens", tokens, (n, k + 1)), ("lens", lens, (n,)),
                           ("err_flag", err_flag, (1,))):
        _need(t, name, (torch.int32,), shape)
    _need(lp, "lp", (torch.float32,), (n, k + 1))
    _launch("hydra_verify_drafts", (target, draft, drafts, u, accepted, tokens, lp, lens, err_flag), stream,
            lambda ws, nb, st: lib().hydra_verify_drafts(
                _ptr(target), _type(target), ld, _ptr(draft), _type(draft), ld_d, _ptr(drafts), _ptr(lens), _ptr(u), n, k, V,
                float(temperature), _ptr(accepted), _ptr(tokens), _ptr(lp), ws, nb, _ptr(err_flag), st),
            workspace, hydra_verify_drafts_workspace_bytes(n, k, V))
