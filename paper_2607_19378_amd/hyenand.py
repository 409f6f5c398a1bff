"""Python binding of libhyenand (ctypes): argument marshalling only.

Every step of the operation runs in the HIP kernels behind the C ABI declared
in include/hyenand.h; PyTorch only provides device memory and the stream.
There is no fallback: if the library is missing or cannot be loaded, every
call raises.
"""
from __future__ import annotations

import ctypes
import functools
import math
import os
import threading
from typing import Optional, Sequence

_PKG = os.path.dirname(os.path.abspath(__file__))
# HYENAND_LIBRARY selects another build of the same library (the sanitizer
# build of paper_2607_19378_amd.build --sanitize)
LIB_PATH = os.environ.get("HYENAND_LIBRARY") or os.path.join(_PKG, "libhyenand.so")

OK, ERR_INVALID_ARGUMENT, ERR_UNSUPPORTED, ERR_WORKSPACE_TOO_SMALL, ERR_HIP = range(5)
PAD_LINEAR, PAD_CIRCULAR, PAD_CENTERED = 0, 1, 2
DTYPE_F32, DTYPE_BF16 = 0, 1

EXPORTED = ("hyenand_fftconv", "hyenand_fftconv_shared_k", "hyenand_fftconv_noalloc", "hyenand_fftconv_modal", "hyenand_fftconv_workspace_size",
            "hyenand_fftconv_shared_k_workspace_size", "hyenand_fftconv_workspace_min",
            "hyenand_kernel_spectrum_size", "hyenand_kernel_spectrum", "hyenand_fftconv_spectrum",
            "hyenand_fftconv_plan_name", "hyenand_fftconv_backward", "hyenand_fftconv_backward_workspace_size",
            "hyenand_fftconv_backward_workspace_min", "hyenand_operator", "hyenand_operator_workspace_size",
            "hyenand_kernel_synth", "hyenand_modal_filter", "hyenand_scan", "hyenand_scan_workspace_size",
            "hyenand_scan_backward", "hyenand_scan_backward_workspace_size", "hyenand_scan_step", "hyenand_block_norm",
            "hyenand_block_norm_backward", "hyenand_block_norm_backward_workspace_size", "hyenand_status_string", "hyenand_last_error", "hyenand_version")

_lock = threading.Lock()
_lib = None


class HyenandError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(msg)
        self.status = status


def lib() -> ctypes.CDLL:
    """Load libhyenand.so (built in-tree by paper_2607_19378_amd.build)."""
    global _lib
    with _lock:
        if _lib is None:
            if not os.path.exists(LIB_PATH):
                raise RuntimeError(f"{LIB_PATH} is not built; run `python -m paper_2607_19378_amd.build`")
            # torch first: its HIP runtime then satisfies the library's
            # dependency on libamdhip64.so.7, so the process holds one HIP
            # runtime.  Loaded before torch, the library would bring in the
            # system one beside torch's, and whichever of the two initialises
            # second finds no device.
            import torch  # noqa: F401
            L = ctypes.CDLL(LIB_PATH)
            i64p = ctypes.POINTER(ctypes.c_int64)
            vp = ctypes.c_void_p
            L.hyenand_fftconv.argtypes = [vp, vp, vp, vp, vp, vp, ctypes.c_int, i64p, ctypes.c_int,
                                          ctypes.c_int, vp, ctypes.c_size_t, vp]
            L.hyenand_fftconv.restype = ctypes.c_int
            L.hyenand_fftconv_shared_k.argtypes = L.hyenand_fftconv.argtypes
            L.hyenand_fftconv_shared_k.restype = ctypes.c_int
            L.hyenand_fftconv_noalloc.argtypes = [vp, vp, vp, vp, vp, vp, ctypes.c_int, i64p, ctypes.c_int,
                                                  ctypes.c_int, vp]
            L.hyenand_fftconv_noalloc.restype = ctypes.c_int
            L.hyenand_fftconv_modal.argtypes = [vp] * 7 + [ctypes.c_int, vp, vp, ctypes.c_int, i64p, ctypes.c_int,
                                                           ctypes.c_int, vp, ctypes.c_size_t, vp]
            L.hyenand_fftconv_modal.restype = ctypes.c_int
            L.hyenand_kernel_spectrum.argtypes = [vp, vp, ctypes.c_size_t, ctypes.c_int, i64p, ctypes.c_int,
                                                  ctypes.c_int, vp]
            L.hyenand_kernel_spectrum.restype = ctypes.c_int
            L.hyenand_fftconv_spectrum.argtypes = [vp, vp, vp, vp, ctypes.c_size_t, vp, vp, ctypes.c_int, i64p,
                                                   ctypes.c_int, ctypes.c_int, vp]
            L.hyenand_fftconv_spectrum.restype = ctypes.c_int
            for name in ("hyenand_fftconv_workspace_size", "hyenand_fftconv_shared_k_workspace_size",
                         "hyenand_fftconv_workspace_min", "hyenand_kernel_spectrum_size"):
                f = getattr(L, name)
                f.argtypes = [ctypes.c_int, i64p, ctypes.c_int, ctypes.c_int,
                              ctypes.POINTER(ctypes.c_size_t)]
                f.restype = ctypes.c_int
            L.hyenand_fftconv_backward.argtypes = [vp] * 11 + [ctypes.c_int, i64p, ctypes.c_int, ctypes.c_int, vp,
                                                           ctypes.c_size_t, vp]
            L.hyenand_fftconv_backward.restype = ctypes.c_int
            L.hyenand_fftconv_backward_workspace_size.argtypes = [ctypes.c_int, i64p, ctypes.c_int, ctypes.c_int,
                                                                  ctypes.POINTER(ctypes.c_size_t)]
            L.hyenand_fftconv_backward_workspace_size.restype = ctypes.c_int
            L.hyenand_fftconv_backward_workspace_min.argtypes = [ctypes.c_int, i64p, ctypes.c_int, ctypes.c_int,
                                                                 ctypes.POINTER(ctypes.c_size_t)]
            L.hyenand_fftconv_backward_workspace_min.restype = ctypes.c_int
            L.hyenand_operator.argtypes = [vp] * 7 + [ctypes.c_float, ctypes.c_float, vp, ctypes.c_int, i64p,
                                                      ctypes.c_int, ctypes.c_int, vp, ctypes.c_size_t, vp]
            L.hyenand_operator.restype = ctypes.c_int
            L.hyenand_operator_workspace_size.argtypes = [ctypes.c_int, i64p, ctypes.c_int, ctypes.c_int,
                                                          ctypes.POINTER(ctypes.c_size_t)]
            L.hyenand_operator_workspace_size.restype = ctypes.c_int
            L.hyenand_kernel_synth.argtypes = [vp] * 8 + [ctypes.c_int] * 3 + [vp, ctypes.c_int, i64p, ctypes.c_int,
                                                                       ctypes.c_int, vp]
            L.hyenand_kernel_synth.restype = ctypes.c_int
            L.hyenand_modal_filter.argtypes = [vp] * 4 + [ctypes.c_int, vp, ctypes.c_int64, ctypes.c_int64,
                                                       ctypes.c_int, vp]
            L.hyenand_modal_filter.restype = ctypes.c_int
            i64 = ctypes.c_int64
            L.hyenand_scan.argtypes = [vp] * 10 + [i64] * 3 + [ctypes.c_int, vp, ctypes.c_size_t, vp]
            L.hyenand_scan_backward.argtypes = [vp] * 15 + [i64] * 3 + [ctypes.c_int, vp, ctypes.c_size_t, vp]
            L.hyenand_scan_step.argtypes = [vp] * 8 + [i64] * 3 + [ctypes.c_int, vp]
            f32 = ctypes.c_float
            L.hyenand_block_norm.argtypes = [vp] * 6 + [f32] * 3 + [vp] * 3 + [i64] * 3 + [ctypes.c_int, vp]
            L.hyenand_block_norm_backward.argtypes = ([vp] * 6 + [f32] * 3 + [vp] * 9 + [i64] * 3
                                                      + [ctypes.c_int, vp, ctypes.c_size_t, vp])
            L.hyenand_block_norm.restype = L.hyenand_block_norm_backward.restype = ctypes.c_int
            for name in ("hyenand_scan_workspace_size", "hyenand_scan_backward_workspace_size",
                         "hyenand_block_norm_backward_workspace_size"):
                getattr(L, name).argtypes = [i64] * 3 + [ctypes.c_int, ctypes.POINTER(ctypes.c_size_t)]
                getattr(L, name).restype = ctypes.c_int
            L.hyenand_scan.restype = L.hyenand_scan_backward.restype = L.hyenand_scan_step.restype = ctypes.c_int
            L.hyenand_fftconv_plan_name.argtypes = [ctypes.c_int, i64p, ctypes.c_int, ctypes.c_int,
                                                    ctypes.c_char_p, ctypes.c_size_t]
            L.hyenand_fftconv_plan_name.restype = ctypes.c_int
            L.hyenand_status_string.argtypes = [ctypes.c_int]
            L.hyenand_status_string.restype = ctypes.c_char_p
            L.hyenand_last_error.argtypes = []
            L.hyenand_last_error.restype = ctypes.c_char_p
            L.hyenand_version.argtypes = []
            L.hyenand_version.restype = ctypes.c_int
            _lib = L
        return _lib


def _check(status: int) -> None:
    if status != OK:
        L = lib()
        detail = L.hyenand_last_error().decode()
        raise HyenandError(status, f"{L.hyenand_status_string(status).decode()}: {detail}")


def _dims(shape: Sequence[int]):
    arr = (ctypes.c_int64 * len(shape))(*[int(s) for s in shape])
    return len(shape) - 2, arr


_MODES = {"linear": 0, "circular": 1, "centered": 2}


def _mode(pad_mode: str) -> int:
    if pad_mode not in _MODES:
        raise ValueError(f"pad_mode must be 'linear', 'circular' or 'centered', got {pad_mode!r}")
    return _MODES[pad_mode]


def kernel_shape(shape, pad_mode: str, shared_k: bool = False):
    """Shape of k for tensors of `shape` ([B, C, L1..LN]): the same, or
    [B, C, 2 L1 - 1, ...] centered; without B with shared_k."""
    shape = tuple(int(x) for x in shape)
    grid = tuple(2 * x - 1 for x in shape[2:]) if pad_mode == "centered" else shape[2:]
    return (shape[1],) + grid if shared_k else shape[:2] + grid


def _dtype_code(dtype) -> int:
    import torch
    if dtype is torch.float32:
        return DTYPE_F32
    if dtype is torch.bfloat16:
        return DTYPE_BF16
    if dtype in ("f32", "float32"):
        return DTYPE_F32
    if dtype in ("bf16", "bfloat16"):
        return DTYPE_BF16
    raise ValueError(f"unsupported dtype {dtype}")


def workspace_size(shape, pad_mode: str, dtype, shared_k: bool = False) -> int:
    """Recommended workspace bytes of hyenand_fftconv (shared_k: of
    hyenand_fftconv_shared_k, which may use more to transform each channel's
    kernel once)."""
    nd, dims = _dims(shape)
    out = ctypes.c_size_t(0)
    fn = lib().hyenand_fftconv_shared_k_workspace_size if shared_k else lib().hyenand_fftconv_workspace_size
    _check(fn(nd, dims, _mode(pad_mode), _dtype_code(dtype), ctypes.byref(out)))
    return int(out.value)


def workspace_min(shape, pad_mode: str, dtype) -> int:
    nd, dims = _dims(shape)
    out = ctypes.c_size_t(0)
    _check(lib().hyenand_fftconv_workspace_min(nd, dims, _mode(pad_mode), _dtype_code(dtype),
                                               ctypes.byref(out)))
    return int(out.value)


def plan_name(shape, pad_mode: str, dtype) -> str:
    nd, dims = _dims(shape)
    buf = ctypes.create_string_buffer(64)
    _check(lib().hyenand_fftconv_plan_name(nd, dims, _mode(pad_mode), _dtype_code(dtype), buf, 64))
    return buf.value.decode()


def version() -> int:
    return int(lib().hyenand_version())


def _ptr(t) -> int:
    return int(t.data_ptr())


def _keep_for_stream(stream, *tensors) -> None:
    """Tensors this module allocates on the current stream but hands to work
    on another `stream`: mark them used there, so that torch's caching
    allocator does not give their memory to a later allocation on the
    current stream while that work is still pending."""
    import torch
    if stream is None:
        return
    for t in tensors:
        if t is not None and stream != torch.cuda.current_stream(t.device):
            t.record_stream(stream)


class Prepared:
    """One hyenand_fftconv call with its arguments checked and marshalled
    once; calling the object enqueues the work again on the same buffers and
    stream (for loops that repeat a call, where per-call Python work would
    otherwise delay the launches)."""

    def __init__(self, y, x1, x2, v, k, D, pad_mode: str = "linear", workspace=None, stream=None,
                 shared_k: bool = False):
        import torch
        shape = tuple(x1.shape)
        kshape = kernel_shape(shape, pad_mode, shared_k)
        for t, want in ((x1, shape), (x2, shape), (v, shape), (k, kshape), (y, shape)):
            if not t.is_cuda:
                raise ValueError("all tensors must be on the GPU")
            if tuple(t.shape) != want or t.dtype != x1.dtype:
                raise ValueError(f"x1, x2, v, y must share shape and dtype; k must be {kshape} "
                                 f"(pad_mode {pad_mode!r}, shared_k {shared_k})")
            if not t.is_contiguous():
                raise ValueError("tensors must be contiguous")
        if not D.is_cuda or D.dtype != x1.dtype or tuple(D.shape) != (shape[1],) or not D.is_contiguous():
            raise ValueError("D must be a contiguous [C] GPU tensor of the same dtype")
        nd, dims = _dims(shape)
        if stream is None:
            stream = torch.cuda.current_stream(x1.device)
        ws_ptr, ws_bytes = None, 0
        if workspace is not None:
            ws_ptr, ws_bytes = _ptr(workspace), workspace.numel() * workspace.element_size()
        self._fn = lib().hyenand_fftconv_shared_k if shared_k else lib().hyenand_fftconv
        self._args = (_ptr(x1), _ptr(x2), _ptr(v), _ptr(k), _ptr(D), _ptr(y), nd, dims, _mode(pad_mode),
                      _dtype_code(x1.dtype), ws_ptr, ws_bytes, ctypes.c_void_p(stream.cuda_stream))
        self._keep = (y, x1, x2, v, k, D, workspace, stream)  # the buffers outlive the object

    def __call__(self) -> None:
        status = self._fn(*self._args)
        if status != OK:
            _check(status)


def fftconv_into(y, x1, x2, v, k, D, pad_mode: str = "linear", workspace=None,
                 stream=None, shared_k: bool = False) -> None:
    """y <- x2 * (k conv (x1*v) + D*(x1*v)); all tensors already allocated on
    the GPU.  shared_k: k is [C, L...], one kernel per channel for every sample."""
    Prepared(y, x1, x2, v, k, D, pad_mode, workspace, stream, shared_k)()


class PreparedModalConv:
    """One hyenand_fftconv_modal call with its arguments checked and
    marshalled once (see Prepared): y from x1, x2, v, D and the [C, M] modal
    filter parameters, the filter generated inside the transform kernels."""

    def __init__(self, y, x1, x2, v, log_mag, angle, res_re, res_im, D, pad_mode: str = "linear", workspace=None,
                 stream=None):
        import torch
        shape = tuple(x1.shape)
        for t in (x1, x2, v, y):
            if not t.is_cuda or tuple(t.shape) != shape or t.dtype != x1.dtype or not t.is_contiguous():
                raise ValueError("x1, x2, v, y must be contiguous GPU tensors of one shape and dtype")
        C, M = (int(n) for n in log_mag.shape)
        if C != shape[1]:
            raise ValueError("the modal parameters must be [C, M]")
        for t in (log_mag, angle, res_re, res_im):
            if not t.is_cuda or t.dtype != torch.float32 or tuple(t.shape) != (C, M) or not t.is_contiguous():
                raise ValueError("log_mag, angle, res_re, res_im must be contiguous fp32 [C, M] GPU tensors")
        if not D.is_cuda or D.dtype != x1.dtype or tuple(D.shape) != (C,) or not D.is_contiguous():
            raise ValueError("D must be a contiguous [C] GPU tensor of the same dtype")
        if workspace is None:
            nbytes = workspace_size(shape, pad_mode, x1.dtype)
            workspace = torch.empty(max(1, nbytes), dtype=torch.uint8, device=x1.device)
            _keep_for_stream(stream, workspace)
        if stream is None:
            stream = torch.cuda.current_stream(x1.device)
        nd, dims = _dims(shape)
        self._fn = lib().hyenand_fftconv_modal
        self._args = (_ptr(x1), _ptr(x2), _ptr(v), _ptr(log_mag), _ptr(angle), _ptr(res_re), _ptr(res_im), M,
                      _ptr(D), _ptr(y), nd, dims, _mode(pad_mode), _dtype_code(x1.dtype), _ptr(workspace),
                      workspace.numel() * workspace.element_size(), ctypes.c_void_p(stream.cuda_stream))
        self._keep = (y, x1, x2, v, log_mag, angle, res_re, res_im, D, workspace, stream)

    def __call__(self) -> None:
        status = self._fn(*self._args)
        if status != OK:
            _check(status)


def fftconv_modal(x1, x2, v, log_mag, angle, res_re, res_im, D, pad_mode: str = "linear", workspace=None,
                  stream=None):
    """y = x2 * (k conv (x1*v) + D*(x1*v)) with k[c] the order-M modal filter
    of channel c (generated inside the transform kernels); torch-allocated y."""
    import torch
    y = torch.empty_like(x1)
    PreparedModalConv(y, x1, x2, v, log_mag, angle, res_re, res_im, D, pad_mode, workspace, stream)()
    _keep_for_stream(stream, y)
    return y


def kernel_spectrum_size(shape, pad_mode: str, dtype) -> int:
    """Bytes of the kept spectra of one kernel per channel for convolutions of
    this [B, C, L1, L2] shape (single-pass 2D plan only)."""
    nd, dims = _dims(shape)
    out = ctypes.c_size_t(0)
    _check(lib().hyenand_kernel_spectrum_size(nd, dims, _mode(pad_mode), _dtype_code(dtype), ctypes.byref(out)))
    return int(out.value)


def kernel_spectrum(k, shape, pad_mode: str = "linear", stream=None):
    """Transform a static kernel k [C, L1, L2] once for convolutions of the
    given [B, C, L1, L2] shape; returns the spectra as a torch uint8 tensor
    (layout private to the library) for fftconv_spectrum."""
    import torch
    shape = tuple(shape)
    if not k.is_cuda or not k.is_contiguous() or tuple(k.shape) != (shape[1],) + shape[2:]:
        raise ValueError(f"k must be a contiguous GPU tensor of shape {(shape[1],) + shape[2:]}")
    khat = torch.empty(kernel_spectrum_size(shape, pad_mode, k.dtype), dtype=torch.uint8, device=k.device)
    if stream is None:
        stream = torch.cuda.current_stream(k.device)
    nd, dims = _dims(shape)
    _check(lib().hyenand_kernel_spectrum(_ptr(k), _ptr(khat), khat.numel(), nd, dims, _mode(pad_mode),
                                         _dtype_code(k.dtype), ctypes.c_void_p(stream.cuda_stream)))
    _keep_for_stream(stream, khat)
    return khat


def fftconv_spectrum(x1, x2, v, khat, D, pad_mode: str = "linear", stream=None):
    """y = x2 * (k conv (x1*v) + D*(x1*v)) for the static kernel whose spectra
    kernel_spectrum returned; torch-allocated y."""
    import torch
    shape = tuple(x1.shape)
    for t in (x1, x2, v):
        if not t.is_cuda or tuple(t.shape) != shape or t.dtype != x1.dtype or not t.is_contiguous():
            raise ValueError("x1, x2, v must be contiguous GPU tensors of one shape and dtype")
    if not D.is_cuda or D.dtype != x1.dtype or tuple(D.shape) != (shape[1],) or not D.is_contiguous():
        raise ValueError("D must be a contiguous [C] GPU tensor of the same dtype")
    if not khat.is_cuda or khat.dtype != torch.uint8:
        raise ValueError("khat must be the uint8 GPU tensor kernel_spectrum returned")
    y = torch.empty_like(x1)
    if stream is None:
        stream = torch.cuda.current_stream(x1.device)
    nd, dims = _dims(shape)
    _check(lib().hyenand_fftconv_spectrum(_ptr(x1), _ptr(x2), _ptr(v), _ptr(khat), khat.numel(), _ptr(D), _ptr(y),
                                          nd, dims, _mode(pad_mode), _dtype_code(x1.dtype),
                                          ctypes.c_void_p(stream.cuda_stream)))
    _keep_for_stream(stream, y)
    return y


NOALLOC_SCRATCH_BYTES = 128 << 20


def fftconv_noalloc_into(y, x1, x2, v, k, D, pad_mode: str = "linear", stream=None) -> None:
    """y <- x2 * (k conv (x1*v) + D*(x1*v)) through hyenand_fftconv_noalloc:
    no workspace argument, the library's static device scratch instead
    (calls overlapping on one GPU race on it)."""
    import torch
    shape = tuple(x1.shape)
    for t, want in ((x1, shape), (x2, shape), (v, shape), (k, kernel_shape(shape, pad_mode)), (y, shape)):
        if not t.is_cuda or tuple(t.shape) != want or t.dtype != x1.dtype or not t.is_contiguous():
            raise ValueError("x1, x2, v, y must be contiguous GPU tensors of one shape and dtype; "
                             f"k must be {kernel_shape(shape, pad_mode)}")
    if not D.is_cuda or D.dtype != x1.dtype or tuple(D.shape) != (shape[1],) or not D.is_contiguous():
        raise ValueError("D must be a contiguous [C] GPU tensor of the same dtype")
    if stream is None:
        stream = torch.cuda.current_stream(x1.device)
    nd, dims = _dims(shape)
    _check(lib().hyenand_fftconv_noalloc(_ptr(x1), _ptr(x2), _ptr(v), _ptr(k), _ptr(D), _ptr(y), nd, dims,
                                         _mode(pad_mode), _dtype_code(x1.dtype),
                                         ctypes.c_void_p(stream.cuda_stream)))


def fftconv(x1, x2, v, k, D, pad_mode: str = "linear", workspace=None, stream=None, shared_k: bool = False):
    """Allocate y (and, unless given, the workspace) with torch and run the op."""
    import torch
    y = torch.empty_like(x1)
    own = None
    if workspace is None:
        nbytes = workspace_size(tuple(x1.shape), pad_mode, x1.dtype, shared_k)
        if nbytes:
            workspace = own = torch.empty(nbytes, dtype=torch.uint8, device=x1.device)
    fftconv_into(y, x1, x2, v, k, D, pad_mode, workspace, stream, shared_k)
    _keep_for_stream(stream, y, own)
    return y


def backward_workspace_size(shape, pad_mode: str, dtype) -> int:
    nd, dims = _dims(shape)
    out = ctypes.c_size_t(0)
    _check(lib().hyenand_fftconv_backward_workspace_size(nd, dims, _mode(pad_mode), _dtype_code(dtype),
                                                         ctypes.byref(out)))
    return int(out.value)


def backward_workspace_min(shape, pad_mode: str, dtype) -> int:
    nd, dims = _dims(shape)
    out = ctypes.c_size_t(0)
    _check(lib().hyenand_fftconv_backward_workspace_min(nd, dims, _mode(pad_mode), _dtype_code(dtype),
                                                        ctypes.byref(out)))
    return int(out.value)


class PreparedBackward:
    """One hyenand_fftconv_backward call with its arguments checked and
    marshalled once (see Prepared)."""

    def __init__(self, gx1, gx2, gv, gk, gD, x1, x2, v, k, D, gy, pad_mode: str = "linear", workspace=None,
                 stream=None):
        import torch
        shape = tuple(x1.shape)
        kshape = kernel_shape(shape, pad_mode)
        for t in (x1, x2, v, k, gy, gx1, gx2, gv, gk):
            want = kshape if (t is k or t is gk) else shape
            if not t.is_cuda or tuple(t.shape) != want or t.dtype != x1.dtype or not t.is_contiguous():
                raise ValueError("x1, x2, v, gy, gx1, gx2, gv must be contiguous GPU tensors of one shape and "
                                 f"dtype; k and gk {kshape} (pad_mode {pad_mode!r})")
        for t in (D, gD):
            if not t.is_cuda or t.dtype != x1.dtype or tuple(t.shape) != (shape[1],) or not t.is_contiguous():
                raise ValueError("D and gD must be contiguous [C] GPU tensors of the same dtype")
        nd, dims = _dims(shape)
        if workspace is None:
            workspace = torch.empty(backward_workspace_size(shape, pad_mode, x1.dtype), dtype=torch.uint8,
                                    device=x1.device)
            _keep_for_stream(stream, workspace)
        if stream is None:
            stream = torch.cuda.current_stream(x1.device)
        self._fn = lib().hyenand_fftconv_backward
        self._args = (_ptr(x1), _ptr(x2), _ptr(v), _ptr(k), _ptr(D), _ptr(gy), _ptr(gx1), _ptr(gx2), _ptr(gv),
                      _ptr(gk), _ptr(gD), nd, dims, _mode(pad_mode), _dtype_code(x1.dtype), _ptr(workspace),
                      workspace.numel() * workspace.element_size(), ctypes.c_void_p(stream.cuda_stream))
        self._keep = (gx1, gx2, gv, gk, gD, x1, x2, v, k, D, gy, workspace, stream)

    def __call__(self) -> None:
        status = self._fn(*self._args)
        if status != OK:
            _check(status)


def backward_into(gx1, gx2, gv, gk, gD, x1, x2, v, k, D, gy, pad_mode: str = "linear", workspace=None,
                  stream=None) -> None:
    """Gradients of a loss through y for dLoss/dy = gy, written into gx1, gx2,
    gv ([B, C, L...]), gk (shaped like k) and gD ([C]); all tensors already on
    the GPU."""
    PreparedBackward(gx1, gx2, gv, gk, gD, x1, x2, v, k, D, gy, pad_mode, workspace, stream)()


def backward(x1, x2, v, k, D, gy, pad_mode: str = "linear", workspace=None, stream=None):
    """(gx1, gx2, gv, gk, gD) with torch-allocated outputs."""
    import torch
    gx1, gx2, gv = (torch.empty_like(x1) for _ in range(3))
    gk = torch.empty_like(k)
    gD = torch.empty_like(D)
    backward_into(gx1, gx2, gv, gk, gD, x1, x2, v, k, D, gy, pad_mode, workspace, stream)
    _keep_for_stream(stream, gx1, gx2, gv, gk, gD)
    return gx1, gx2, gv, gk, gD


def operator_workspace_size(shape, pad_mode: str, dtype) -> int:
    nd, dims = _dims(shape)
    out = ctypes.c_size_t(0)
    _check(lib().hyenand_operator_workspace_size(nd, dims, _mode(pad_mode), _dtype_code(dtype), ctypes.byref(out)))
    return int(out.value)


class PreparedOperator:
    """One hyenand_operator call with its arguments checked and marshalled
    once (see Prepared)."""

    def __init__(self, y, q, kin, vin, k, D, w_in, w_out, eps_l2: float = 1e-6, eps_rms: float = 1e-6,
                 pad_mode: str = "linear", workspace=None, stream=None):
        import torch
        shape = tuple(q.shape)
        for t, want in ((q, shape), (kin, shape), (vin, shape), (y, shape),
                        (k, kernel_shape(shape, pad_mode))):
            if not t.is_cuda or tuple(t.shape) != want or t.dtype != q.dtype or not t.is_contiguous():
                raise ValueError("q, kin, vin, y must be contiguous GPU tensors of one shape and dtype; "
                                 f"k must be {kernel_shape(shape, pad_mode)}")
        for t in (D, w_in, w_out):
            if not t.is_cuda or t.dtype != q.dtype or tuple(t.shape) != (shape[1],) or not t.is_contiguous():
                raise ValueError("D, w_in and w_out must be contiguous [C] GPU tensors of the same dtype")
        if workspace is None:
            workspace = torch.empty(operator_workspace_size(shape, pad_mode, q.dtype), dtype=torch.uint8,
                                    device=q.device)
            _keep_for_stream(stream, workspace)
        nd, dims = _dims(shape)
        if stream is None:
            stream = torch.cuda.current_stream(q.device)
        self._fn = lib().hyenand_operator
        self._args = (_ptr(q), _ptr(kin), _ptr(vin), _ptr(k), _ptr(D), _ptr(w_in), _ptr(w_out), float(eps_l2),
                      float(eps_rms), _ptr(y), nd, dims, _mode(pad_mode), _dtype_code(q.dtype), _ptr(workspace),
                      workspace.numel() * workspace.element_size(), ctypes.c_void_p(stream.cuda_stream))
        self._keep = (y, q, kin, vin, k, D, w_in, w_out, workspace, stream)

    def __call__(self) -> None:
        status = self._fn(*self._args)
        if status != OK:
            _check(status)


def operator(q, kin, vin, k, D, w_in, w_out, eps_l2: float = 1e-6, eps_rms: float = 1e-6,
             pad_mode: str = "linear", workspace=None, stream=None):
    """The HyenaND operator, Eq. (HyenaND): RMSNorm(Sigmoid(vin) * (k conv
    RMSNorm(l2(q) * SiLU(kin)) + D * .)) with torch-allocated y."""
    import torch
    y = torch.empty_like(q)
    PreparedOperator(y, q, kin, vin, k, D, w_in, w_out, eps_l2, eps_rms, pad_mode, workspace, stream)()
    _keep_for_stream(stream, y)
    return y


WINDOWS = {"gaussian": 0, "exponential": 1}


class PreparedSynth:
    """One hyenand_kernel_synth call with its arguments checked and
    marshalled once (see Prepared).  k is [B, C, grid...] when gamma and beta
    are given, else [C, grid...]; the grid is kernel_shape(shape, pad_mode)'s."""

    def __init__(self, k, shape, omega0, W1, Wh, Wout, window, gamma=None, beta=None, bias=None,
                 window_kind: str = "gaussian", pad_mode: str = "linear", stream=None):
        import torch
        shape = tuple(int(x) for x in shape)
        nd = len(shape) - 2
        B, C = shape[:2]
        Hf = int(omega0.shape[0])
        J = 1 if Wh is None else int(Wh.shape[0]) + 1
        if window_kind not in WINDOWS:
            raise ValueError(f"window_kind must be one of {sorted(WINDOWS)}")
        want = [(omega0, (Hf,)), (W1, (nd, Hf)), (Wout, (Hf, C)),
                (window, (nd, C) if window_kind == "gaussian" else (C,))]
        if Wh is not None:
            want.append((Wh, (J - 1, Hf, Hf)))
        if bias is not None:
            want.append((bias, (J, Hf)))
        if (gamma is None) != (beta is None):
            raise ValueError("gamma and beta go together")
        if gamma is not None:
            want += [(gamma, (B, J, Hf)), (beta, (B, J, Hf))]
        for t, sh in want:
            if not t.is_cuda or t.dtype != torch.float32 or tuple(t.shape) != sh or not t.is_contiguous():
                raise ValueError(f"parameters must be contiguous fp32 GPU tensors; expected shape {sh}, "
                                 f"got {tuple(t.shape)}")
        kshape = kernel_shape(shape, pad_mode, shared_k=gamma is None)
        if not k.is_cuda or tuple(k.shape) != kshape or not k.is_contiguous():
            raise ValueError(f"k must be a contiguous GPU tensor of shape {kshape}")
        nd_, dims = _dims(shape)
        if stream is None:
            stream = torch.cuda.current_stream(k.device)
        opt = lambda t: None if t is None else _ptr(t)
        self._fn = lib().hyenand_kernel_synth
        self._args = (_ptr(omega0), _ptr(W1), opt(Wh), opt(bias), opt(gamma), opt(beta), _ptr(Wout), _ptr(window),
                      WINDOWS[window_kind], Hf, J, _ptr(k), nd_, dims, _mode(pad_mode), _dtype_code(k.dtype),
                      ctypes.c_void_p(stream.cuda_stream))
        self._keep = (k, omega0, W1, Wh, Wout, window, gamma, beta, bias, stream)

    def __call__(self) -> None:
        status = self._fn(*self._args)
        if status != OK:
            _check(status)


def kernel_synth(shape, omega0, W1, Wh, Wout, window, gamma=None, beta=None, bias=None,
                 window_kind: str = "gaussian", pad_mode: str = "linear", dtype=None, stream=None):
    """The HyenaND kernel K(x) for a convolution on tensors of `shape`
    ([B, C, L...]), with a torch-allocated k of `dtype` (fp32 by default)."""
    import torch
    dtype = dtype or torch.float32
    kshape = kernel_shape(shape, pad_mode, shared_k=gamma is None)
    k = torch.empty(kshape, dtype=dtype, device=omega0.device)
    PreparedSynth(k, shape, omega0, W1, Wh, Wout, window, gamma, beta, bias, window_kind, pad_mode, stream)()
    _keep_for_stream(stream, k)
    return k


class PreparedModal:
    """One hyenand_modal_filter call with its arguments checked and marshalled
    once (see Prepared): k [C, L] from the [C, M] poles and residues."""

    def __init__(self, k, log_mag, angle, res_re, res_im, stream=None):
        import torch
        C, M = (int(x) for x in log_mag.shape)
        for t in (log_mag, angle, res_re, res_im):
            if not t.is_cuda or t.dtype != torch.float32 or tuple(t.shape) != (C, M) or not t.is_contiguous():
                raise ValueError("log_mag, angle, res_re, res_im must be contiguous fp32 GPU tensors of one [C, M] shape")
        if not k.is_cuda or k.dim() != 2 or k.shape[0] != C or not k.is_contiguous():
            raise ValueError("k must be a contiguous [C, L] GPU tensor")
        if stream is None:
            stream = torch.cuda.current_stream(k.device)
        self._fn = lib().hyenand_modal_filter
        self._args = (_ptr(log_mag), _ptr(angle), _ptr(res_re), _ptr(res_im), M, _ptr(k), C, int(k.shape[1]),
                      _dtype_code(k.dtype), ctypes.c_void_p(stream.cuda_stream))
        self._keep = (k, log_mag, angle, res_re, res_im, stream)

    def __call__(self) -> None:
        status = self._fn(*self._args)
        if status != OK:
            _check(status)


def modal_filter(log_mag, angle, res_re, res_im, L: int, dtype=None, stream=None):
    """k [C, L] = Re sum_m R lambda^t (the modal long filter) with a
    torch-allocated k of `dtype` (fp32 by default)."""
    import torch
    k = torch.empty((log_mag.shape[0], int(L)), dtype=dtype or torch.float32, device=log_mag.device)
    PreparedModal(k, log_mag, angle, res_re, res_im, stream)()
    _keep_for_stream(stream, k)
    return k


SCAN_BLOCK = 512  # HYENAND_SCAN_BLOCK: positions between two states that the forward keeps for the backward


def _expect(like, shape, dtype, **tensors) -> None:
    """Every given tensor is contiguous, of this shape and dtype, on `like`'s device."""
    device = like.get_device()
    for t in tensors.values():
        if t is None or (t.shape == shape and t.dtype is dtype and t.is_contiguous() and t.get_device() == device):
            continue
        name = next(n for n, u in tensors.items() if u is t)
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of shape {shape} on {like.device}, got "
                         f"{t.dtype} {tuple(t.shape)} on {t.device}" + ("" if t.is_contiguous() else ", not contiguous"))


def _gpu_dtype(t) -> int:
    if not t.is_cuda:
        raise ValueError("all tensors must be on the GPU")
    return _dtype_code(t.dtype)


def _pointers(*tensors):
    return tuple([None if t is None else t.data_ptr() for t in tensors])


class _Call:
    """A marshalled call: enqueues its work again each time it is called, on
    the same buffers and stream, which it keeps alive."""

    def _prepare(self, fn, args, like, stream, keep) -> None:
        import torch
        self._device = like.get_device()
        if stream is None:
            handle = torch._C._cuda_getCurrentRawStream(self._device)  # current_stream() without its object
        else:
            handle = stream.cuda_stream
        self._fn = fn
        self._args = args + (handle,)
        self._current = torch._C._cuda_getDevice  # torch.cuda.current_device() once CUDA is initialised
        self._keep = (keep, stream)

    def __call__(self) -> None:
        if self._device == self._current():
            status = self._fn(*self._args)
        else:  # launches go to the current device's streams
            import torch
            with torch.cuda.device(self._device):
                status = self._fn(*self._args)
        if status != OK:
            _check(status)


def _scratch(nbytes: int, workspace, device, stream):
    """The caller's workspace, or one of nbytes for this call (None if it takes none)."""
    import torch
    if workspace is not None:
        if workspace.device != device or not workspace.is_contiguous():
            raise ValueError(f"workspace must be a contiguous tensor on {device}")
    elif nbytes:
        workspace = torch.empty(nbytes, dtype=torch.uint8, device=device)
        _keep_for_stream(stream, workspace)
    if workspace is None:
        return None, None, 0
    return workspace, workspace.data_ptr(), workspace.numel() * workspace.element_size()


@functools.lru_cache(maxsize=1024)
def _query(name: str, shape, code: int) -> int:
    out = ctypes.c_size_t(0)
    _check(getattr(lib(), name)(*[int(n) for n in shape], code, ctypes.byref(out)))
    return int(out.value)


def scan_workspace_size(shape, dtype) -> int:
    """Workspace bytes of hyenand_scan on [B, C, L] tensors."""
    return _query("hyenand_scan_workspace_size", tuple(shape), _dtype_code(dtype))


def scan_backward_workspace_size(shape, dtype) -> int:
    return _query("hyenand_scan_backward_workspace_size", tuple(shape), _dtype_code(dtype))


def scan_states_shape(shape):
    """Shape of the states that hyenand_scan keeps for its backward: one before every SCAN_BLOCK-th position."""
    B, C, L = (int(n) for n in shape)
    return B, C, -(-L // SCAN_BLOCK)


def _scan_inputs(x1, D, lengths, gD=None, **like_x1):
    import torch
    if x1.dim() != 3:
        raise ValueError(f"x1 must be [B, C, L], got {tuple(x1.shape)}")
    code, shape = _gpu_dtype(x1), tuple(x1.shape)
    _expect(x1, shape, x1.dtype, x1=x1, **like_x1)
    _expect(x1, shape[1:2], x1.dtype, D=D, gD=gD)
    if lengths is not None:
        _expect(x1, shape[:1], torch.int64, lengths=lengths)
    return code, shape


class PreparedScan(_Call):
    """One hyenand_scan call with its arguments checked and marshalled once
    (see Prepared).  h0, lengths, h_last and states may be None; h_last may be
    h0, which then holds the state behind the last position."""

    def __init__(self, y, x1, x2, v, log_a, D, h0=None, lengths=None, h_last=None, states=None, workspace=None,
                 stream=None):
        import torch
        code, shape = _scan_inputs(x1, D, lengths, x2=x2, v=v, log_a=log_a, y=y)
        _expect(x1, shape[:2], torch.float32, h0=h0, h_last=h_last)
        _expect(x1, scan_states_shape(shape), torch.float32, states=states)
        ws, ws_ptr, ws_bytes = _scratch(scan_workspace_size(shape, x1.dtype), workspace, x1.device, stream)
        self._prepare(lib().hyenand_scan,
                      _pointers(x1, x2, v, log_a, D, h0, lengths, y, h_last, states) + shape + (code, ws_ptr, ws_bytes),
                      x1, stream,
                      (y, x1, x2, v, log_a, D, h0, lengths, h_last, states, ws))


def scan(x1, x2, v, log_a, D, h0=None, lengths=None, return_last: bool = False, return_states: bool = False,
         workspace=None, stream=None):
    """y = x2 * (h + D*u), u = x1*v, h_t = exp(log_a_t) h_{t-1} + u_t on [B, C, L]
    tensors.  Returns (y, h_last, states), torch-allocated: h_last [B, C] and
    the states that scan_backward takes where they are asked for, else None."""
    import torch
    y = torch.empty_like(x1)
    last = torch.empty(tuple(x1.shape[:2]), dtype=torch.float32, device=x1.device) if return_last else None
    states = torch.empty(scan_states_shape(x1.shape), dtype=torch.float32, device=x1.device) if return_states else None
    PreparedScan(y, x1, x2, v, log_a, D, h0, lengths, last, states, workspace, stream)()
    _keep_for_stream(stream, y, last, states)
    return y, last, states


class PreparedScanBackward(_Call):
    """One hyenand_scan_backward call with its arguments checked and
    marshalled once (see Prepared); lengths, gh_last and gh0 may be None."""

    def __init__(self, gx1, gx2, gv, glog_a, gD, gh0, x1, x2, v, log_a, D, states, gy, lengths=None, gh_last=None,
                 workspace=None, stream=None):
        import torch
        code, shape = _scan_inputs(x1, D, lengths, gD, x2=x2, v=v, log_a=log_a, gy=gy, gx1=gx1, gx2=gx2, gv=gv,
                                   glog_a=glog_a)
        _expect(x1, shape[:2], torch.float32, gh_last=gh_last, gh0=gh0)
        _expect(x1, scan_states_shape(shape), torch.float32, states=states)
        ws, ws_ptr, ws_bytes = _scratch(scan_backward_workspace_size(shape, x1.dtype), workspace, x1.device, stream)
        self._prepare(lib().hyenand_scan_backward,
                      _pointers(x1, x2, v, log_a, D, lengths, states, gy, gh_last, gx1, gx2, gv, glog_a, gD, gh0)
                      + shape + (code, ws_ptr, ws_bytes), x1, stream,
                      (gx1, gx2, gv, glog_a, gD, gh0, x1, x2, v, log_a, D, states, gy, lengths, gh_last, ws))


def scan_backward(x1, x2, v, log_a, D, states, gy, lengths=None, gh_last=None, return_gh0: bool = False,
                  workspace=None, stream=None):
    """(gx1, gx2, gv, glog_a, gD), and gh0 with return_gh0, for gy = dLoss/dy
    (and gh_last = dLoss/dh_last), from the states that scan returned."""
    import torch
    gx1, gx2, gv, gla = (torch.empty_like(x1) for _ in range(4))
    gD = torch.empty_like(D)
    gh0 = torch.empty(tuple(x1.shape[:2]), dtype=torch.float32, device=x1.device) if return_gh0 else None
    PreparedScanBackward(gx1, gx2, gv, gla, gD, gh0, x1, x2, v, log_a, D, states, gy, lengths, gh_last, workspace,
                         stream)()
    _keep_for_stream(stream, gx1, gx2, gv, gla, gD, gh0)
    return (gx1, gx2, gv, gla, gD) + ((gh0,) if return_gh0 else ())


class PreparedScanStep(_Call):
    """One hyenand_scan_step call with its arguments checked and marshalled
    once (see Prepared): y and x1, x2, v, log_a are [B, C], state [slots, C]."""

    def __init__(self, y, x1, x2, v, log_a, D, state, slots=None, stream=None):
        import torch
        if x1.dim() != 2 or state.dim() != 2:
            raise ValueError("x1 must be [B, C] and state [num_slots, C]")
        code, shape = _gpu_dtype(x1), tuple(x1.shape)
        _expect(x1, shape, x1.dtype, x1=x1, x2=x2, v=v, log_a=log_a, y=y)
        _expect(x1, shape[1:], x1.dtype, D=D)
        _expect(x1, (state.shape[0], shape[1]), torch.float32, state=state)
        _expect(x1, shape[:1], torch.int64, slots=slots)
        self._prepare(lib().hyenand_scan_step,
                      _pointers(x1, x2, v, log_a, D, slots, state, y) + shape + (int(state.shape[0]), code), x1, stream, (y, x1, x2, v, log_a, D, state, slots))


def scan_step(x1, x2, v, log_a, D, state, slots=None, stream=None):
    """One position of scan for every row of [B, C] tensors: the rows' states
    (state[slots[b]], or state[b]) are updated in place; returns y."""
    import torch
    y = torch.empty_like(x1)
    PreparedScanStep(y, x1, x2, v, log_a, D, state, slots, stream)()
    _keep_for_stream(stream, y)
    return y


def _points(shape):
    """(B, C, P) of a [B, C, grid...] tensor."""
    if len(shape) < 2:
        raise ValueError(f"tensors must be [B, C, grid...], got {shape}")
    return shape[0], shape[1], math.prod(shape[2:])


def block_norm_backward_workspace_size(shape, dtype) -> int:
    """Workspace bytes of hyenand_block_norm_backward on [B, C, P] tensors."""
    return _query("hyenand_block_norm_backward_workspace_size", tuple(shape), _dtype_code(dtype))


def _norm_inputs(x, rng, like_x, like_w):
    import torch
    code, shape = _gpu_dtype(x), tuple(x.shape)
    BCP = _points(shape)
    _expect(x, shape, x.dtype, **like_x)
    _expect(x, shape[1:2], x.dtype, **like_w)
    if rng is not None:
        _expect(x, (2,), torch.int64, rng=rng)
    return code, BCP


class PreparedBlockNorm(_Call):
    """One hyenand_block_norm call with its arguments checked and marshalled
    once (see Prepared): x_out and n from x, and of z, gate, w_post, scale,
    w_pre, x_out, n and rng what the call has; the others are None."""

    def __init__(self, x_out, n, x, z=None, gate=None, w_post=None, scale=None, w_pre=None, eps_post: float = 1e-6,
                 eps_pre: float = 1e-6, dropout_p: float = 0.0, rng=None, stream=None):
        code, BCP = _norm_inputs(x, rng, dict(x=x, z=z, gate=gate, x_out=x_out, n=n),
                                 dict(w_post=w_post, scale=scale, w_pre=w_pre))
        self._prepare(lib().hyenand_block_norm,
                      _pointers(x, z, gate, w_post, scale, w_pre) + (eps_post, eps_pre, dropout_p)
                      + _pointers(rng, x_out, n) + BCP + (code,), x, stream, (x_out, n, x, z, gate, w_post, scale, w_pre, rng))


def block_norm(x, z=None, gate=None, w_post=None, scale=None, w_pre=None, eps_post: float = 1e-6, eps_pre: float = 1e-6,
               dropout_p: float = 0.0, rng=None, stream=None):
    """(x_out, n) = (x + scale * drop(RMSNorm(sigmoid(gate) * z) w_post), RMSNorm(x_out) w_pre) on [B, C, grid...]
    tensors, the norms across the channels, torch-allocated.  Without z: (x, RMSNorm(x) w_pre); without w_pre:
    (x_out, None).  rng: an int64 GPU tensor (seed, offset), which fixes what dropout drops."""
    import torch
    x_out = None if z is None else torch.empty_like(x)
    n = None if w_pre is None else torch.empty_like(x)
    PreparedBlockNorm(x_out, n, x, z, gate, w_post, scale, w_pre, eps_post, eps_pre, dropout_p, rng, stream)()
    _keep_for_stream(stream, x_out, n)
    return x if z is None else x_out, n


class PreparedBlockNormBackward(_Call):
    """One hyenand_block_norm_backward call with its arguments checked and
    marshalled once (see Prepared); each gradient but gx is None where its
    input is (gw_pre, and w_pre, where gn is)."""

    def __init__(self, gx, gz, ggate, gw_post, gscale, gw_pre, x_out, z, gate, w_post, scale, w_pre, gx_out, gn,
                 eps_post: float = 1e-6, eps_pre: float = 1e-6, dropout_p: float = 0.0, rng=None, workspace=None,
                 stream=None):
        code, BCP = _norm_inputs(x_out, rng, dict(x_out=x_out, z=z, gate=gate, gx_out=gx_out, gn=gn, gx=gx, gz=gz, ggate=ggate),
                                 dict(w_post=w_post, scale=scale, w_pre=w_pre, gw_post=gw_post, gscale=gscale, gw_pre=gw_pre))
        ws, ws_ptr, ws_bytes = _scratch(block_norm_backward_workspace_size(BCP, x_out.dtype), workspace, x_out.device,
                                        stream)
        self._prepare(lib().hyenand_block_norm_backward,
                      _pointers(x_out, z, gate, w_post, scale, w_pre) + (eps_post, eps_pre, dropout_p)
                      + _pointers(rng, gx_out, gn, gx, gz, ggate, gw_post, gscale, gw_pre) + BCP + (code, ws_ptr, ws_bytes), x_out, stream,
                      (gx, gz, ggate, gw_post, gscale, gw_pre, x_out, z, gate, w_post, scale, w_pre, gx_out, gn, rng, ws))


def block_norm_backward(x_out, z, gate, w_post, scale, w_pre, gx_out, gn, eps_post: float = 1e-6, eps_pre: float = 1e-6,
                        dropout_p: float = 0.0, rng=None, workspace=None, stream=None):
    """(gx, gz, ggate, gw_post, gscale, gw_pre) of block_norm, from its x_out (x where it had no z) and the gradients
    of x_out and n (either may be None), torch-allocated; None for those of inputs that are None."""
    import torch
    if gn is None:
        w_pre = None
    like = lambda t: None if t is None else torch.empty_like(t)  # noqa: E731
    g = (torch.empty_like(x_out),) + tuple(like(t) for t in (z, gate, w_post, scale, w_pre))
    PreparedBlockNormBackward(*g, x_out, z, gate, w_post, scale, w_pre, gx_out, gn, eps_post, eps_pre, dropout_p, rng,
                              workspace, stream)()
    _keep_for_stream(stream, *g)
    return g
