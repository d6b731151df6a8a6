"""Thin Python binding of libams.so, the MI355X AMS-Quant weight-only quantized Linear.

Argument marshalling only (of the Linear's eager calls in native code, csrc/ams_binding.cpp): every step of the path
(quantize, pack, restore, multiply) runs inside the C-ABI library declared in include/ams.h.  PyTorch is used for device
memory and streams.  If the library has not been built (``python __graft_entry__.py``) every call raises; without the
native binding, which needs torch's headers, the same calls go through ctypes.
"""

from __future__ import annotations

import ctypes
import functools
import importlib.machinery
import os
import sys
import warnings

import numpy as np

FP533 = 0  # AMS_FMT_FP533_E2M3
FP425 = 1  # AMS_FMT_FP425_E2M2
FP45 = 2  # AMS_FMT_FP45_E2M2
FP433 = 3  # AMS_FMT_FP433_E2M2
FP6 = 4  # AMS_FMT_FP6_E2M3
FP5 = 5  # AMS_FMT_FP5_E2M2
FP4 = 6  # AMS_FMT_FP4_E2M1
SEARCH_SET_BIT = 0  # AMS_SEARCH_SET_BIT
SEARCH_REROUND = 1  # AMS_SEARCH_REROUND
MAX_M = 32
KV_WORKSPACE_BYTES = 64 << 20  # AMS_KV_WORKSPACE_BYTES

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libams.so")
_lib = None

_i64, _int, _vp = ctypes.c_int64, ctypes.c_int, ctypes.c_void_p


class AmsError(RuntimeError):
    pass


class _KvCache(ctypes.Structure):
    """ams_kv_cache of include/ams.h."""

    _fields_ = [
        ("pages", _vp), ("block_table", _vp), ("kv_lens", _vp), ("q_starts", _vp), ("n_pages", _i64), ("table_stride", _i64),
        *((name, ctypes.c_int32) for name in ("table_width", "batch", "kv_heads", "head_dim", "page_size", "scale_group")),
    ]


def load_library():
    """Load libams.so (once) and declare the signatures of include/ams.h."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise AmsError(f"{_LIB_PATH} is missing: build it with `python __graft_entry__.py`")
    lib = ctypes.CDLL(_LIB_PATH)
    lib.ams_version.restype = _int
    lib.ams_init.restype = _int
    lib.ams_strerror.restype = ctypes.c_char_p
    lib.ams_strerror.argtypes = [_int]
    lib.ams_group_size.argtypes = [_int]
    lib.ams_code_bits.argtypes = [_int]
    lib.ams_packed_bytes.argtypes = [_int, _i64, _i64, ctypes.POINTER(ctypes.c_size_t)]
    lib.ams_canonical_bytes.argtypes = [_int, _i64, _i64, ctypes.POINTER(ctypes.c_size_t)]
    lib.ams_pack.argtypes = [_int, _vp, _i64, _i64, _i64, _vp, _vp, _vp]
    lib.ams_pack_ex.argtypes = [_int, _int, _vp, _i64, _i64, _i64, _vp, _vp, _vp]
    lib.ams_group_scales_count.argtypes = [_int, _i64, _i64, _i64, ctypes.POINTER(ctypes.c_size_t)]
    lib.ams_pack_grouped.argtypes = [_int, _int, _i64, _vp, _i64, _i64, _i64, _vp, _vp, _vp]
    lib.ams_dequant_grouped.argtypes = [_int, _vp, _vp, _i64, _vp, _i64, _i64, _int, _vp]
    lib.ams_linear_grouped.argtypes = [_vp, _vp, _i64, _vp, _vp, _int, _i64, _i64, _int, _vp]
    lib.ams_pack_per_tensor.argtypes = [_int, _int, _vp, _i64, _i64, _i64, _vp, _vp, _vp]
    lib.ams_pack_codes.argtypes = [_int, _vp, _i64, _i64, _vp]
    lib.ams_unpack_host.argtypes = [_int, _vp, _i64, _i64, _vp]
    lib.ams_dequant.argtypes = [_int, _vp, _vp, _vp, _i64, _i64, _int, _vp]
    lib.ams_linear.argtypes = [_vp, _vp, _vp, _vp, _int, _i64, _i64, _int, _vp]
    lib.ams_fp16_linear.argtypes = [_vp, _vp, _vp, _int, _i64, _i64, _vp]
    lib.ams_linear_workspace_bytes.argtypes = [_int, _int, _i64, _i64, ctypes.POINTER(ctypes.c_size_t)]
    lib.ams_linear_static_ws.argtypes = [_vp, _vp, _vp, _vp, _int, _i64, _i64, _int, _vp]
    lib.ams_linear_ws.argtypes = [_vp, _vp, _vp, _vp, _int, _i64, _i64, _int, _vp, ctypes.c_size_t, _vp]
    lib.ams_fp16_linear_ws.argtypes = [_vp, _vp, _vp, _int, _i64, _i64, _vp, ctypes.c_size_t, _vp]
    lib.ams_linear_plan.argtypes = [_int, _int, _i64, _i64, _int, ctypes.c_char_p, ctypes.c_size_t]
    lib.ams_kv_block_bytes.argtypes = [_int, _int, _int, ctypes.POINTER(ctypes.c_size_t)]
    lib.ams_kv_write.argtypes = lib.ams_kv_read.argtypes = [ctypes.POINTER(_KvCache), _vp, _vp, *[_i64] * 5, _vp]
    lib.ams_kv_attention_workspace_bytes.argtypes = [ctypes.POINTER(_KvCache), _i64, _int, _i64, ctypes.POINTER(ctypes.c_size_t)]
    lib.ams_kv_attention_plan.argtypes = [ctypes.POINTER(_KvCache), _i64, _int, _i64, _i64, ctypes.c_size_t, ctypes.c_char_p, ctypes.c_size_t]
    lib.ams_kv_attention.argtypes = [ctypes.POINTER(_KvCache), _vp, _vp, _vp, _i64, _int, *[_i64] * 5, ctypes.c_float, _int, _i64, _i64, _vp, ctypes.c_size_t, _vp]
    lib.ams_read_probe.argtypes = [_vp, ctypes.c_size_t, _vp, _vp]
    _lib = lib
    return lib


def _check(rc: int, what: str):
    if rc != 0:
        raise AmsError(f"{what}: {load_library().ams_strerror(rc).decode()} ({rc})")


def _np_ptr(a: np.ndarray):
    return a.ctypes.data_as(_vp)


def ams_version() -> int:
    return load_library().ams_version()


def ams_init() -> None:
    """Check the current device and raise the kernels' LDS limits (needed only before a first call under stream capture)."""
    _check(load_library().ams_init(), "ams_init")
    if "torch" in sys.modules and _call is _first_call:
        _bind_call()


def _packed_bytes(fmt, N, K):
    out = ctypes.c_size_t()
    _check(load_library().ams_packed_bytes(fmt, N, K, ctypes.byref(out)), "ams_packed_bytes")
    return out.value


_packed_bytes_of_ints = functools.lru_cache(maxsize=4096)(_packed_bytes)


def ams_packed_bytes(fmt: int, N: int, K: int) -> int:
    # a pure function of its arguments, asked on every call of the Linear; only plain ints may share an answer (16.0 equals
    # 16 but is refused by ctypes, and a ctypes integer can change its value)
    if type(fmt) is int and type(N) is int and type(K) is int:
        return _packed_bytes_of_ints(fmt, N, K)
    return _packed_bytes(fmt, N, K)


def ams_canonical_bytes(fmt: int, N: int, K: int) -> int:
    out = ctypes.c_size_t()
    _check(load_library().ams_canonical_bytes(fmt, N, K, ctypes.byref(out)), "ams_canonical_bytes")
    return out.value


def ams_pack_ex(fmt: int, search: int, W: np.ndarray, return_codes: bool = False):
    """Quantize + pack host fp16 weights [N,K] with the given search.  Returns (packed uint8, scales float16[, codes uint8])."""
    if W.dtype != np.float16 or W.ndim != 2:
        raise TypeError("W must be a 2-D float16 array")
    W = np.ascontiguousarray(W)
    N, K = W.shape
    packed = np.empty(ams_packed_bytes(fmt, N, K), dtype=np.uint8)
    scales = np.empty(N, dtype=np.float16)
    codes = np.empty((N, K), dtype=np.uint8) if return_codes else None
    rc = load_library().ams_pack_ex(fmt, search, _np_ptr(W), N, K, K, _np_ptr(packed), _np_ptr(scales), _np_ptr(codes) if return_codes else None)
    _check(rc, "ams_pack_ex")
    return (packed, scales, codes) if return_codes else (packed, scales)


def ams_pack(fmt: int, W: np.ndarray, return_codes: bool = False):
    """Quantize + pack host fp16 weights [N,K].  Returns (packed uint8, scales float16[, codes uint8])."""
    if W.dtype != np.float16 or W.ndim != 2:
        raise TypeError("W must be a 2-D float16 array")
    W = np.ascontiguousarray(W)
    N, K = W.shape
    packed = np.empty(ams_packed_bytes(fmt, N, K), dtype=np.uint8)
    scales = np.empty(N, dtype=np.float16)
    codes = np.empty((N, K), dtype=np.uint8) if return_codes else None
    rc = load_library().ams_pack(fmt, _np_ptr(W), N, K, K, _np_ptr(packed), _np_ptr(scales), _np_ptr(codes) if return_codes else None)
    _check(rc, "ams_pack")
    return (packed, scales, codes) if return_codes else (packed, scales)


def ams_pack_codes(fmt: int, codes: np.ndarray) -> np.ndarray:
    codes = np.ascontiguousarray(codes, dtype=np.uint8)
    N, K = codes.shape
    packed = np.empty(ams_packed_bytes(fmt, N, K), dtype=np.uint8)
    _check(load_library().ams_pack_codes(fmt, _np_ptr(codes), N, K, _np_ptr(packed)), "ams_pack_codes")
    return packed


def ams_unpack_host(fmt: int, packed: np.ndarray, N: int, K: int) -> np.ndarray:
    packed = np.ascontiguousarray(packed, dtype=np.uint8)
    if packed.size != ams_packed_bytes(fmt, N, K):
        raise ValueError("packed buffer has the wrong size")
    codes = np.empty((N, K), dtype=np.uint8)
    _check(load_library().ams_unpack_host(fmt, _np_ptr(packed), N, K, _np_ptr(codes)), "ams_unpack_host")
    return codes


_current_stream = None


def _bind_current_stream():
    import torch

    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)  # not a public name: a torch without it goes the long way
    if raw is None:
        return lambda: torch.cuda.current_stream().cuda_stream
    device = torch.cuda.current_device
    return lambda: raw(device())


def _stream():
    """The current stream of the current device.  Read as the raw handle: building torch's Stream object
    took 2.8 us of the 8.4 us that a whole call of ams_linear took, the handle takes 0.3."""
    global _current_stream
    if _current_stream is None:
        _current_stream = _bind_current_stream()
    return _current_stream()


def _first_call(*args):
    """One of the calls of the Linear below in native code (csrc/ams_binding.cpp): the same checks, stream and library.  None, and nothing
    done, for arguments that are not plain tensors and ints or that something is wrong with: those go the long way, which raises.
    A whole call of ams_linear(..., out=...) takes 3.1 us with it and 5.3 without; calls that allocate their output don't ask it.
    This one stands in until ams_init or the first call."""
    _bind_call()
    return _call(*args)


_call = _first_call


def _first_kv_call(*args):
    """The same for the calls of the KV cache: (entry, cache, block_table, kv_lens, scale_group, q_starts, ...)."""
    _bind_call()
    return _kv_call(*args)


_kv_call = _first_kv_call
_KV_WRITE, _KV_READ, _KV_ATTENTION = range(3)  # of csrc/ams_binding.cpp


def _bind_call():
    global _call, _kv_call
    _call = _kv_call = lambda *args: None  # the long way
    try:
        import torch  # its libraries first
    except ImportError:
        return
    here = f"{torch.__version__} {torch.version.git_version}"
    if not any(os.path.exists(os.path.join(os.path.dirname(_LIB_PATH), "_binding" + s)) for s in importlib.machinery.EXTENSION_SUFFIXES):
        return  # a package without it, or with another Python's, is whole
    try:
        from . import _binding

        if getattr(_binding, "BUILT_FOR", None) != here:  # it reads tensors as that torch lays them out
            raise ImportError(f"{_binding.__file__} was not built for torch {here}")
    except ImportError as e:
        warnings.warn(f"calls of the Linear are slower than they need be: {e} (build again with `python __graft_entry__.py`)", RuntimeWarning, stacklevel=3)
        return
    lib = load_library()
    _binding.bind(*(ctypes.cast(f, _vp).value for f in (lib.ams_packed_bytes, lib.ams_group_scales_count, lib.ams_linear, lib.ams_linear_ws, lib.ams_linear_static_ws, lib.ams_linear_grouped)))
    _binding.bind_kv(*(ctypes.cast(f, _vp).value for f in (lib.ams_kv_block_bytes, lib.ams_kv_write, lib.ams_kv_read, lib.ams_kv_attention)))
    _call, _kv_call = _binding.linear, _binding.kv


_PLAIN, _WORKSPACE, _STATIC, _GROUPED = range(4)  # of csrc/ams_binding.cpp


_devices = 0  # of this machine, once asked: with one of them no tensor is on another


def _check_device(t):
    # the kernels run on the current device and in the order of its stream
    global _devices
    import torch

    _devices = torch.cuda.device_count()
    if t.get_device() != torch.cuda.current_device():
        raise ValueError(f"expected a tensor on the current device, cuda:{torch.cuda.current_device()}, got one on cuda:{t.get_device()}")


def _dev_ptr(t, dtype=None):
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError("expected a contiguous CUDA tensor")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"expected {dtype}, got {t.dtype}")
    if _devices != 1:
        _check_device(t)
    return t.data_ptr()


def _too_small(out, rows, columns):
    # the kernels write that many values (a buffer for a larger batch may be given)
    return ValueError(f"out must hold {rows} x {columns} values, it has {out.numel()}")


def ams_dequant(fmt: int, W_packed, scales, N: int, K: int, scaled: bool = True, out=None):
    """Restore a packed matrix (uint8 CUDA tensor) to fp16 [N,K] on the GPU."""
    import torch

    if W_packed.numel() != ams_packed_bytes(fmt, N, K):
        raise ValueError("packed buffer has the wrong size")
    if out is None:
        out = torch.empty((N, K), dtype=torch.float16, device=W_packed.device)
    elif out.numel() < N * K:
        raise _too_small(out, N, K)
    sp = _dev_ptr(scales, torch.float16) if scales is not None else None
    if scales is not None and scales.numel() != N:
        raise ValueError("scales must have N entries")
    rc = load_library().ams_dequant(fmt, _dev_ptr(W_packed, torch.uint8), sp, _dev_ptr(out, torch.float16), N, K, int(scaled), _stream())
    _check(rc, "ams_dequant")
    return out


def ams_linear(W_packed, scales, X, N: int, fmt: int, out=None):
    """Y = X @ DeQ(W)^T on the GPU.  X fp16 [M,K] CUDA tensor; returns fp16 [M,N]."""
    if out is not None and _call(_PLAIN, W_packed, scales, X, N, fmt, out, None) is not None:
        return out
    import torch

    M, K = X.shape
    if W_packed.numel() != ams_packed_bytes(fmt, N, K):
        raise ValueError("packed buffer has the wrong size")
    if scales.numel() != N:
        raise ValueError("scales must have N entries")
    if out is None:
        out = torch.empty((M, N), dtype=torch.float16, device=X.device)
    elif out.numel() < M * N:
        raise _too_small(out, M, N)
    rc = load_library().ams_linear(
        _dev_ptr(W_packed, torch.uint8), _dev_ptr(scales, torch.float16), _dev_ptr(X, torch.float16), _dev_ptr(out, torch.float16), M, N, K, fmt, _stream()
    )
    _check(rc, "ams_linear")
    return out


def ams_fp16_linear(W, X, out=None):
    """The fp16 baseline Y = X @ W^T on the GPU.  W fp16 [N,K], X fp16 [M,K]."""
    import torch

    N, K = W.shape
    M = X.shape[0]
    if X.shape[1] != K:
        raise ValueError("X and W disagree in K")
    if out is None:
        out = torch.empty((M, N), dtype=torch.float16, device=X.device)
    elif out.numel() < M * N:
        raise _too_small(out, M, N)
    rc = load_library().ams_fp16_linear(_dev_ptr(W, torch.float16), _dev_ptr(X, torch.float16), _dev_ptr(out, torch.float16), M, N, K, _stream())
    _check(rc, "ams_fp16_linear")
    return out


def ams_read_probe(buf, nbytes: int = None):
    """Measurement aid: a bare streaming read of the first nbytes of a CUDA tensor (default: all of it)."""
    if nbytes is None:
        nbytes = buf.numel() * buf.element_size()
    if nbytes > buf.numel() * buf.element_size():
        raise ValueError("nbytes exceeds the buffer")
    _check(load_library().ams_read_probe(_dev_ptr(buf), nbytes, None, _stream()), "ams_read_probe")


def ams_group_scales_count(fmt: int, N: int, K: int, scale_group: int) -> int:
    out = ctypes.c_size_t(0)
    _check(load_library().ams_group_scales_count(fmt, N, K, scale_group, ctypes.byref(out)), "ams_group_scales_count")
    return out.value


def ams_pack_grouped(fmt: int, W: np.ndarray, scale_group: int, search: int = SEARCH_SET_BIT, return_codes: bool = False):
    """Quantize + pack with one scale per run of scale_group input channels.  The scales come back in the
    order the kernels read them: [strip of 16 rows, run, row inside the strip]."""
    if W.dtype != np.float16 or W.ndim != 2:
        raise TypeError("W must be a 2-D float16 array")
    W = np.ascontiguousarray(W)
    N, K = W.shape
    packed = np.empty(ams_packed_bytes(fmt, N, K), dtype=np.uint8)
    n_sg = -(-K // scale_group)
    scales = np.empty(ams_group_scales_count(fmt, N, K, scale_group), dtype=np.float16).reshape(-1, n_sg, 16)
    codes = np.empty((N, K), dtype=np.uint8) if return_codes else None
    rc = load_library().ams_pack_grouped(fmt, search, scale_group, _np_ptr(W), N, K, K, _np_ptr(packed), _np_ptr(scales), _np_ptr(codes) if return_codes else None)
    _check(rc, "ams_pack_grouped")
    return (packed, scales, codes) if return_codes else (packed, scales)


def ams_dequant_grouped(fmt: int, W_packed, scales, scale_group: int, N: int, K: int, scaled: bool = True, out=None):
    import torch

    if W_packed.numel() != ams_packed_bytes(fmt, N, K):
        raise ValueError("packed buffer has the wrong size")
    if scales.numel() != ams_group_scales_count(fmt, N, K, scale_group):
        raise ValueError("scale buffer has the wrong size")
    if out is None:
        out = torch.empty((N, K), dtype=torch.float16, device=W_packed.device)
    elif out.numel() < N * K:
        raise _too_small(out, N, K)
    rc = load_library().ams_dequant_grouped(fmt, _dev_ptr(W_packed, torch.uint8), _dev_ptr(scales, torch.float16), scale_group, _dev_ptr(out, torch.float16), N, K, int(scaled), _stream())
    _check(rc, "ams_dequant_grouped")
    return out


def ams_linear_grouped(W_packed, scales, scale_group: int, X, N: int, fmt: int, out=None):
    if out is not None and _call(_GROUPED, W_packed, scales, X, N, fmt, out, scale_group) is not None:
        return out
    import torch

    M, K = X.shape
    if W_packed.numel() != ams_packed_bytes(fmt, N, K):
        raise ValueError("packed buffer has the wrong size")
    if scales.numel() != ams_group_scales_count(fmt, N, K, scale_group):
        raise ValueError("scale buffer has the wrong size")
    if out is None:
        out = torch.empty((M, N), dtype=torch.float16, device=X.device)
    elif out.numel() < M * N:
        raise _too_small(out, M, N)
    rc = load_library().ams_linear_grouped(
        _dev_ptr(W_packed, torch.uint8), _dev_ptr(scales, torch.float16), scale_group, _dev_ptr(X, torch.float16), _dev_ptr(out, torch.float16), M, N, K, fmt, _stream()
    )
    _check(rc, "ams_linear_grouped")
    return out


def ams_linear_workspace_bytes(fmt: int, M: int, N: int, K: int) -> int:
    """Bytes of workspace ams_linear_ws wants for this shape (fmt = -1: the fp16 baseline); may be 0."""
    out = ctypes.c_size_t(0)
    _check(load_library().ams_linear_workspace_bytes(fmt, M, N, K, ctypes.byref(out)), "ams_linear_workspace_bytes")
    return out.value


def ams_linear_ws(W_packed, scales, X, N: int, fmt: int, workspace, out=None):
    """ams_linear with a workspace (a zero-filled uint8 CUDA tensor, reusable from call to call)."""
    if out is not None and _call(_WORKSPACE, W_packed, scales, X, N, fmt, out, workspace) is not None:
        return out
    import torch

    M, K = X.shape
    if W_packed.numel() != ams_packed_bytes(fmt, N, K):
        raise ValueError("packed buffer has the wrong size")
    if scales.numel() != N:
        raise ValueError("scales must have N entries")
    if out is None:
        out = torch.empty((M, N), dtype=torch.float16, device=X.device)
    elif out.numel() < M * N:
        raise _too_small(out, M, N)
    rc = load_library().ams_linear_ws(
        _dev_ptr(W_packed, torch.uint8), _dev_ptr(scales, torch.float16), _dev_ptr(X, torch.float16), _dev_ptr(out, torch.float16), M, N, K, fmt,
        _dev_ptr(workspace, torch.uint8) if workspace is not None else None, workspace.numel() if workspace is not None else 0, _stream()
    )
    _check(rc, "ams_linear_ws")
    return out


def ams_linear_static_ws(W_packed, scales, X, N: int, fmt: int, out=None):
    """ams_linear_ws with the library's own static scratch as the workspace (allocates nothing)."""
    if out is not None and _call(_STATIC, W_packed, scales, X, N, fmt, out, None) is not None:
        return out
    import torch

    M, K = X.shape
    if W_packed.numel() != ams_packed_bytes(fmt, N, K):
        raise ValueError("packed buffer has the wrong size")
    if scales.numel() != N:
        raise ValueError("scales must have N entries")
    if out is None:
        out = torch.empty((M, N), dtype=torch.float16, device=X.device)
    elif out.numel() < M * N:
        raise _too_small(out, M, N)
    rc = load_library().ams_linear_static_ws(
        _dev_ptr(W_packed, torch.uint8), _dev_ptr(scales, torch.float16), _dev_ptr(X, torch.float16), _dev_ptr(out, torch.float16), M, N, K, fmt, _stream()
    )
    _check(rc, "ams_linear_static_ws")
    return out


def ams_fp16_linear_ws(W, X, workspace, out=None):
    import torch

    N, K = W.shape
    M = X.shape[0]
    if X.shape[1] != K:
        raise ValueError("X and W disagree in K")
    if out is None:
        out = torch.empty((M, N), dtype=torch.float16, device=X.device)
    elif out.numel() < M * N:
        raise _too_small(out, M, N)
    rc = load_library().ams_fp16_linear_ws(
        _dev_ptr(W, torch.float16), _dev_ptr(X, torch.float16), _dev_ptr(out, torch.float16), M, N, K,
        _dev_ptr(workspace, torch.uint8) if workspace is not None else None, workspace.numel() if workspace is not None else 0, _stream()
    )
    _check(rc, "ams_fp16_linear_ws")
    return out


def ams_linear_plan(fmt: int, M: int, N: int, K: int, with_workspace: bool = False) -> str:
    """Which kernel and launch shape the library would use for this problem (fmt = -1: the fp16 baseline; with_workspace = 2:
    ams_linear_grouped)."""
    buf = ctypes.create_string_buffer(256)
    _check(load_library().ams_linear_plan(fmt, M, N, K, int(with_workspace), buf, len(buf)), "ams_linear_plan")
    return buf.value.decode()


def ams_pack_per_tensor(fmt: int, W: np.ndarray, search: int = SEARCH_SET_BIT, return_codes: bool = False):
    """Quantize + pack with one scale for the whole matrix; returns it once per row, like ams_pack."""
    if W.dtype != np.float16 or W.ndim != 2:
        raise TypeError("W must be a 2-D float16 array")
    W = np.ascontiguousarray(W)
    N, K = W.shape
    packed = np.empty(ams_packed_bytes(fmt, N, K), dtype=np.uint8)
    scales = np.empty(N, dtype=np.float16)
    codes = np.empty((N, K), dtype=np.uint8) if return_codes else None
    rc = load_library().ams_pack_per_tensor(fmt, search, _np_ptr(W), N, K, K, _np_ptr(packed), _np_ptr(scales), _np_ptr(codes) if return_codes else None)
    _check(rc, "ams_pack_per_tensor")
    return (packed, scales, codes) if return_codes else (packed, scales)


def ams_kv_block_bytes(head_dim: int, page_size: int, scale_group: int) -> int:
    """Bytes that page_size tokens of one kv head take in a 4-bit cache."""
    out = ctypes.c_size_t(0)
    _check(load_library().ams_kv_block_bytes(head_dim, page_size, scale_group, ctypes.byref(out)), "ams_kv_block_bytes")
    return out.value


def ams_kv_cache(n_pages: int, kv_heads: int, head_dim: int, page_size: int = 64, scale_group: int = 32, device="cuda"):
    """An empty 4-bit KV cache: uint8 [n_pages, kv_heads, block], a block holding page_size tokens of a head."""
    import torch

    return torch.zeros((n_pages, kv_heads, ams_kv_block_bytes(head_dim, page_size, scale_group)), dtype=torch.uint8, device=device)


def _kv_rows(t, name, heads, head_dim):
    # [rows, heads, head_dim] with the channels of a head side by side
    import torch

    if t.dim() != 3 or t.shape[1] != heads or t.shape[2] != head_dim:
        raise ValueError(f"{name} must be [rows, {heads}, {head_dim}], it is {list(t.shape)}")
    if t.dtype != torch.float16:
        raise TypeError(f"expected {torch.float16}, got {t.dtype}")
    if not t.is_cuda or t.stride(2) != 1:
        raise ValueError(f"{name} must be a CUDA tensor whose last dimension is contiguous")
    if _devices != 1:
        _check_device(t)
    return t.data_ptr()


def _kv_view(cache, block_table, kv_lens, q_starts, head_dim, scale_group):
    import torch

    if cache.dim() != 3 or block_table.dim() != 2 or kv_lens.dim() != 1:
        raise ValueError("expected cache [pages, kv_heads, block], block_table [batch, pages of a sequence] and kv_lens [batch]")
    batch, width = block_table.shape
    if kv_lens.shape[0] != batch:
        raise ValueError(f"block_table has {batch} sequences, kv_lens {kv_lens.shape[0]}")
    if q_starts is not None and tuple(q_starts.shape) != (batch + 1,):
        raise ValueError(f"q_starts must have {batch + 1} entries")
    token = ams_kv_block_bytes(head_dim, 16, scale_group) // 16
    page_size, rest = divmod(cache.shape[2], token)
    if rest:
        raise ValueError(f"a block of {cache.shape[2]} bytes holds no whole number of tokens of {token} bytes")
    if block_table.dtype != torch.int32:
        raise TypeError(f"expected {torch.int32}, got {block_table.dtype}")
    if not block_table.is_cuda or (width > 1 and block_table.stride(1) != 1):
        raise ValueError("block_table must be a CUDA tensor whose last dimension is contiguous")
    if _devices != 1:
        _check_device(block_table)
    return _KvCache(
        _dev_ptr(cache, torch.uint8), block_table.data_ptr(), _dev_ptr(kv_lens, torch.int32), None if q_starts is None else _dev_ptr(q_starts, torch.int32), cache.shape[0],
        block_table.stride(0) if batch > 1 else width, width, batch, cache.shape[1], head_dim, page_size, scale_group
    )


def ams_kv_write(cache, k, v, block_table, kv_lens, scale_group: int = 32, q_starts=None):
    """Quantize rows of k and v, fp16 [rows, kv_heads, head_dim] (views too), into the cache as the last rows of their sequences.

    Sequence b has kv_lens[b] tokens, the new ones among them, in the pages block_table[b] (int32 [batch, pages]); its rows of k and v
    are q_starts[b] .. q_starts[b + 1] - 1 (int32 [batch + 1]; None: one row per sequence).  Returns the cache."""
    if _kv_call(_KV_WRITE, cache, block_table, kv_lens, scale_group, q_starts, k, v):
        return cache
    view = _kv_view(cache, block_table, kv_lens, q_starts, k.shape[-1], scale_group)
    kp, vp = _kv_rows(k, "k", cache.shape[1], k.shape[-1]), _kv_rows(v, "v", cache.shape[1], k.shape[-1])
    if v.shape[0] != k.shape[0]:
        raise ValueError(f"k has {k.shape[0]} rows, v {v.shape[0]}")
    rc = load_library().ams_kv_write(ctypes.byref(view), kp, vp, k.shape[0], k.stride(0), k.stride(1), v.stride(0), v.stride(1), _stream())
    _check(rc, "ams_kv_write")
    return cache


def ams_kv_read(cache, block_table, kv_lens, scale_group: int = 32, head_dim: int = 128, q_starts=None, rows: int = None, out=None):
    """The values that the cache holds for the last rows of each sequence: (k, v), fp16 [rows, kv_heads, head_dim].

    Rows as in ams_kv_write: with q_starts = the cumulated kv_lens whole sequences are read.  `rows` is q_starts[-1] (one per
    sequence without q_starts); with out=(k, v) it is theirs."""
    if out is not None and rows is None and _kv_call(_KV_READ, cache, block_table, kv_lens, scale_group, q_starts, head_dim, *out):
        return out
    import torch

    if out is None and rows is None and q_starts is not None:
        raise ValueError("rows or out must be given with q_starts")
    view = _kv_view(cache, block_table, kv_lens, q_starts, head_dim, scale_group)
    if out is None:
        rows = block_table.shape[0] if rows is None else rows
        out = tuple(torch.empty((rows, cache.shape[1], head_dim), dtype=torch.float16, device=cache.device) for _ in range(2))
    k, v = out
    kp, vp = _kv_rows(k, "out", cache.shape[1], head_dim), _kv_rows(v, "out", cache.shape[1], head_dim)
    if v.shape[0] != k.shape[0] or (rows is not None and rows != k.shape[0]):
        raise ValueError(f"out must hold {k.shape[0] if rows is None else rows} rows, it has {k.shape[0]} and {v.shape[0]}")
    rc = load_library().ams_kv_read(ctypes.byref(view), kp, vp, k.shape[0], k.stride(0), k.stride(1), v.stride(0), v.stride(1), _stream())
    _check(rc, "ams_kv_read")
    return k, v


def ams_kv_attention_workspace_bytes(q, cache, block_table, kv_lens, scale_group: int = 32, q_starts=None, max_q_len: int = None) -> int:
    """Bytes of workspace that ams_kv_attention uses at most for such a call (never more than KV_WORKSPACE_BYTES)."""
    out = ctypes.c_size_t(0)
    view = _kv_view(cache, block_table, kv_lens, q_starts, q.shape[-1], scale_group)
    _check(load_library().ams_kv_attention_workspace_bytes(ctypes.byref(view), q.shape[0], q.shape[1], max_q_len or 0, ctypes.byref(out)), "ams_kv_attention_workspace_bytes")
    return out.value


def ams_kv_attention_plan(q, cache, block_table, kv_lens, scale_group: int = 32, q_starts=None, max_q_len: int = None, window: int = 0, workspace_bytes: int = KV_WORKSPACE_BYTES) -> str:
    """Which kernel and launch shape ams_kv_attention would use for such a call with so much workspace."""
    buf = ctypes.create_string_buffer(256)
    view = _kv_view(cache, block_table, kv_lens, q_starts, q.shape[-1], scale_group)
    _check(load_library().ams_kv_attention_plan(ctypes.byref(view), q.shape[0], q.shape[1], window, max_q_len or 0, workspace_bytes, buf, len(buf)), "ams_kv_attention_plan")
    return buf.value.decode()


def ams_kv_attention(q, cache, block_table, kv_lens, scale_group: int = 32, q_starts=None, max_q_len: int = None, softmax_scale: float = None, causal: bool = True, window: int = 0,
                     workspace=None, out=None, lse=None):
    """softmax(softmax_scale * q k^T) v over the cache, fp16 [rows, heads, head_dim] like q (a view too); heads / kv_heads of them share a kv head.

    q's rows are the last rows of their sequences, as in ams_kv_write: a row sees the keys up to its own (causal), of these the last
    `window` if that is not 0.  softmax_scale: head_dim ** -0.5 by default.  max_q_len: the most rows of a sequence, if
    known (drafts are faster with it; the table's width stands for the lengths where a kernel is chosen).
    workspace: a uint8 CUDA tensor, zero-filled once, that calls may share one after the other; without one a row's keys are not shared out
    to several workgroups.
    lse: fp32 [rows, heads], receives log(sum(exp(scores)))."""
    if out is not None and _kv_call(_KV_ATTENTION, cache, block_table, kv_lens, scale_group, q_starts, q, out, max_q_len, softmax_scale, causal, window, workspace, lse):
        return out
    import torch

    if q.dim() != 3:
        raise ValueError("q must be [rows, heads, head_dim]")
    rows, heads, head_dim = q.shape
    view = _kv_view(cache, block_table, kv_lens, q_starts, head_dim, scale_group)
    if out is None:
        out = torch.empty((rows, heads, head_dim), dtype=torch.float16, device=q.device)
    elif out.dim() != 3 or out.shape[0] != rows:
        raise ValueError(f"out must hold {rows} rows of [{heads}, {head_dim}], it is {list(out.shape)}")
    if lse is not None and (tuple(lse.shape) != (rows, heads) or (heads > 1 and lse.stride(1) != 1)):
        raise ValueError(f"lse must be [{rows}, {heads}] with a contiguous last dimension")
    if lse is not None and (lse.dtype != torch.float32 or not lse.is_cuda):
        raise TypeError("lse must be a float32 CUDA tensor")
    if lse is not None and _devices != 1:
        _check_device(lse)
    rc = load_library().ams_kv_attention(
        ctypes.byref(view), _kv_rows(q, "q", heads, head_dim), _kv_rows(out, "out", heads, head_dim), lse.data_ptr() if lse is not None else None, rows, heads, q.stride(0), q.stride(1),
        out.stride(0), out.stride(1), lse.stride(0) if lse is not None else 0, head_dim**-0.5 if softmax_scale is None else softmax_scale, int(causal), window, max_q_len or 0,
        _dev_ptr(workspace, torch.uint8) if workspace is not None else None, workspace.numel() if workspace is not None else 0, _stream()
    )
    _check(rc, "ams_kv_attention")
    return out
