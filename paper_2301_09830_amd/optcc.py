"""Python binding of liboptcc (ctypes): argument marshalling only.

Every function here converts torch tensors to the pointers, sizes and the
stream the C ABI expects and calls the function of the same name in
liboptcc.so (the layers through csrc/bind_layers.cpp, native for its host time); all computation happens in the library's HIP kernels.  There is
no fallback: if the library is missing or fails to load, every call raises.

Tensors are row-major 2-D CUDA (HIP) tensors with unit column stride; the
leading dimension is taken from stride(0).  M is torch.float32 or
torch.bfloat16; err, P, Q and M_hat are torch.float32; P is rows x rank and Q
is cols x rank, contiguous.  Work is enqueued on torch's current stream.
"""

from __future__ import annotations

import contextlib
import ctypes
import os
import re
from typing import Any, NamedTuple

PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(PKG, "liboptcc.so")
HEADER = os.path.join(os.path.dirname(PKG), "include", "optcc.h")

OCC_OK = 0
OCC_F32, OCC_BF16 = 0, 1
OCC_F_NONFINITE, OCC_F_RANK_DEFICIENT, OCC_F_BAD_ROWS = 1, 2, 4
OCC_NO_MHAT = 1
OCC_DEC_SPLIT_BF16, OCC_DEC_OUT_BF16 = 1, 2
OCC_MAX_RANK = 128
OCC_NOALLOC_MAX_BYTES = 64 << 20
OCC_MAX_ITERS = 64
OCC_ACT_NONE, OCC_ACT_RELU, OCC_ACT_GELU, OCC_ACT_GELU_TANH, OCC_ACT_SILU = range(5)
OCC_GRAD_ACCUMULATE = 1
OCC_SCALE_RUN = 256   # columns that share one scale of an 8-bit moment
OCC_MAX_EXPERTS, OCC_MAX_CHOICES, OCC_MAX_TEACHER = 1024, 32, 1024

STATUS_NAMES = {
    0: "OCC_OK", 1: "OCC_E_NULL", 2: "OCC_E_SHAPE", 3: "OCC_E_RANK", 4: "OCC_E_ITERS",
    5: "OCC_E_DTYPE", 6: "OCC_E_ALIGN", 7: "OCC_E_ALIAS", 8: "OCC_E_WORKSPACE",
    9: "OCC_E_HIP", 10: "OCC_E_FLAGS", 11: "OCC_E_VALUE",
}


class OccError(RuntimeError):
    """A liboptcc call returned a non-zero occ_status_t."""

    def __init__(self, fn: str, status: int):
        self.status = status
        self.code = STATUS_NAMES.get(status, str(status))
        super().__init__(f"{fn}: {self.code} ({occ_status_str(status)})")


class occ_mat_t(ctypes.Structure):
    _fields_ = [
        ("M", ctypes.c_void_p),
        ("m_dtype", ctypes.c_int32),
        ("reserved", ctypes.c_int32),
        ("rows", ctypes.c_int64),
        ("cols", ctypes.c_int64),
        ("ldm", ctypes.c_int64),
        ("err", ctypes.c_void_p),
        ("lde", ctypes.c_int64),
        ("P", ctypes.c_void_p),
        ("Q", ctypes.c_void_p),
        ("M_hat", ctypes.c_void_p),
        ("ldh", ctypes.c_int64),
    ]


class occ_stage_t(ctypes.Structure):
    _fields_ = [
        ("bwd_done", ctypes.c_double),
        ("comm", ctypes.c_double),
        ("comm_compressed", ctypes.c_double),
        ("compress", ctypes.c_double),
    ]


class occ_kernel_time_t(ctypes.Structure):
    _fields_ = [
        ("name", ctypes.c_char * 48),
        ("launches", ctypes.c_int32),
        ("reserved", ctypes.c_int32),
        ("total_ms", ctypes.c_double),
    ]


class occ_linear_t(ctypes.Structure):
    _fields_ = [
        ("dtype", ctypes.c_int32),
        ("act", ctypes.c_int32),
        ("tokens", ctypes.c_int64),
        ("in_", ctypes.c_int64),
        ("out", ctypes.c_int64),
        ("X", ctypes.c_void_p),
        ("ldx", ctypes.c_int64),
        ("W", ctypes.c_void_p),
        ("ldw", ctypes.c_int64),
        ("bias", ctypes.c_void_p),
        ("R", ctypes.c_void_p),
        ("ldr", ctypes.c_int64),
        ("Z", ctypes.c_void_p),
        ("ldz", ctypes.c_int64),
        ("Y", ctypes.c_void_p),
        ("ldy", ctypes.c_int64),
    ]


class occ_linear_grad_t(ctypes.Structure):
    _fields_ = [
        ("dtype", ctypes.c_int32),
        ("dw_dtype", ctypes.c_int32),
        ("act", ctypes.c_int32),
        ("reserved", ctypes.c_int32),
        ("tokens", ctypes.c_int64),
        ("in_", ctypes.c_int64),
        ("out", ctypes.c_int64),
        ("dY", ctypes.c_void_p),
        ("lddy", ctypes.c_int64),
        ("X", ctypes.c_void_p),
        ("ldx", ctypes.c_int64),
        ("W", ctypes.c_void_p),
        ("ldw", ctypes.c_int64),
        ("Z", ctypes.c_void_p),
        ("ldz", ctypes.c_int64),
        ("dX", ctypes.c_void_p),
        ("lddx", ctypes.c_int64),
        ("dW", ctypes.c_void_p),
        ("lddw", ctypes.c_int64),
        ("dbias", ctypes.c_void_p),
    ]


class occ_experts_t(ctypes.Structure):
    _fields_ = [
        ("l", occ_linear_t),
        ("experts", ctypes.c_int64),
        ("stride_w", ctypes.c_int64),
        ("offsets", ctypes.c_void_p),
        ("flags", ctypes.c_void_p),
    ]


class occ_experts_grad_t(ctypes.Structure):
    _fields_ = [
        ("l", occ_linear_grad_t),
        ("experts", ctypes.c_int64),
        ("stride_w", ctypes.c_int64),
        ("stride_dw", ctypes.c_int64),
        ("offsets", ctypes.c_void_p),
        ("flags", ctypes.c_void_p),
    ]


class occ_route_t(ctypes.Structure):
    _fields_ = [
        ("dtype", ctypes.c_int32),
        ("k", ctypes.c_int32),
        ("renorm", ctypes.c_int32),
        ("reserved", ctypes.c_int32),
        ("tokens", ctypes.c_int64),
        ("experts", ctypes.c_int64),
        ("logits", ctypes.c_void_p),
        ("ldl", ctypes.c_int64),
        ("index", ctypes.c_void_p),
        ("weights", ctypes.c_void_p),
        ("offsets", ctypes.c_void_p),
        ("order", ctypes.c_void_p),
        ("slots", ctypes.c_void_p),
    ]


class occ_exchange_t(ctypes.Structure):
    _fields_ = [
        ("dtype", ctypes.c_int32),
        ("k", ctypes.c_int32),
        ("tokens", ctypes.c_int64),
        ("experts", ctypes.c_int64),
        ("rows", ctypes.c_int64),
        ("width", ctypes.c_int64),
        ("offsets", ctypes.c_void_p),
        ("order", ctypes.c_void_p),
        ("slots", ctypes.c_void_p),
        ("flags", ctypes.c_void_p),
    ]


class occ_distill_t(ctypes.Structure):
    _fields_ = [
        ("dtype", ctypes.c_int32),
        ("t_dtype", ctypes.c_int32),
        ("tokens", ctypes.c_int64),
        ("vocab", ctypes.c_int64),
        ("S", ctypes.c_void_p),
        ("lds", ctypes.c_int64),
        ("k", ctypes.c_int32),
        ("reserved", ctypes.c_int32),
        ("index", ctypes.c_void_p),
        ("ldi", ctypes.c_int64),
        ("teacher", ctypes.c_void_p),
        ("ldt", ctypes.c_int64),
        ("labels", ctypes.c_void_p),
        ("scale", ctypes.c_void_p),
        ("temperature", ctypes.c_float),
        ("alpha", ctypes.c_float),
        ("loss", ctypes.c_void_p),
        ("lse", ctypes.c_void_p),
        ("dS", ctypes.c_void_p),
        ("ldds", ctypes.c_int64),
        ("flags", ctypes.c_void_p),
    ]


class occ_param_t(ctypes.Structure):
    _fields_ = [
        ("rows", ctypes.c_int64),
        ("cols", ctypes.c_int64),
        ("W", ctypes.c_void_p),
        ("W16", ctypes.c_void_p),
        ("G", ctypes.c_void_p),
        ("ldg", ctypes.c_int64),
        ("g_dtype", ctypes.c_int32),
        ("rank", ctypes.c_int32),
        ("P", ctypes.c_void_p),
        ("Q", ctypes.c_void_p),
        ("m", ctypes.c_void_p),
        ("v", ctypes.c_void_p),
        ("m_scale", ctypes.c_void_p),
        ("v_scale", ctypes.c_void_p),
        ("state_bits", ctypes.c_int32),
        ("decay", ctypes.c_float),
    ]


class occ_adamw_t(ctypes.Structure):
    _fields_ = [
        ("lr", ctypes.c_double),
        ("beta1", ctypes.c_double),
        ("beta2", ctypes.c_double),
        ("eps", ctypes.c_double),
        ("step", ctypes.c_int64),
        ("seed", ctypes.c_uint32),
        ("reserved", ctypes.c_uint32),
        ("grad_scale", ctypes.c_void_p),
        ("flags", ctypes.c_void_p),
    ]


_lib = None

_SIGS = {
    "occ_abi_version": (ctypes.c_int, []),
    "occ_status_str": (ctypes.c_char_p, [ctypes.c_int]),
    "occ_workspace_bytes": (ctypes.c_size_t, [ctypes.POINTER(occ_mat_t), ctypes.c_int,
                                              ctypes.c_int, ctypes.c_int]),
    "occ_compress_workspace_bytes": (ctypes.c_size_t, [ctypes.c_int64, ctypes.c_int64,
                                                       ctypes.c_int, ctypes.c_int, ctypes.c_int]),
    "occ_workspace_init": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]),
    "occ_compress": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_int64,
                                    ctypes.c_int64, ctypes.c_void_p, ctypes.c_int64,
                                    ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int, ctypes.c_int,
                                    ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]),
    "occ_decompress": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int64,
                                      ctypes.c_int64, ctypes.c_int, ctypes.c_void_p,
                                      ctypes.c_int64, ctypes.c_void_p]),
    "occ_decompress_ex": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int64,
                                         ctypes.c_int64, ctypes.c_int, ctypes.c_uint,
                                         ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p]),
    "occ_err_update": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_int, ctypes.c_int64,
                                      ctypes.c_int64, ctypes.c_int64, ctypes.c_void_p,
                                      ctypes.c_int64, ctypes.c_void_p, ctypes.c_int64,
                                      ctypes.c_void_p, ctypes.c_void_p]),
    "occ_step": (ctypes.c_int, [ctypes.POINTER(occ_mat_t), ctypes.c_int, ctypes.c_int,
                                ctypes.c_uint, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]),
    "occ_step_batched": (ctypes.c_int, [ctypes.POINTER(occ_mat_t), ctypes.c_int, ctypes.c_int,
                                        ctypes.c_int, ctypes.c_uint, ctypes.c_void_p,
                                        ctypes.c_size_t, ctypes.c_void_p]),
    "occ_step_rows": (ctypes.c_int, [ctypes.POINTER(occ_mat_t), ctypes.c_void_p, ctypes.c_int64,
                                     ctypes.c_int, ctypes.c_int, ctypes.c_uint, ctypes.c_void_p,
                                     ctypes.c_size_t, ctypes.c_void_p]),
    "occ_step_rows_workspace_bytes": (ctypes.c_size_t, [ctypes.c_int64, ctypes.c_int64,
                                                        ctypes.c_int, ctypes.c_int, ctypes.c_int]),
    "occ_step_batched_noalloc": (ctypes.c_int, [ctypes.POINTER(occ_mat_t), ctypes.c_int,
                                                ctypes.c_int, ctypes.c_int, ctypes.c_uint,
                                                ctypes.c_void_p, ctypes.c_void_p]),
    "occ_get_flags": (ctypes.c_int, [ctypes.c_void_p, ctypes.POINTER(ctypes.c_uint32),
                                     ctypes.c_int, ctypes.c_void_p]),
    "occ_pipeline_1f1b": (ctypes.c_int, [ctypes.c_int, ctypes.c_int, ctypes.c_double,
                                         ctypes.c_double, ctypes.c_double,
                                         ctypes.POINTER(ctypes.c_double),
                                         ctypes.POINTER(ctypes.c_double)]),
    "occ_sc_select": (ctypes.c_int, [ctypes.POINTER(occ_stage_t), ctypes.c_int, ctypes.c_int,
                                     ctypes.POINTER(ctypes.c_uint8), ctypes.POINTER(ctypes.c_int),
                                     ctypes.POINTER(ctypes.c_double)]),
    "occ_linear_fwd_workspace_bytes": (ctypes.c_size_t, [ctypes.POINTER(occ_linear_t)]),
    "occ_gated_fwd_workspace_bytes": (ctypes.c_size_t, [ctypes.POINTER(occ_linear_t)]),
    "occ_linear_bwd_workspace_bytes": (ctypes.c_size_t, [ctypes.POINTER(occ_linear_grad_t)]),
    "occ_gated_bwd_workspace_bytes": (ctypes.c_size_t, [ctypes.POINTER(occ_linear_grad_t)]),
    "occ_linear_fwd": (ctypes.c_int, [ctypes.POINTER(occ_linear_t), ctypes.c_void_p,
                                      ctypes.c_size_t, ctypes.c_void_p]),
    "occ_gated_fwd": (ctypes.c_int, [ctypes.POINTER(occ_linear_t), ctypes.c_void_p,
                                     ctypes.c_size_t, ctypes.c_void_p]),
    "occ_linear_bwd": (ctypes.c_int, [ctypes.POINTER(occ_linear_grad_t), ctypes.c_uint,
                                      ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]),
    "occ_gated_bwd": (ctypes.c_int, [ctypes.POINTER(occ_linear_grad_t), ctypes.c_uint,
                                     ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]),
    **{f"occ_experts_{n}_{d}_workspace_bytes": (ctypes.c_size_t, [ctypes.POINTER(t)])
       for n in ("linear", "gated") for d, t in (("fwd", occ_experts_t),
                                                 ("bwd", occ_experts_grad_t))},
    **{f"occ_experts_{n}_fwd": (ctypes.c_int, [ctypes.POINTER(occ_experts_t), ctypes.c_void_p,
                                               ctypes.c_size_t, ctypes.c_void_p])
       for n in ("linear", "gated")},
    **{f"occ_experts_{n}_bwd": (ctypes.c_int, [ctypes.POINTER(occ_experts_grad_t), ctypes.c_uint,
                                               ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p])
       for n in ("linear", "gated")},
    "occ_route_fwd_workspace_bytes": (ctypes.c_size_t, [ctypes.POINTER(occ_route_t)]),
    "occ_route_fwd": (ctypes.c_int, [ctypes.POINTER(occ_route_t), ctypes.c_void_p,
                                     ctypes.c_size_t, ctypes.c_void_p]),
    "occ_route_bwd": (ctypes.c_int, [ctypes.POINTER(occ_route_t), ctypes.c_void_p,
                                     ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p]),
    "occ_dispatch": (ctypes.c_int, [ctypes.POINTER(occ_exchange_t), ctypes.c_void_p,
                                    ctypes.c_int64, ctypes.c_void_p, ctypes.c_int64,
                                    ctypes.c_void_p]),
    "occ_combine": (ctypes.c_int, [ctypes.POINTER(occ_exchange_t), ctypes.c_void_p,
                                   ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p,
                                   ctypes.c_int64, ctypes.c_void_p, ctypes.c_int64,
                                   ctypes.c_void_p]),
    "occ_combine_bwd": (ctypes.c_int, [ctypes.POINTER(occ_exchange_t), ctypes.c_void_p,
                                       ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p,
                                       ctypes.c_int64, ctypes.c_void_p, ctypes.c_int64,
                                       ctypes.c_void_p, ctypes.c_void_p]),
    "occ_distill_fwd": (ctypes.c_int, [ctypes.POINTER(occ_distill_t), ctypes.c_void_p]),
    "occ_distill_bwd": (ctypes.c_int, [ctypes.POINTER(occ_distill_t), ctypes.c_void_p]),
    "occ_adamw_step": (ctypes.c_int, [ctypes.POINTER(occ_param_t), ctypes.c_int,
                                      ctypes.POINTER(occ_adamw_t), ctypes.c_void_p]),
    "occ_profile_begin": (ctypes.c_int, []),
    "occ_profile_end": (ctypes.c_int, [ctypes.POINTER(occ_kernel_time_t), ctypes.c_int,
                                       ctypes.POINTER(ctypes.c_int)]),
}


def lib() -> ctypes.CDLL:
    """The loaded in-tree liboptcc.so; raises if it has not been built."""
    global _lib
    if _lib is None:
        path = LIB_PATH
        if not os.path.exists(path):
            raise RuntimeError(f"{path} is missing: build it with "
                               "`python -m paper_2301_09830_amd.build`")
        handle = ctypes.CDLL(path)
        for name, (res, args) in _SIGS.items():
            fn = getattr(handle, name)
            fn.restype = res
            fn.argtypes = args
        _lib = handle
    return _lib


def header_symbols() -> list:
    """Names of the functions declared in include/optcc.h."""
    text = open(HEADER).read()
    return sorted(set(re.findall(r"\b(occ_[a-z_]+)\s*\(", text)))


def _check(fn: str, status: int) -> None:
    if status != OCC_OK:
        raise OccError(fn, status)


def occ_abi_version() -> int:
    return lib().occ_abi_version()


def occ_status_str(status: int) -> str:
    return lib().occ_status_str(status).decode()


# ----------------------------------------------------------------------------
# tensor marshalling
# ----------------------------------------------------------------------------
_torch_module = None


def _torch():
    global _torch_module
    if _torch_module is None:
        import torch
        _torch_module = torch
    return _torch_module


def _stream(stream=None) -> int:
    if stream is not None:
        return int(stream.cuda_stream)
    torch = _torch()
    # torch.cuda.current_stream().cuda_stream without the Stream object (3 us a call)
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


def _ptr(t) -> int | None:
    return None if t is None else int(t.data_ptr())


def _ld(t, name: str) -> int:
    if t.dim() != 2:
        raise ValueError(f"{name} must be 2-D")
    if t.shape[1] > 1 and t.stride(1) != 1:
        raise ValueError(f"{name} must have unit column stride (row-major)")
    return int(t.stride(0)) if t.shape[0] > 1 else int(t.shape[1])


def _mdtype(M) -> int:
    torch = _torch()
    if M.dtype == torch.float32:
        return OCC_F32
    if M.dtype == torch.bfloat16:
        return OCC_BF16
    raise TypeError("M must be float32 or bfloat16")


def _f32(t, name: str):
    torch = _torch()
    if t is not None and t.dtype != torch.float32:
        raise TypeError(f"{name} must be float32")
    return t


def make_mat(M, err, P, Q, M_hat=None) -> occ_mat_t:
    """occ_mat_t describing one matrix and its compressor state."""
    _f32(err, "err"), _f32(P, "P"), _f32(Q, "Q"), _f32(M_hat, "M_hat")
    if P.dim() != 2 or Q.dim() != 2 or P.shape[0] != M.shape[0] or Q.shape[0] != M.shape[1] \
            or P.shape[1] != Q.shape[1]:
        raise ValueError("P must be rows x rank and Q cols x rank")
    if not (P.is_contiguous() and Q.is_contiguous()):
        raise ValueError("P and Q must be contiguous")
    a = occ_mat_t()
    a.M = _ptr(M)
    a.m_dtype = _mdtype(M)
    a.rows, a.cols = int(M.shape[0]), int(M.shape[1])
    a.ldm = _ld(M, "M")
    a.err = _ptr(err)
    a.lde = _ld(err, "err")
    a.P = _ptr(P)
    a.Q = _ptr(Q)
    a.M_hat = _ptr(M_hat)
    a.ldh = _ld(M_hat, "M_hat") if M_hat is not None else 0
    return a


def occ_workspace_bytes(shapes, rank: int, iters: int, m_dtype: int = OCC_F32) -> int:
    """Workspace bytes for matrices of the given (rows, cols) shapes whose M
    has dtype m_dtype (OCC_F32 or OCC_BF16)."""
    arr = (occ_mat_t * len(shapes))()
    for a, (m, n) in zip(arr, shapes):
        a.rows, a.cols, a.ldm, a.m_dtype = m, n, n, m_dtype
    return int(lib().occ_workspace_bytes(arr, len(shapes), rank, iters))


def occ_compress_workspace_bytes(m: int, n: int, rank: int, iters: int,
                                 m_dtype: int = OCC_F32) -> int:
    return int(lib().occ_compress_workspace_bytes(m, n, m_dtype, rank, iters))


def alloc_workspace(nbytes: int, device="cuda", stream=None):
    """A zero-headed workspace tensor of at least nbytes (256-byte aligned)."""
    torch = _torch()
    ws = torch.empty(max(int(nbytes), 256) + 256, dtype=torch.uint8, device=device)
    off = (-ws.data_ptr()) % 256
    ws = ws[off:off + max(int(nbytes), 256)]
    occ_workspace_init(ws, stream)
    return ws


def occ_workspace_init(ws, stream=None) -> None:
    _check("occ_workspace_init", lib().occ_workspace_init(_ptr(ws), ws.numel(), _stream(stream)))


def occ_step(M, err, Q, rank: int, iters: int, P=None, M_hat=None, write_mhat: bool = True,
             ws=None, stream=None):
    """Fused compress + decompress + error update; err and Q updated in place.

    Returns (P, M_hat) (M_hat is None when write_mhat is False).
    """
    torch = _torch()
    m, n = M.shape
    if P is None:
        P = torch.empty((m, rank), dtype=torch.float32, device=M.device)
    if write_mhat and M_hat is None:
        M_hat = torch.empty((m, n), dtype=torch.float32, device=M.device)
    if P.shape[1] != rank:
        raise ValueError("P and Q must have `rank` columns")
    mat = make_mat(M, err, P, Q, M_hat if write_mhat else None)
    if ws is None:
        ws = alloc_workspace(lib().occ_workspace_bytes(ctypes.byref(mat), 1, rank, iters),
                             M.device, stream)
    flags = 0 if write_mhat else OCC_NO_MHAT
    _check("occ_step", lib().occ_step(ctypes.byref(mat), rank, iters, flags, _ptr(ws),
                                      ws.numel(), _stream(stream)))
    return P, (M_hat if write_mhat else None)


def occ_step_batched(items, rank: int, iters: int, write_mhat: bool = True, ws=None,
                     stream=None):
    """occ_step on independent matrices in one launch per pass.

    items: sequence of (M, err, Q, P, M_hat) tuples (P and M_hat preallocated;
    M_hat may be None when write_mhat is False).
    """
    arr = (occ_mat_t * len(items))()
    for a, (M, err, Q, P, M_hat) in zip(arr, items):
        ctypes.memmove(ctypes.byref(a), ctypes.byref(make_mat(M, err, P, Q,
                                                              M_hat if write_mhat else None)),
                       ctypes.sizeof(occ_mat_t))
    if ws is None:
        ws = alloc_workspace(lib().occ_workspace_bytes(arr, len(items), rank, iters),
                             items[0][0].device, stream)
    flags = 0 if write_mhat else OCC_NO_MHAT
    _check("occ_step_batched", lib().occ_step_batched(arr, len(items), rank, iters, flags,
                                                      _ptr(ws), ws.numel(), _stream(stream)))
    return ws


def occ_step_batched_noalloc(items, rank: int, iters: int, write_mhat: bool = True,
                             flags_out=None, stream=None) -> None:
    """occ_step_batched on the library's static per-GPU workspace (no device
    allocation by the library or by this binding).  items as for
    occ_step_batched; flags_out: optional int32 CUDA tensor of one element
    that receives the numeric flags (OR-ed in)."""
    arr = (occ_mat_t * len(items))()
    for a, (M, err, Q, P, M_hat) in zip(arr, items):
        ctypes.memmove(ctypes.byref(a), ctypes.byref(make_mat(M, err, P, Q,
                                                              M_hat if write_mhat else None)),
                       ctypes.sizeof(occ_mat_t))
    flags = 0 if write_mhat else OCC_NO_MHAT
    _check("occ_step_batched_noalloc",
           lib().occ_step_batched_noalloc(arr, len(items), rank, iters, flags, _ptr(flags_out),
                                          _stream(stream)))


def occ_step_rows_workspace_bytes(n_rows: int, cols: int, rank: int, iters: int,
                                  m_dtype: int = OCC_F32) -> int:
    return int(lib().occ_step_rows_workspace_bytes(n_rows, cols, m_dtype, rank, iters))


def occ_step_rows(M, err, Q, rows, rank: int, iters: int, P=None, M_hat=None,
                  write_mhat: bool = True, ws=None, stream=None):
    """Row-sparse step: compress the listed rows of M + err (rows: int32 CUDA
    tensor, strictly increasing); err and Q updated in place, only the listed
    rows of err and M_hat are written.  Returns (P, M_hat) with P compact
    (len(rows) x rank).  A newly allocated M_hat is zero-filled, so that its
    unlisted rows hold the dense step's zeros."""
    torch = _torch()
    m, n = M.shape
    if rows.dtype != torch.int32 or rows.dim() != 1 or not rows.is_contiguous():
        raise TypeError("rows must be a contiguous 1-D int32 tensor")
    n_rows = int(rows.numel())
    if P is None:
        P = torch.empty((n_rows, rank), dtype=torch.float32, device=M.device)
    if write_mhat and M_hat is None:
        M_hat = torch.zeros((m, n), dtype=torch.float32, device=M.device)
    _f32(err, "err"), _f32(P, "P"), _f32(Q, "Q"), _f32(M_hat, "M_hat")
    if P.shape != (n_rows, rank) or Q.shape != (n, rank) or not (P.is_contiguous() and
                                                                 Q.is_contiguous()):
        raise ValueError("P must be len(rows) x rank and Q cols x rank, both contiguous")
    a = occ_mat_t()
    a.M = _ptr(M)
    a.m_dtype = _mdtype(M)
    a.rows, a.cols = m, n
    a.ldm = _ld(M, "M")
    a.err = _ptr(err)
    a.lde = _ld(err, "err")
    a.P = _ptr(P) if n_rows else None
    a.Q = _ptr(Q)
    a.M_hat = _ptr(M_hat) if write_mhat else None
    a.ldh = _ld(M_hat, "M_hat") if write_mhat else 0
    if ws is None:
        ws = alloc_workspace(occ_step_rows_workspace_bytes(n_rows, n, rank, iters, a.m_dtype),
                             M.device, stream)
    flags = 0 if write_mhat else OCC_NO_MHAT
    _check("occ_step_rows", lib().occ_step_rows(ctypes.byref(a), _ptr(rows) if n_rows else None,
                                                n_rows, rank, iters, flags, _ptr(ws), ws.numel(),
                                                _stream(stream)))
    return P, (M_hat if write_mhat else None)


def occ_compress(M, err_prev, Q, rank: int, iters: int, P=None, ws=None, stream=None):
    """A = M + err_prev (err_prev may be None); Q updated in place; returns P_hat."""
    torch = _torch()
    m, n = M.shape
    _f32(err_prev, "err_prev"), _f32(Q, "Q")
    if P is None:
        P = torch.empty((m, rank), dtype=torch.float32, device=M.device)
    if ws is None:
        ws = alloc_workspace(occ_compress_workspace_bytes(m, n, rank, iters, _mdtype(M)),
                             M.device, stream)
    lde = _ld(err_prev, "err_prev") if err_prev is not None else 0
    _check("occ_compress", lib().occ_compress(_ptr(M), _mdtype(M), m, n, _ld(M, "M"),
                                              _ptr(err_prev), lde, _ptr(P), _ptr(Q), rank, iters,
                                              _ptr(ws), ws.numel(), _stream(stream)))
    return P


def occ_decompress(P, Q, M_hat=None, stream=None):
    """M_hat = P Q^T (fp32 products, fp32 M_hat)."""
    torch = _torch()
    _f32(P, "P"), _f32(Q, "Q"), _f32(M_hat, "M_hat")
    m, rank = P.shape
    n = Q.shape[0]
    if M_hat is None:
        M_hat = torch.empty((m, n), dtype=torch.float32, device=P.device)
    _check("occ_decompress", lib().occ_decompress(_ptr(P), _ptr(Q), m, n, rank, _ptr(M_hat),
                                                  _ld(M_hat, "M_hat"), _stream(stream)))
    return M_hat


def occ_decompress_ex(P, Q, flags: int = 0, M_hat=None, stream=None):
    """M_hat = P Q^T with OCC_DEC_* flags: OCC_DEC_SPLIT_BF16 runs the products
    occ_step uses for a bf16 M; OCC_DEC_OUT_BF16 stores M_hat as bfloat16."""
    torch = _torch()
    _f32(P, "P"), _f32(Q, "Q")
    m, rank = P.shape
    n = Q.shape[0]
    out_dtype = torch.bfloat16 if flags & OCC_DEC_OUT_BF16 else torch.float32
    if M_hat is None:
        M_hat = torch.empty((m, n), dtype=out_dtype, device=P.device)
    if M_hat.dtype != out_dtype:
        raise TypeError(f"M_hat must be {out_dtype} for these flags")
    _check("occ_decompress_ex", lib().occ_decompress_ex(_ptr(P), _ptr(Q), m, n, rank, flags,
                                                        _ptr(M_hat), _ld(M_hat, "M_hat"),
                                                        _stream(stream)))
    return M_hat


def occ_err_update(M, err_prev, M_hat, err_new=None, stream=None):
    """err_new = (M + err_prev) - M_hat; err_new may be err_prev (in place).
    err_prev and err_new share one leading dimension."""
    torch = _torch()
    m, n = M.shape
    if err_new is None:
        ld = _ld(err_prev, "err_prev") if err_prev is not None else n
        err_new = torch.empty((m, ld), dtype=torch.float32, device=M.device)[:, :n]
    lde = _ld(err_new, "err_new")
    if err_prev is not None and _ld(err_prev, "err_prev") != lde:
        raise ValueError("err_prev and err_new must share one leading dimension")
    _check("occ_err_update", lib().occ_err_update(_ptr(M), _mdtype(M), m, n, _ld(M, "M"),
                                                  _ptr(err_prev), lde, _ptr(M_hat),
                                                  _ld(M_hat, "M_hat"), _ptr(err_new),
                                                  _stream(stream)))
    return err_new


def occ_pipeline_1f1b(n_stages: int, n_micro: int, t_fwd: float, t_bwd: float,
                      t_p2p: float = 0.0):
    """(bwd_done per stage, end of the schedule) under one-forward-one-backward."""
    out = (ctypes.c_double * n_stages)()
    end = ctypes.c_double(0.0)
    _check("occ_pipeline_1f1b", lib().occ_pipeline_1f1b(n_stages, n_micro, t_fwd, t_bwd, t_p2p,
                                                        out, ctypes.byref(end)))
    return list(out), end.value


def occ_sc_select(stages, max_compressed: int):
    """stages: sequence of (bwd_done, comm, comm_compressed, compress).
    Returns (selected flags per stage, end of the last exchange)."""
    arr = (occ_stage_t * len(stages))(*[occ_stage_t(*map(float, t)) for t in stages])
    sel = (ctypes.c_uint8 * len(stages))()
    n = ctypes.c_int(0)
    end = ctypes.c_double(0.0)
    _check("occ_sc_select", lib().occ_sc_select(arr, len(stages), max_compressed, sel,
                                                ctypes.byref(n), ctypes.byref(end)))
    return [int(x) for x in sel], end.value


def occ_get_flags(ws, clear: bool = False, stream=None) -> int:
    out = ctypes.c_uint32(0)
    _check("occ_get_flags", lib().occ_get_flags(_ptr(ws), ctypes.byref(out), int(clear),
                                                _stream(stream)))
    return int(out.value)


# ----------------------------------------------------------------------------
# stage operators
# ----------------------------------------------------------------------------
def _vec(t, name: str, n: int):
    if t.dtype is not _torch().float32:
        raise TypeError(f"{name} must be float32")
    if t.numel() != n or not t.is_contiguous():
        raise ValueError(f"{name} must hold {n} contiguous values")
    return t.data_ptr()


_layers_module = None


def _layers():
    """The native binding of the layers, on the loaded library's functions."""
    global _layers_module
    if _layers_module is None:
        torch, L = _torch(), lib()
        path = os.path.join(PKG, "_layers.so")
        if not os.path.exists(path):
            raise RuntimeError(f"{path} is missing: build it with "
                               "`python -m paper_2301_09830_amd.build`")
        from . import _layers as module
        names = [n + e for e in ("", "_workspace_bytes")
                 for n in ("occ_linear_fwd", "occ_gated_fwd", "occ_linear_bwd", "occ_gated_bwd")]
        def address(name):
            return ctypes.cast(getattr(L, name), ctypes.c_void_p).value

        module.setup(*map(address, names), torch._C._cuda_getCurrentRawStream)
        experts = [f"occ_experts_{n}_{d}{e}" for e in ("", "_workspace_bytes")
                   for d in ("fwd", "bwd") for n in ("linear", "gated")]
        module.setup_experts(*map(address, experts + [
            "occ_route_fwd", "occ_route_fwd_workspace_bytes", "occ_route_bwd", "occ_dispatch",
            "occ_combine", "occ_combine_bwd", "occ_distill_fwd", "occ_distill_bwd"]))
        _layers_module = module
    return _layers_module


def _on(stream, call, *args):
    """A layer's call on a given stream: what it allocates belongs to it too."""
    with _torch().cuda.stream(stream):
        return call(*args)


def _layer_fwd(name: str, gated: bool, X, W, bias, act, R, Y, Z, ws):
    if Y is None:
        if X.dim() != 2 or W.dim() != 2:
            raise ValueError("X and W must be 2-D")
        Y = X.new_empty((X.shape[0], W.shape[0] // 2 if gated else W.shape[0]))
    status = (_layers_module or _layers()).forward(gated, X, W, bias, act, R, Y, Z, ws)
    if status:
        raise OccError(name, status)
    return Y


def occ_linear_fwd(X, W, bias=None, act: int = OCC_ACT_NONE, R=None, Y=None, Z=None, ws=None,
                   stream=None):
    """Y = act(X W^T + bias) + R; Z, if given, receives the pre-activation.

    X tokens x in, W out x in, R, Y and Z tokens x out, all float32 or all
    bfloat16; bias float32.  R may be Y.  Returns Y.
    """
    if stream is not None:
        return _on(stream, occ_linear_fwd, X, W, bias, act, R, Y, Z, ws)
    return _layer_fwd("occ_linear_fwd", False, X, W, bias, act, R, Y, Z, ws)


def occ_gated_fwd(X, W, bias=None, act: int = OCC_ACT_SILU, R=None, Y=None, Z=None, ws=None,
                  stream=None):
    """[G U] = X W^T + bias; Y = act(G) * U + R; Z, if given, receives [G U].

    W is 2 out x in: the gate's rows, then the other projection's.
    """
    if stream is not None:
        return _on(stream, occ_gated_fwd, X, W, bias, act, R, Y, Z, ws)
    return _layer_fwd("occ_gated_fwd", True, X, W, bias, act, R, Y, Z, ws)


def _layer_bwd(name: str, gated: bool, dY, X, W, Z, act, dX, dW, dbias, accumulate, ws):
    status = (_layers_module or _layers()).backward(
        gated, dY, X, W, Z, act, dX, dW, dbias, OCC_GRAD_ACCUMULATE if accumulate else 0, ws)
    if status:
        raise OccError(name, status)


def occ_linear_bwd(dY, X=None, W=None, Z=None, act: int = OCC_ACT_NONE, dX=None, dW=None,
                   dbias=None, accumulate: bool = False, ws=None, stream=None) -> None:
    """Gradients of occ_linear_fwd, each made if a tensor is given for it:
    dX (needs W), dW (needs X; may be float32 for a bfloat16 layer), dbias.
    Z is the stored pre-activation (not needed with OCC_ACT_NONE).  accumulate:
    dW and dbias are added to.  The gradient of R is dY itself.
    """
    if stream is not None:
        return _on(stream, occ_linear_bwd, dY, X, W, Z, act, dX, dW, dbias, accumulate, ws)
    _layer_bwd("occ_linear_bwd", False, dY, X, W, Z, act, dX, dW, dbias, accumulate, ws)


def occ_gated_bwd(dY, X=None, W=None, Z=None, act: int = OCC_ACT_SILU, dX=None, dW=None,
                  dbias=None, accumulate: bool = False, ws=None, stream=None) -> None:
    """Gradients of occ_gated_fwd (W, dW and dbias hold both projections); as
    occ_linear_bwd, with Z = [G U] always needed."""
    if stream is not None:
        return _on(stream, occ_gated_bwd, dY, X, W, Z, act, dX, dW, dbias, accumulate, ws)
    _layer_bwd("occ_gated_bwd", True, dY, X, W, Z, act, dX, dW, dbias, accumulate, ws)


# ----------------------------------------------------------------------------
# layers of experts
# ----------------------------------------------------------------------------
class Route(NamedTuple):
    """The experts of every token and the plan of their rows (occ_route_fwd)."""
    index: Any     # tokens x k int32: the experts chosen, -1: none
    weights: Any   # tokens x k float32
    offsets: Any   # experts + 1 int32: where each expert's rows begin, and their number
    order: Any     # tokens k int32: the entries (token k + j), expert by expert
    slots: Any     # tokens x k int32: each entry's place in order, -1: none


def _made(name: str, result):
    """What a native call made, its status checked."""
    if result[0]:
        raise OccError(name, result[0])
    return result[1:]


def occ_route_fwd(logits, k: int, renorm: bool = True, route=None, ws=None, stream=None) -> Route:
    """The k largest logits of each token (tokens x experts, float32 or bfloat16),
    their softmax weights (renorm: among the chosen; else over all the experts)
    and the plan of the experts' rows.  route: the tensors to write to."""
    if stream is not None:
        return _on(stream, occ_route_fwd, logits, k, renorm, route, ws)
    out = (None,) * 5 if route is None else route
    return Route(*_made("occ_route_fwd", (_layers_module or _layers()).route_forward(
        logits, k, bool(renorm), *out, ws)))


def occ_route_bwd(dweights, logits, route, renorm: bool = True, dlogits=None, stream=None):
    """Gradient of the logits from that of the weights (float32, tokens x k);
    dlogits may be logits itself."""
    if stream is not None:
        return _on(stream, occ_route_bwd, dweights, logits, route, renorm, dlogits)
    return _made("occ_route_bwd", (_layers_module or _layers()).route_backward(
        dweights, logits, route.index, route.weights, bool(renorm), dlogits))[0]


def occ_dispatch(X, route, Xs=None, flags=None, stream=None):
    """Xs: the tokens' rows of X in the order of the experts (route.order).  Rows
    behind the last expert's are left alone.  Its gradient is occ_combine of dXs
    without weights.  flags, here and in occ_combine and its backward pass: an int32
    word that takes OCC_F_BAD_ROWS where an entry or a place is out of range."""
    if stream is not None:
        return _on(stream, occ_dispatch, X, route, Xs, flags)
    return _made("occ_dispatch", (_layers_module or _layers()).dispatch(
        X, route.offsets, route.order, route.slots, Xs, flags))[0]


def occ_combine(Ys, route, weights=None, R=None, Y=None, flags=None, stream=None):
    """Y: for each token the sum of its experts' rows of Ys, times `weights`
    (float32, tokens x k) if given, and R.  R may be Y."""
    if stream is not None:
        return _on(stream, occ_combine, Ys, route, weights, R, Y, flags)
    return _made("occ_combine", (_layers_module or _layers()).combine(
        Ys, route.slots, weights, R, Y, flags))[0]


def occ_combine_bwd(dY, Ys, route, weights=None, dYs=None, dweights=None, flags=None, stream=None):
    """(dYs, dweights) of occ_combine; Ys None: dYs alone.  The gradient of R is
    dY itself."""
    if stream is not None:
        return _on(stream, occ_combine_bwd, dY, Ys, route, weights, dYs, dweights, flags)
    return _made("occ_combine_bwd", (_layers_module or _layers()).combine_backward(
        dY, Ys, route.order, route.slots, weights, dYs, dweights, flags))


def _experts_fwd(name: str, gated: bool, X, W, offsets, bias, act, R, Y, Z, flags, ws):
    if Y is None:
        if X.dim() != 2 or W.dim() != 3:
            raise ValueError("X must be 2-D and W 3-D")
        Y = X.new_empty((X.shape[0], W.shape[1] // 2 if gated else W.shape[1]))
    status = (_layers_module or _layers()).experts_forward(gated, X, W, offsets, bias, act, R, Y,
                                                           Z, flags, ws)
    if status:
        raise OccError(name, status)
    return Y


def occ_experts_linear_fwd(X, W, offsets, bias=None, act: int = OCC_ACT_NONE, R=None, Y=None,
                           Z=None, flags=None, ws=None, stream=None):
    """occ_linear_fwd with a weight (experts x out x in) and bias (experts x out) of
    each expert, whose rows of X, R, Y and Z offsets bounds (int32, experts + 1,
    on the GPU).  flags: an int32 word that takes OCC_F_BAD_ROWS where offsets
    fit no plan.  Rows that belong to no expert are left alone.  Returns Y."""
    if stream is not None:
        return _on(stream, occ_experts_linear_fwd, X, W, offsets, bias, act, R, Y, Z, flags, ws)
    return _experts_fwd("occ_experts_linear_fwd", False, X, W, offsets, bias, act, R, Y, Z, flags,
                        ws)


def occ_experts_gated_fwd(X, W, offsets, bias=None, act: int = OCC_ACT_SILU, R=None, Y=None,
                          Z=None, flags=None, ws=None, stream=None):
    """occ_gated_fwd with a weight (experts x 2 out x in) of each expert; as
    occ_experts_linear_fwd."""
    if stream is not None:
        return _on(stream, occ_experts_gated_fwd, X, W, offsets, bias, act, R, Y, Z, flags, ws)
    return _experts_fwd("occ_experts_gated_fwd", True, X, W, offsets, bias, act, R, Y, Z, flags, ws)


def _experts_bwd(name: str, gated: bool, dY, offsets, X, W, Z, act, dX, dW, dbias, accumulate,
                 flags, ws):
    status = (_layers_module or _layers()).experts_backward(
        gated, dY, X, W, offsets, Z, act, dX, dW, dbias, bool(accumulate), flags, ws)
    if status:
        raise OccError(name, status)


def occ_experts_linear_bwd(dY, offsets, X=None, W=None, Z=None, act: int = OCC_ACT_NONE, dX=None,
                           dW=None, dbias=None, accumulate: bool = False, flags=None, ws=None,
                           stream=None) -> None:
    """Gradients of occ_experts_linear_fwd, each made if a tensor is given for it;
    as occ_linear_bwd.  An expert without rows has zeros in dW and dbias."""
    if stream is not None:
        return _on(stream, occ_experts_linear_bwd, dY, offsets, X, W, Z, act, dX, dW, dbias,
                   accumulate, flags, ws)
    _experts_bwd("occ_experts_linear_bwd", False, dY, offsets, X, W, Z, act, dX, dW, dbias,
                 accumulate, flags, ws)


def occ_experts_gated_bwd(dY, offsets, X=None, W=None, Z=None, act: int = OCC_ACT_SILU, dX=None,
                          dW=None, dbias=None, accumulate: bool = False, flags=None, ws=None,
                          stream=None) -> None:
    """Gradients of occ_experts_gated_fwd; as occ_gated_bwd."""
    if stream is not None:
        return _on(stream, occ_experts_gated_bwd, dY, offsets, X, W, Z, act, dX, dW, dbias,
                   accumulate, flags, ws)
    _experts_bwd("occ_experts_gated_bwd", True, dY, offsets, X, W, Z, act, dX, dW, dbias,
                 accumulate, flags, ws)


# ----------------------------------------------------------------------------
# loss
# ----------------------------------------------------------------------------
def occ_distill_fwd(S, index, teacher, temperature: float = 1.0, alpha: float = 1.0, labels=None,
                    scale=None, loss=None, lse=None, dS=None, flags=None, stream=None):
    """The loss (float32, one value a token) of logits S (tokens x vocab, float32 or
    bfloat16) against the teacher's top logits (tokens x k, float32 or bfloat16)
    at columns `index` (int32; a negative one is masked), alpha of it, and against
    labels (int32; a negative one is none), 1 - alpha.  scale: a factor for each
    token.  dS, if given, receives the gradient of the sum of the losses in the
    same pass (it may be S); lse (float32, tokens x 2) what occ_distill_bwd needs.
    flags: an int32 word that takes OCC_F_BAD_ROWS where a column is none of S's.
    temperature: above 0, its square a normal float32."""
    if stream is not None:
        return _on(stream, occ_distill_fwd, S, index, teacher, temperature, alpha, labels, scale,
                   loss, lse, dS, flags)
    return _made("occ_distill_fwd", (_layers_module or _layers()).distill(
        False, S, index, teacher, labels, scale, temperature, alpha, loss, lse, dS, flags))[0]


def occ_distill_bwd(S, index, teacher, lse, temperature: float = 1.0, alpha: float = 1.0,
                    labels=None, scale=None, dS=None, flags=None, stream=None):
    """The gradient dS of occ_distill_fwd's losses from the lse that it stored.
    scale: the forward's, times the gradient of each loss.  dS may be S."""
    if stream is not None:
        return _on(stream, occ_distill_bwd, S, index, teacher, lse, temperature, alpha, labels,
                   scale, dS, flags)
    return _made("occ_distill_bwd", (_layers_module or _layers()).distill(
        True, S, index, teacher, labels, scale, temperature, alpha, None, lse, dS, flags))[1]


def make_param(W, m, v, G=None, P=None, Q=None, W16=None, m_scale=None, v_scale=None,
               decay: float = 0.0) -> occ_param_t:
    """One tensor of occ_adamw_step: float32 W (a matrix, or a vector), its
    gradient G (float32 or bfloat16) or the factors P and Q of one, and its
    moments: float32, or float8_e4m3fn / uint8 codes with their scales.  The
    result holds their addresses, and the tensors themselves so that they live
    as long as it does."""
    torch = _torch()
    shape = (1, W.shape[0]) if W.dim() == 1 else tuple(W.shape)
    if len(shape) != 2:
        raise ValueError("W must be 1-D or 2-D")
    rows, cols = shape

    def whole(t, name, of, *dtypes):   # flat, or a matrix of this shape
        if t is None:
            return None
        n = of[0] * of[1]
        if t.dtype not in dtypes:
            raise TypeError(f"{name} must be {' or '.join(map(str, dtypes))}")
        if t.numel() != n or not t.is_contiguous():
            raise ValueError(f"{name} must hold {n} contiguous values")
        if t.dim() == 2 and 1 not in t.shape and tuple(t.shape) != of:
            raise ValueError(f"{name} must be {of[0]} x {of[1]}")
        return t.data_ptr()

    given = {"W": W, "m": m, "v": v, "G": G, "P": P, "Q": Q, "W16": W16, "m_scale": m_scale,
             "v_scale": v_scale}
    a = occ_param_t()
    a.rows, a.cols = rows, cols
    a.W = whole(W, "W", shape, torch.float32)
    a.W16 = whole(W16, "W16", shape, torch.bfloat16)
    if G is not None:
        if P is not None or Q is not None:
            raise ValueError("give G, or P and Q")
        G2 = G.reshape(1, -1) if G.dim() == 1 and G.is_contiguous() else G
        if tuple(G2.shape) != shape:
            raise ValueError(f"G must be {rows} x {cols}")
        a.G, a.ldg, a.g_dtype = G2.data_ptr(), _ld(G2, "G"), _mdtype(G2)
    elif P is not None and Q is not None:
        if P.dim() != 2 or Q.dim() != 2 or P.shape[0] != rows or Q.shape[0] != cols \
                or P.shape[1] != Q.shape[1]:
            raise ValueError("P must be rows x rank and Q cols x rank")
        a.rank = P.shape[1]
        a.P = whole(P, "P", (rows, a.rank), torch.float32)
        a.Q = whole(Q, "Q", (cols, a.rank), torch.float32)
    else:
        raise ValueError("give G, or P and Q")
    codes = (torch.float8_e4m3fn, torch.uint8)
    a.state_bits = 8 if m.dtype in codes else 32
    kinds = codes if a.state_bits == 8 else (torch.float32,)
    a.m, a.v = whole(m, "m", shape, *kinds), whole(v, "v", shape, *kinds)
    if a.state_bits == 8:
        if m_scale is None or v_scale is None:
            raise ValueError("8-bit moments need m_scale and v_scale")
        runs = (rows, -(-cols // OCC_SCALE_RUN))
        a.m_scale = whole(m_scale, "m_scale", runs, torch.float32)
        a.v_scale = whole(v_scale, "v_scale", runs, torch.float32)
    a.decay = float(decay)
    for name, t in given.items():
        if t is not None and t.device != W.device:
            raise ValueError(f"{name} lies on another device than W")
    if not W.is_cuda:
        raise ValueError("the tensors must lie on a GPU")
    a._tensors = tuple(given.values())   # they live as long as their addresses are held
    return a


def make_params(params):
    """The array occ_adamw_step takes, made once.  It keeps the tensors alive:
    a tensor replaced in the program needs a new array."""
    items = list(params)
    array = (occ_param_t * len(items))(*items)
    array._params = items   # the structures are copied, what they keep is not
    devices = {p._tensors[0].device for p in items if hasattr(p, "_tensors")}
    if len(devices) > 1:
        raise ValueError("the tensors lie on different GPUs")
    array._device = devices.pop() if devices else None
    return array


def occ_adamw_step(params, lr: float, step: int, beta1: float = 0.9, beta2: float = 0.95,
                   eps: float = 1e-8, seed: int = 0, grad_scale=None, flags=None,
                   stream=None) -> None:
    """AdamW over every tensor of `params` (make_params, or a sequence of
    make_param); see occ_adamw_step in include/optcc.h.  grad_scale: float32
    CUDA tensor of one value; flags: int32 CUDA tensor of one value."""
    if not isinstance(params, ctypes.Array):
        params = make_params(params)
    device = getattr(params, "_device", None)   # None: structures of addresses alone
    for name, t in (("grad_scale", grad_scale), ("flags", flags)):
        if t is None:
            continue
        if not t.is_cuda:
            raise ValueError(f"{name} must lie on a GPU")
        if device is not None and t.device != device:
            raise ValueError(f"{name} lies on another device than the tensors")
    h = occ_adamw_t(lr, beta1, beta2, eps, step, seed & 0xFFFFFFFF, 0,
                    None if grad_scale is None else _vec(grad_scale, "grad_scale", 1), None)
    if flags is not None:
        if flags.numel() != 1 or flags.element_size() != 4:
            raise ValueError("flags must be one 32-bit word")
        h.flags = flags.data_ptr()
    cuda = _torch().cuda
    # a default stream's handle is null: it is the current GPU's
    other = device is not None and device.index != cuda.current_device()
    with cuda.device(device) if other else contextlib.nullcontext():
        status = lib().occ_adamw_step(params, len(params), ctypes.byref(h), _stream(stream))
    _check("occ_adamw_step", status)


def occ_profile_begin() -> None:
    _check("occ_profile_begin", lib().occ_profile_begin())


def occ_profile_end(max_kernels: int = 64) -> dict:
    """{kernel name: (launches, total_ms)} recorded since occ_profile_begin."""
    buf = (occ_kernel_time_t * max_kernels)()
    n = ctypes.c_int(0)
    _check("occ_profile_end", lib().occ_profile_end(buf, max_kernels, ctypes.byref(n)))
    return {buf[i].name.decode(): (int(buf[i].launches), float(buf[i].total_ms))
            for i in range(min(n.value, max_kernels))}
