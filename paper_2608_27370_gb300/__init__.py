"""GB300 (sm_103a) FP8 linear-layer training path of Puro-2B.

Python binding of ``libpuro_fp8.so`` (C ABI in ``include/puro_fp8.h``).
Every function here is argument marshalling only: it checks that the torch
tensors it is handed are CUDA, contiguous and of the right dtype, and passes
their device pointers, the sizes and the current CUDA stream to the library
entry point of the same name.  The calls of a training step do this in native
code (``csrc/binding.cpp``) for ordinary arguments; anything else it hands
back, and the ctypes path below it checks the arguments one by one (as every
call does where that module was compiled for another torch).  All
arithmetic runs in the library's CUDA kernels.  There is no fallback: if the
library is missing, every call raises.

The method (paper section "FP8 Mixed-Precision Training"; appendix
"Production Training Details", paragraph "FP8 implementation pipeline"):
E4M3 operands for all three GEMMs of every linear layer, power-of-two scales
computed online for 1x128 groups along the reduction dimension (activations
and activation gradients) or 128x128 blocks (weights), FP32 accumulation and
BF16 output.
"""
from __future__ import annotations

import ctypes
import importlib.machinery
import importlib.util
import os
import warnings
from dataclasses import dataclass
from typing import Optional

import torch

from . import _build

E4M3, E5M2 = 0, 1
SCALE_TENSOR, SCALE_BLOCK = 0, 1
ROLE_ACT, ROLE_WEIGHT = 0, 1
ACT_NONE, ACT_RELU, ACT_SILU, ACT_GELU, ACT_GELU_TANH = range(5)
ROPE_NONE, ROPE_LINEAR, ROPE_BASE, ROPE_TURNS, ROPE_INDEX = range(5)

PURO_OK = 0
PURO_ERR_INVALID_ARG = 1
PURO_ERR_UNSUPPORTED = 2
PURO_ERR_CUDA = 3
PURO_ERR_TIMEOUT = 4

LIB_PATH = _build.LIB
HEADER_PATH = os.path.join(_build.INCLUDE, "puro_fp8.h")


class PuroError(RuntimeError):
    def __init__(self, fn: str, status: int):
        self.status = status
        names = {1: "PURO_ERR_INVALID_ARG", 2: "PURO_ERR_UNSUPPORTED", 3: "PURO_ERR_CUDA", 4: "PURO_ERR_TIMEOUT"}
        super().__init__(f"{fn} returned {names.get(status, status)}")


class puro_fp8_tensor_t(ctypes.Structure):
    """Mirror of the C struct puro_fp8_tensor_t."""
    _fields_ = [
        ("data", ctypes.c_void_p),
        ("scale", ctypes.c_void_p),
        ("rows", ctypes.c_int64),
        ("red", ctypes.c_int64),
        ("fmt", ctypes.c_int32),
        ("scaling", ctypes.c_int32),
        ("role", ctypes.c_int32),
        ("reserved", ctypes.c_int32),
    ]


_P = ctypes.c_void_p
_I64 = ctypes.c_int64
_I32 = ctypes.c_int32
_SIGNATURES = {
    "puro_fp8_amax": (_I32, [_P, _I64, _I64, _P, _P]),
    "puro_fp8_quantize": (_I32, [_P, _I64, _I64, _I32, _I32, _I32, _P, _P, _P, _P, _P, _P, _P]),
    "puro_fp8_quantize_rmsnorm": (_I32, [_P, _I64, _I64, _P, ctypes.c_float, _I32, _P, _P, _P, _P, _P, _P, _P, _P]),
    "puro_rmsnorm_bf16": (_I32, [_P, _I64, _I64, _P, ctypes.c_float, _P, _P, _P]),
    "puro_fp8_quantize_swiglu": (_I32, [_P, _P, _I64, _I64, _I64, _I32, _P, _P, _P, _P, _P, _P, _P]),
    "puro_muonh_workspace_size": (ctypes.c_size_t, [_I64]),
    "puro_muonh_reduce": (_I32, [_P, _P, _I64, _P, _P, ctypes.c_size_t, _P]),
    "puro_muonh_apply": (_I32, [_P, _P, _I64, _P, ctypes.c_double, ctypes.c_double, _P, _P]),
    "puro_muonh_step": (_I32, [_P, _P, _I64, ctypes.c_double, ctypes.c_double, _P, _P, ctypes.c_size_t, _P, _P]),
    "puro_muonh_grouped_workspace_size": (ctypes.c_size_t, [_P, _I32]),
    "puro_muonh_step_grouped": (_I32, [_P, _I32, ctypes.c_double, _P, _P, ctypes.c_size_t, _P]),
    "puro_muon_direction_workspace_size": (ctypes.c_size_t, [_P, _I32]),
    "puro_muon_direction_grouped": (_I32, [_P, _I32, ctypes.c_double, _I32, _P, _I32, _P, ctypes.c_size_t, _P, _P]),
    "puro_swiglu_bf16": (_I32, [_P, _P, _I64, _I64, _I64, _P, _P]),
    "puro_fp8_linear_fprop": (_I32, [_P, _P, _P, _P, ctypes.c_size_t, _P, _P]),
    "puro_fp8_linear_dgrad": (_I32, [_P, _P, _P, _P, ctypes.c_size_t, _P, _P]),
    "puro_fp8_linear_wgrad": (_I32, [_P, _P, _P, _P, ctypes.c_size_t, _P, _P]),
    "puro_fp8_linear_dgrad_quantize": (_I32, [_P, _P, _I32, _P, _P, _P, _P, _P, _P, _P]),
    "puro_fp8_linear_backward": (_I32, [_P, _P, _P, _P, _P, _P, _P, ctypes.c_size_t, _P, _P]),
    "puro_fp8_quantize_weights": (_I32, [_P, _I32, _I32, _P, _P]),
    "puro_fp8_linear_wgrad_main_grad": (_I32, [_P, _P, _P, _P, ctypes.c_size_t, _P, _P]),
    "puro_fp8_linear_wgrad_noalloc": (_I32, [_P, _P, _P, _P, _P]),
    "puro_fp8_workspace_size": (ctypes.c_size_t, [_I64, _I64, _I64]),
    "puro_fp8_linear_backward_launches": (_I32, [_I64, _I64, _I64, ctypes.c_size_t]),
    "puro_fp8_scale_bytes": (ctypes.c_size_t, [_I64, _I64]),
    "puro_fp8_get_status": (_I32, [_P, _P, _P]),
    "puro_bf16_linear_fprop": (_I32, [_P, _P, _P, _I64, _I64, _I64, _P, _P]),
    "puro_bf16_linear_dgrad": (_I32, [_P, _P, _P, _I64, _I64, _I64, _P, _P]),
    "puro_bf16_linear_wgrad": (_I32, [_P, _P, _P, _I64, _I64, _I64, _P, _P]),
    "puro_fp8_linear_fprop_epilogue": (_I32, [_P, _P, _P, _I32, _P, _I64, _P, _P, _P, ctypes.c_size_t, _P, _P]),
    "puro_bf16_linear_fprop_epilogue": (_I32, [_P, _P, _I64, _I64, _I64, _P, _I32, _P, _I64, _P, _P, _P, _P]),
    "puro_fp8_gated_fprop": (_I32, [_P, _P, _I32, _I32, _P, _P, _P, _P, _P, _P, _P, _P]),
    "puro_bf16_gated_fprop": (_I32, [_P, _P, _I64, _I64, _I64, _I32, _P, _P, _P, _P]),
    "puro_fp8_quantize_act_backward": (_I32, [_P, _P, _I64, _I64, _I32, _I32, _P, _P, _P, ctypes.c_size_t, _P, _P, _P, _P, _P,
                                              _P]),
    "puro_act_backward_bf16": (_I32, [_P, _P, _I64, _I64, _I32, _P, _P, _P, ctypes.c_size_t, _P]),
    "puro_act_backward_workspace_size": (ctypes.c_size_t, [_I64, _I64]),
    "puro_fp8_quantize_gated_backward": (_I32, [_P, _P, _P, _I64, _I64, _I64, _I32, _I32, _P, _P, _P, _P, _P, _P, _P]),
    "puro_gated_backward_bf16": (_I32, [_P, _P, _P, _I64, _I64, _I64, _I32, _P, _P]),
    "puro_qk_norm_rope": (_I32, [_P, _P, _I64, _I32, _P, _P, ctypes.c_float, _P, _P, _I64, _I32, _I32, _P, _P, _P, _P, _P,
                                 _P]),
    "puro_qk_norm_rope_backward": (_I32, [_P, _P, _P, _P, _P, _I64, _I32, _P, _P, _P, _P, _I64, _I32, _I32, _P, _P, _P, _P,
                                          _P, _P, ctypes.c_size_t, _P, _P]),
    "puro_qk_norm_rope_workspace_size": (ctypes.c_size_t, [_I64, _I32, _I32, _I32]),
    "puro_rope_frequencies": (_I32, [_I32, ctypes.c_double, _I32, ctypes.c_double, _I64, ctypes.c_double, ctypes.c_double, _P]),
    "puro_rope_tables": (_I32, [_P, _I32, ctypes.c_float, _I64, _I64, _P, _P, _P]),
    "puro_rope": (_I32, [_P, _P, _I64, _I32, _P, _I32, ctypes.c_float, _I32, _P, _P, _P, _P]),
    "puro_rope_backward": (_I32, [_P, _P, _I64, _I32, _P, _I32, ctypes.c_float, _I32, _P, _P, _P, _P]),
    "puro_set_wait_timeout_ns": (None, [ctypes.c_uint64]),
    "puro_set_gemm_tile_n": (ctypes.c_int, [ctypes.c_int32]),
    "puro_status_string": (ctypes.c_char_p, [_I32]),
}

_lib = None


def load_library(path: Optional[str] = None):
    """Load libpuro_fp8.so (built by ``__graft_entry__.build()``); raises if absent."""
    global _lib
    if _lib is not None and path is None:
        return _lib
    p = path or LIB_PATH
    if not os.path.exists(p):
        raise RuntimeError(
            f"libpuro_fp8.so not found at {p}: build it with `python -c 'import __graft_entry__ as g; g.build()'`")
    lib = ctypes.CDLL(p)
    for name, (res, args) in _SIGNATURES.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    if path is None:
        _lib = lib
    return lib


_native = None


class _CtypesOnly:
    """Stands in for the native module: hands every call back."""

    def __getattr__(self, name):
        return lambda *args: None


def _load_native():
    """The native marshalling module, calling the library that load_library() returns.  Without
    one for this torch and interpreter every call takes its ctypes path."""
    global _native
    lib = load_library()
    name = __name__ + "._native"
    loader = importlib.machinery.ExtensionFileLoader(name, _build.NATIVE)
    try:
        module = importlib.util.module_from_spec(importlib.util.spec_from_loader(name, loader))
        loader.exec_module(module)
        made_for = getattr(module, "native_for", "another version")
        if made_for != _build.native_for():
            raise ImportError(f"it was compiled for {made_for}, this is {_build.native_for()}")
    except ImportError as e:
        warnings.warn(f"calls are marshalled by ctypes (9 us more each), {_build.NATIVE} cannot be used: {e}; rebuild "
                      "with `python -c 'import __graft_entry__ as g; g.build()'`", stacklevel=3)
        _native = _CtypesOnly()
        return _native
    module.set_operand_type(FP8Operand)
    module.set_library({n: ctypes.cast(getattr(lib, n), ctypes.c_void_p).value for n in _SIGNATURES})
    _native = module
    return module


def _check(fn: str, status: int) -> None:
    if status != PURO_OK:
        raise PuroError(fn, status)


def _stream(stream) -> int:
    if stream is None:
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, torch.cuda.Stream):
        return stream.cuda_stream
    return int(stream)


def _ptr(t: Optional[torch.Tensor], dtype=None, name: str = "tensor") -> Optional[int]:
    if t is None:
        return None
    if t.numel() == 0:
        return t.data_ptr() or None
    if not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if dtype is not None and t.dtype not in (dtype if isinstance(dtype, tuple) else (dtype,)):
        raise ValueError(f"{name} has dtype {t.dtype}, expected {dtype}")
    return t.data_ptr()


def _sized(t: Optional[torch.Tensor], dtype, n: int, name: str) -> Optional[int]:
    if t is not None and t.numel() != n:
        raise ValueError(f"{name} has {t.numel()} values, expected {n}")
    return _ptr(t, dtype, name)


def _copies(q, scale, q_t, scale_t, rows: int, cols: int):
    """Pointers of an FP8 copy [rows, cols] and its transpose with their scale vectors."""
    u8 = torch.uint8

    def vectors(t, r, red, name):
        return _sized(t, u8, r * ((red // 128 + 3) // 4) * 4, name)

    return (_sized(q, u8, rows * cols, "q"), vectors(scale, rows, cols, "scale"), _sized(q_t, u8, rows * cols, "q_t"),
            vectors(scale_t, cols, rows, "scale_t"))


def _ws(workspace: Optional[torch.Tensor]):
    return _ptr(workspace, None, "workspace"), workspace.numel() * workspace.element_size() if workspace is not None else 0


def _same_shape(t: torch.Tensor, like: torch.Tensor, name: str) -> None:
    if t.shape != like.shape:
        raise ValueError(f"{name} is {tuple(t.shape)}, expected {tuple(like.shape)}")


def _rows_of(t: Optional[torch.Tensor], rows: int, cols: int, name: str):
    """Pointer and row stride of an optional bf16 [rows, cols] view with unit column stride."""
    if t is None:
        return None, cols
    if not t.is_cuda or t.dtype != torch.bfloat16 or tuple(t.shape) != (rows, cols):
        raise ValueError(f"{name} must be a bf16 CUDA tensor [{rows}, {cols}]")
    if t.numel() and t.stride(1) != 1:
        raise ValueError(f"{name} must have unit column stride")
    return t.data_ptr() or None, t.stride(0) if rows > 1 else cols


def _current_device() -> int:
    return torch.cuda.current_device()


def _on_current_device(*tensors) -> None:
    """Kernels are launched on the current device: every tensor has to be there.  (The native
    module looks only whether all are on one device, so one is looked at ahead of it.)"""
    here = _current_device()
    for t in tensors:
        if t is not None and t.is_cuda and t.get_device() != here:
            raise ValueError(f"a tensor is on cuda:{t.get_device()}, the current device is cuda:{here}")


# --------------------------------------------------------------------------
# Entry points (same names as the C ABI)
# --------------------------------------------------------------------------
def puro_fp8_amax(x: torch.Tensor, amax_bits: torch.Tensor, stream=None) -> None:
    st = (_native or _load_native()).puro_fp8_amax(x, amax_bits, stream)
    if st is not None:
        return _check("puro_fp8_amax", st)
    rows, cols = (x.shape[0], x.shape[1]) if x.dim() == 2 else (1, x.numel())
    st = load_library().puro_fp8_amax(_ptr(x, torch.bfloat16, "x"), rows, cols,
                                      _ptr(amax_bits, (torch.int32, torch.uint32), "amax_bits"), _stream(stream))
    _check("puro_fp8_amax", st)


def puro_fp8_quantize(x: torch.Tensor, fmt: int, scaling: int, role: int, amax_bits: Optional[torch.Tensor],
                      q: torch.Tensor, scale: torch.Tensor, q_t: Optional[torch.Tensor] = None,
                      scale_t: Optional[torch.Tensor] = None, dev_status: Optional[torch.Tensor] = None,
                      stream=None) -> None:
    st = (_native or _load_native()).puro_fp8_quantize(x, fmt, scaling, role, amax_bits, q, scale, q_t,
                                                    scale_t, dev_status, stream)
    if st is not None:
        return _check("puro_fp8_quantize", st)
    rows, cols = x.shape
    u8 = torch.uint8
    sdt = u8 if scaling == SCALE_BLOCK else torch.float32
    st = load_library().puro_fp8_quantize(
        _ptr(x, torch.bfloat16, "x"), rows, cols, fmt, scaling, role,
        _ptr(amax_bits, (torch.int32, torch.uint32), "amax_bits"), _ptr(q, u8, "q"), _ptr(scale, sdt, "scale"),
        _ptr(q_t, u8, "q_t"), _ptr(scale_t, sdt, "scale_t"), _ptr(dev_status, torch.int32, "dev_status"),
        _stream(stream))
    _check("puro_fp8_quantize", st)


def puro_fp8_quantize_rmsnorm(h: torch.Tensor, gamma: Optional[torch.Tensor], eps: float, fmt: int,
                              rstd: torch.Tensor, y: Optional[torch.Tensor], q: torch.Tensor, scale: torch.Tensor,
                              q_t: Optional[torch.Tensor] = None, scale_t: Optional[torch.Tensor] = None,
                              dev_status: Optional[torch.Tensor] = None, stream=None) -> None:
    """RMSNorm of the rows of h (bf16, optional bf16 gain) fused ahead of the
    blockwise activation quantiser: writes rstd (fp32 [rows]), optionally y
    (bf16), and the codes and scales as puro_fp8_quantize does."""
    st = (_native or _load_native()).puro_fp8_quantize_rmsnorm(h, gamma, eps, fmt, rstd, y, q, scale, q_t,
                                                            scale_t, dev_status, stream)
    if st is not None:
        return _check("puro_fp8_quantize_rmsnorm", st)
    rows, cols = h.shape
    u8 = torch.uint8
    st = load_library().puro_fp8_quantize_rmsnorm(
        _ptr(h, torch.bfloat16, "h"), rows, cols, _ptr(gamma, torch.bfloat16, "gamma"), float(eps), fmt,
        _ptr(rstd, torch.float32, "rstd"), _ptr(y, torch.bfloat16, "y"), _ptr(q, u8, "q"), _ptr(scale, u8, "scale"),
        _ptr(q_t, u8, "q_t"), _ptr(scale_t, u8, "scale_t"), _ptr(dev_status, torch.int32, "dev_status"),
        _stream(stream))
    _check("puro_fp8_quantize_rmsnorm", st)


def _gate_up(gate: torch.Tensor, up: torch.Tensor):
    """Pointers and the shared row stride of gate / up (bf16 [rows, cols]
    CUDA tensors with unit column stride, e.g. the halves of one output)."""
    for name, t in (("gate", gate), ("up", up)):
        if not t.is_cuda or t.dtype != torch.bfloat16 or t.dim() != 2:
            raise ValueError(f"{name} must be a 2-D bf16 CUDA tensor")
        if t.numel() and t.stride(1) != 1:
            raise ValueError(f"{name} must have unit column stride")
    if gate.shape != up.shape:
        raise ValueError("gate and up differ in shape")
    rows, cols = gate.shape
    ld = gate.stride(0) if rows > 1 else cols
    if rows > 1 and up.stride(0) != ld:
        raise ValueError("gate and up must share one row stride")
    return gate.data_ptr() or None, up.data_ptr() or None, rows, cols, ld


class puro_fp8_weight_t(ctypes.Structure):
    _fields_ = [("w", ctypes.c_void_p), ("rows", ctypes.c_int64), ("cols", ctypes.c_int64),
                ("q", ctypes.c_void_p), ("scale", ctypes.c_void_p), ("q_t", ctypes.c_void_p),
                ("scale_t", ctypes.c_void_p)]


def weight_table(entries):
    """The host table of puro_fp8_quantize_weights for a fixed list of
    (w bf16 [rows, cols], Quantized with rowwise [rows, cols] and optional
    colwise [cols, rows] operands): build it once and pass it to every call
    (the tensors must stay alive and in place)."""
    table = (puro_fp8_weight_t * max(1, len(entries)))()
    u8 = torch.uint8
    for i, (w, q) in enumerate(entries):
        col = q.colwise
        table[i] = puro_fp8_weight_t(_ptr(w, torch.bfloat16, "w"), w.shape[0], w.shape[1],
                                     _ptr(q.rowwise.data, u8, "q"), _ptr(q.rowwise.scale, u8, "scale"),
                                     _ptr(col.data, u8, "q_t") if col is not None else None,
                                     _ptr(col.scale, u8, "scale_t") if col is not None else None)
    table.count = len(entries)
    return table


def puro_fp8_quantize_weights(entries, fmt: int = E4M3, dev_status: Optional[torch.Tensor] = None,
                              stream=None) -> None:
    """Quantise many weights in 128x128 blocks in one call: entries is a list
    of (w, Quantized) pairs or a table from weight_table().  Same bytes as
    quantize(w, fmt, SCALE_BLOCK, ROLE_WEIGHT, out=q) for each."""
    table = entries if isinstance(entries, ctypes.Array) else weight_table(entries)
    st = (_native or _load_native()).puro_fp8_quantize_weights(ctypes.addressof(table), table.count, fmt, dev_status,
                                                               stream)
    if st is not None:
        return _check("puro_fp8_quantize_weights", st)
    st = load_library().puro_fp8_quantize_weights(table, table.count, fmt,
                                                  _ptr(dev_status, torch.int32, "dev_status"), _stream(stream))
    _check("puro_fp8_quantize_weights", st)


def puro_fp8_quantize_swiglu(gate: torch.Tensor, up: torch.Tensor, fmt: int, y: Optional[torch.Tensor],
                             q: torch.Tensor, scale: torch.Tensor, q_t: Optional[torch.Tensor] = None,
                             scale_t: Optional[torch.Tensor] = None, dev_status: Optional[torch.Tensor] = None,
                             stream=None) -> None:
    """SwiGLU (silu(gate) * up, bf16) fused ahead of the blockwise activation
    quantiser: writes the codes and scales as puro_fp8_quantize does, and y
    (bf16) only when given.  gate and up may be row-strided views."""
    st = (_native or _load_native()).puro_fp8_quantize_swiglu(gate, up, fmt, y, q, scale, q_t, scale_t,
                                                           dev_status, stream)
    if st is not None:
        return _check("puro_fp8_quantize_swiglu", st)
    g, u, rows, cols, ld = _gate_up(gate, up)
    u8 = torch.uint8
    st = load_library().puro_fp8_quantize_swiglu(
        g, u, rows, cols, ld, fmt, _ptr(y, torch.bfloat16, "y"), _ptr(q, u8, "q"), _ptr(scale, u8, "scale"),
        _ptr(q_t, u8, "q_t"), _ptr(scale_t, u8, "scale_t"), _ptr(dev_status, torch.int32, "dev_status"),
        _stream(stream))
    _check("puro_fp8_quantize_swiglu", st)


def puro_swiglu_bf16(gate: torch.Tensor, up: torch.Tensor, y: torch.Tensor, stream=None) -> None:
    g, u, rows, cols, ld = _gate_up(gate, up)
    st = load_library().puro_swiglu_bf16(g, u, rows, cols, ld, _ptr(y, torch.bfloat16, "y"), _stream(stream))
    _check("puro_swiglu_bf16", st)


def puro_muonh_workspace_size(n: int) -> int:
    return int(load_library().puro_muonh_workspace_size(n))


def puro_muonh_reduce(w: torch.Tensor, u: torch.Tensor, sums: torch.Tensor, workspace: torch.Tensor,
                      stream=None) -> None:
    """sums (fp64 [3], device) = {sum W^2, sum W u, sum u^2} of fp32 W and u."""
    if w.numel() != u.numel():
        raise ValueError("w and u differ in size")
    st = load_library().puro_muonh_reduce(_ptr(w, torch.float32, "w"), _ptr(u, torch.float32, "u"), w.numel(),
                                          _ptr(sums, torch.float64, "sums"), _ptr(workspace, None, "workspace"),
                                          workspace.numel() * workspace.element_size(), _stream(stream))
    _check("puro_muonh_reduce", st)


def puro_muonh_apply(w: torch.Tensor, u: torch.Tensor, sums: torch.Tensor, eta: float, radius: float,
                     w_bf16: Optional[torch.Tensor] = None, stream=None) -> None:
    if w.numel() != u.numel() or (w_bf16 is not None and w_bf16.numel() != w.numel()):
        raise ValueError("w, u and w_bf16 differ in size")
    st = load_library().puro_muonh_apply(_ptr(w, torch.float32, "w"), _ptr(u, torch.float32, "u"), w.numel(),
                                         _ptr(sums, torch.float64, "sums"), float(eta), float(radius),
                                         _ptr(w_bf16, torch.bfloat16, "w_bf16"), _stream(stream))
    _check("puro_muonh_apply", st)


def puro_muonh_step(w: torch.Tensor, u: torch.Tensor, eta: float, radius: float, sums: torch.Tensor,
                    workspace: torch.Tensor, w_bf16: Optional[torch.Tensor] = None, stream=None) -> None:
    """One MuonH hyperball update of the fp32 master weight w (in place)
    along the Muon direction u; optionally writes the bf16 copy."""
    if w.numel() != u.numel() or (w_bf16 is not None and w_bf16.numel() != w.numel()):
        raise ValueError("w, u and w_bf16 differ in size")
    st = load_library().puro_muonh_step(_ptr(w, torch.float32, "w"), _ptr(u, torch.float32, "u"), w.numel(),
                                        float(eta), float(radius), _ptr(sums, torch.float64, "sums"),
                                        _ptr(workspace, None, "workspace"),
                                        workspace.numel() * workspace.element_size(),
                                        _ptr(w_bf16, torch.bfloat16, "w_bf16"), _stream(stream))
    _check("puro_muonh_step", st)


class puro_muonh_matrix_t(ctypes.Structure):
    _fields_ = [("w", ctypes.c_void_p), ("u", ctypes.c_void_p), ("w_bf16", ctypes.c_void_p),
                ("n", ctypes.c_int64), ("radius", ctypes.c_double)]


def _muonh_table(mats):
    """ctypes array of descriptors from (w, u, w_bf16 or None, radius) tuples."""
    arr = (puro_muonh_matrix_t * max(1, len(mats)))()
    for i, (w, u, wb, r) in enumerate(mats):
        if w.numel() != u.numel() or (wb is not None and wb.numel() != w.numel()):
            raise ValueError(f"matrix {i}: w, u and w_bf16 differ in size")
        arr[i] = puro_muonh_matrix_t(_ptr(w, torch.float32, "w"), _ptr(u, torch.float32, "u"),
                                     _ptr(wb, torch.bfloat16, "w_bf16"), w.numel(), float(r))
    return arr


def puro_muonh_grouped_workspace_size(mats) -> int:
    return int(load_library().puro_muonh_grouped_workspace_size(_muonh_table(mats), len(mats)))


def puro_muonh_step_grouped(mats, eta: float, sums: torch.Tensor, workspace: torch.Tensor, stream=None) -> None:
    """The hyperball step for every (w, u, w_bf16 or None, radius) in mats;
    sums: fp64 [len(mats), 3] on the device."""
    table = _muonh_table(mats)
    st = load_library().puro_muonh_step_grouped(table, len(mats), float(eta), _ptr(sums, torch.float64, "sums"),
                                                _ptr(workspace, None, "workspace"),
                                                workspace.numel() * workspace.element_size(), _stream(stream))
    _check("puro_muonh_step_grouped", st)


MUON_STEPS = ((3.4445, -4.7750, 2.0315),) * 5  # Muon's Newton-Schulz coefficients


class puro_muon_matrix_t(ctypes.Structure):
    """Mirror of the C struct puro_muon_matrix_t."""
    _fields_ = [("grad", ctypes.c_void_p), ("momentum", ctypes.c_void_p), ("u", ctypes.c_void_p),
                ("rows", ctypes.c_int64), ("cols", ctypes.c_int64), ("grad_stride", ctypes.c_int64),
                ("u_stride", ctypes.c_int64), ("grad_type", ctypes.c_int32), ("u_type", ctypes.c_int32),
                ("reserved", ctypes.c_int64)]


def muon_table(mats):
    """The host table of puro_muon_direction_grouped for a fixed list of (grad,
    momentum or None, u): grad and u are bf16 or fp32 [rows, cols] with unit column
    stride, momentum is fp32 [rows, cols].  Build it once and pass it to every call
    (the tensors must stay alive and in place).  No momentum and no u may share memory
    with anything else of the list, but u may lie in its own grad."""
    table = (puro_muon_matrix_t * max(1, len(mats)))()
    types = {torch.bfloat16: 0, torch.float32: 1}
    table.tensors = []
    for i, (g, m, u) in enumerate(mats):
        for t, name in ((g, "grad"), (u, "u")):
            if not t.is_cuda or t.dtype not in types or t.dim() != 2 or t.shape != g.shape:
                raise ValueError(f"matrix {i}: {name} must be a bf16 or fp32 CUDA tensor {tuple(g.shape)}")
            if t.numel() and t.shape[1] > 1 and t.stride(1) != 1:
                raise ValueError(f"matrix {i}: {name} must have unit column stride")
        if m is not None and m.shape != g.shape:
            raise ValueError(f"matrix {i}: momentum is {tuple(m.shape)}, expected {tuple(g.shape)}")
        rows, cols = g.shape
        table[i] = puro_muon_matrix_t(g.data_ptr() or None, _ptr(m, torch.float32, "momentum"), u.data_ptr() or None, rows, cols,
                                      g.stride(0) if rows > 1 else cols, u.stride(0) if rows > 1 else cols, types[g.dtype],
                                      types[u.dtype], 0)
        table.tensors += [t for t in (g, m, u) if t is not None]
    table.count = len(mats)
    written = [t.data_ptr() for _, m, u in mats for t in (m, u) if t is not None and t.numel()]
    if len(set(written)) < len(written):
        raise ValueError("a momentum or u is there twice")
    devices = {t.get_device() for t in table.tensors if t.numel()}
    if len(devices) > 1:
        raise ValueError(f"the matrices are on several devices: {sorted(devices)}")
    table.device = devices.pop() if devices else None
    return table


def _muon_table(mats):
    return mats if isinstance(mats, ctypes.Array) else muon_table(mats)


def puro_muon_direction_workspace_size(mats) -> int:
    table = _muon_table(mats)
    return int(load_library().puro_muon_direction_workspace_size(table, table.count))


def puro_muon_direction_grouped(mats, workspace: torch.Tensor, momentum: float = 0.95, nesterov: bool = True,
                                coefficients=MUON_STEPS, dev_status: Optional[torch.Tensor] = None, stream=None) -> None:
    """The Muon direction u of every matrix: the momentum buffer takes the gradient,
    and its update, divided by its Frobenius norm, is orthogonalised by a
    Newton-Schulz step for each (a, b, c) of coefficients.  mats: a list of (grad,
    momentum or None, u) or a table from muon_table()."""
    table = _muon_table(mats)
    if table.device not in (None, _current_device()):
        raise ValueError(f"the matrices are on cuda:{table.device}, the current device is cuda:{_current_device()}")
    _on_current_device(workspace, dev_status)
    flat = [float(x) for step in coefficients for x in step]
    if any(len(step) != 3 for step in coefficients):
        raise ValueError("coefficients are triples (a, b, c)")
    st = load_library().puro_muon_direction_grouped(table, table.count, float(momentum), int(bool(nesterov)),
                                                    (ctypes.c_double * max(1, len(flat)))(*flat), len(coefficients),
                                                    *_ws(workspace), _ptr(dev_status, torch.int32, "dev_status"), _stream(stream))
    _check("puro_muon_direction_grouped", st)


def muonh_radius(w0: torch.Tensor) -> float:
    """R = ||W_0||_F (fp64, through puro_muonh_reduce; synchronises)."""
    sums = torch.empty(3, dtype=torch.float64, device=w0.device)
    ws = torch.empty(max(8, puro_muonh_workspace_size(w0.numel())), dtype=torch.uint8, device=w0.device)
    puro_muonh_reduce(w0, w0, sums, ws)
    return float(sums[0].sqrt().item())


def puro_rmsnorm_bf16(h: torch.Tensor, gamma: Optional[torch.Tensor], eps: float, rstd: torch.Tensor,
                      y: torch.Tensor, stream=None) -> None:
    """The same RMSNorm without the quantiser (rstd fp32, y bf16)."""
    rows, cols = h.shape
    st = load_library().puro_rmsnorm_bf16(_ptr(h, torch.bfloat16, "h"), rows, cols,
                                          _ptr(gamma, torch.bfloat16, "gamma"), float(eps),
                                          _ptr(rstd, torch.float32, "rstd"), _ptr(y, torch.bfloat16, "y"),
                                          _stream(stream))
    _check("puro_rmsnorm_bf16", st)


@dataclass
class FP8Operand:
    """A quantised GEMM operand: codes [rows, red] plus scales (torch tensors kept alive here)."""
    data: torch.Tensor
    scale: torch.Tensor
    fmt: int = E4M3
    scaling: int = SCALE_BLOCK
    role: int = ROLE_ACT

    @property
    def rows(self) -> int:
        return self.data.shape[0]

    @property
    def red(self) -> int:
        return self.data.shape[1]

    def as_c(self) -> puro_fp8_tensor_t:
        return puro_fp8_tensor_t(_ptr(self.data, torch.uint8, "data"), _ptr(self.scale, None, "scale"),
                                 self.data.shape[0], self.data.shape[1], self.fmt, self.scaling, self.role, 0)


def _gemm(name: str, a: FP8Operand, b: FP8Operand, out: torch.Tensor, workspace, dev_status, stream,
          out_dtype=torch.bfloat16) -> None:
    st = getattr(_native or _load_native(), name)(a, b, out, workspace, dev_status, stream)
    if st is not None:
        return _check(name, st)
    ca, cb = a.as_c(), b.as_c()
    ws_ptr = _ptr(workspace, None, "workspace")
    ws_bytes = workspace.numel() * workspace.element_size() if workspace is not None else 0
    fn = getattr(load_library(), name)
    st = fn(ctypes.byref(ca), ctypes.byref(cb), _ptr(out, out_dtype, "out"), ws_ptr, ws_bytes,
            _ptr(dev_status, torch.int32, "dev_status"), _stream(stream))
    _check(name, st)


def puro_fp8_linear_fprop(x: FP8Operand, w: FP8Operand, y: torch.Tensor, workspace=None, dev_status=None,
                          stream=None) -> None:
    """Y [M,N] = X [M,K] . W [N,K]^T."""
    _gemm("puro_fp8_linear_fprop", x, w, y, workspace, dev_status, stream)


def puro_fp8_linear_dgrad(dy: FP8Operand, w_t: FP8Operand, dx: torch.Tensor, workspace=None, dev_status=None,
                          stream=None) -> None:
    """dX [M,K] = dY [M,N] . W [N,K] (B operand = W^T [K,N])."""
    _gemm("puro_fp8_linear_dgrad", dy, w_t, dx, workspace, dev_status, stream)


def puro_fp8_linear_backward(dy: FP8Operand, w_t: FP8Operand, dx: torch.Tensor, dy_t: FP8Operand,
                             x_t: FP8Operand, dw: torch.Tensor, workspace=None, dev_status=None, stream=None) -> None:
    """dX [M,K] = dY . W and dW [N,K] = dY^T . X in one call (one grouped
    launch when both are unsplit block-scaled GEMMs)."""
    st = (_native or _load_native()).puro_fp8_linear_backward(dy, w_t, dx, dy_t, x_t, dw, workspace,
                                                           dev_status, stream)
    if st is not None:
        return _check("puro_fp8_linear_backward", st)
    c = [op.as_c() for op in (dy, w_t, dy_t, x_t)]
    ws_bytes = workspace.numel() * workspace.element_size() if workspace is not None else 0
    st = load_library().puro_fp8_linear_backward(
        ctypes.byref(c[0]), ctypes.byref(c[1]), _ptr(dx, torch.bfloat16, "dx"), ctypes.byref(c[2]),
        ctypes.byref(c[3]), _ptr(dw, torch.bfloat16, "dw"), _ptr(workspace, None, "workspace"), ws_bytes,
        _ptr(dev_status, torch.int32, "dev_status"), _stream(stream))
    _check("puro_fp8_linear_backward", st)


def puro_fp8_linear_dgrad_quantize(dy: FP8Operand, w_t: FP8Operand, fmt: int, dx: Optional[torch.Tensor],
                                   dxq: torch.Tensor, dxq_scale: torch.Tensor, dxq_t: Optional[torch.Tensor] = None,
                                   dxq_t_scale: Optional[torch.Tensor] = None, dev_status=None, stream=None) -> None:
    """dX [M,K] = dY [M,N] . W [N,K], rounded to BF16 and quantised in the
    GEMM's epilogue into the blockwise activation copies (dxq [M,K] with
    1x128 groups; dxq_t [K,M] with 128-row groups, optional); dx (bf16) is
    written only when given."""
    st = (_native or _load_native()).puro_fp8_linear_dgrad_quantize(dy, w_t, fmt, dx, dxq, dxq_scale, dxq_t,
                                                                 dxq_t_scale, dev_status, stream)
    if st is not None:
        return _check("puro_fp8_linear_dgrad_quantize", st)
    ca, cb = dy.as_c(), w_t.as_c()
    u8 = torch.uint8
    st = load_library().puro_fp8_linear_dgrad_quantize(
        ctypes.byref(ca), ctypes.byref(cb), fmt, _ptr(dx, torch.bfloat16, "dx"), _ptr(dxq, u8, "dxq"),
        _ptr(dxq_scale, u8, "dxq_scale"), _ptr(dxq_t, u8, "dxq_t"), _ptr(dxq_t_scale, u8, "dxq_t_scale"),
        _ptr(dev_status, torch.int32, "dev_status"), _stream(stream))
    _check("puro_fp8_linear_dgrad_quantize", st)


def puro_fp8_linear_wgrad(dy_t: FP8Operand, x_t: FP8Operand, dw: torch.Tensor, workspace=None, dev_status=None,
                          stream=None) -> None:
    """dW [N,K] = dY^T [N,M] . X [M,K] (operands dY^T [N,M], X^T [K,M])."""
    _gemm("puro_fp8_linear_wgrad", dy_t, x_t, dw, workspace, dev_status, stream)


def puro_fp8_linear_wgrad_main_grad(dy_t: FP8Operand, x_t: FP8Operand, main_grad: torch.Tensor, workspace=None,
                                    dev_status=None, stream=None) -> None:
    """main_grad [N,K] (FP32) += dY^T [N,M] . X [M,K]: the weight gradient
    accumulated in FP32 (operands dY^T [N,M], X^T [K,M])."""
    _gemm("puro_fp8_linear_wgrad_main_grad", dy_t, x_t, main_grad, workspace, dev_status, stream,
          out_dtype=torch.float32)


def puro_fp8_linear_wgrad_noalloc(dy_t: FP8Operand, x_t: FP8Operand, dw: torch.Tensor, dev_status=None,
                                  stream=None) -> None:
    """dW [N,K] = dY^T X without allocating and without caller scratch: for
    callers that cannot obtain device memory while running the backward
    pass.  The split-reduction scratch is a fixed 40 MiB array inside the
    library (see the header for the limits and ordering rules)."""
    ca, cb = dy_t.as_c(), x_t.as_c()
    st = load_library().puro_fp8_linear_wgrad_noalloc(ctypes.byref(ca), ctypes.byref(cb),
                                                      _ptr(dw, torch.bfloat16, "dw"),
                                                      _ptr(dev_status, torch.int32, "dev_status"), _stream(stream))
    _check("puro_fp8_linear_wgrad_noalloc", st)


def puro_fp8_linear_backward_launches(M: int, N: int, K: int, workspace_bytes: int) -> int:
    """Kernel launches of puro_fp8_linear_backward for block-scaled operands
    (M tokens, N out, K in features) given a workspace of that many bytes."""
    return int(load_library().puro_fp8_linear_backward_launches(M, N, K, workspace_bytes))


def puro_fp8_workspace_size(rows_out: int, cols_out: int, red: int) -> int:
    return int(load_library().puro_fp8_workspace_size(rows_out, cols_out, red))


def puro_fp8_get_status(dev_status: torch.Tensor, stream=None) -> int:
    out = ctypes.c_int32(0)
    st = load_library().puro_fp8_get_status(_ptr(dev_status, torch.int32, "dev_status"), ctypes.byref(out),
                                            _stream(stream))
    _check("puro_fp8_get_status", st)
    return out.value


def _bf16(name, a, b, out, M, N, K, dev_status, stream):
    st = getattr(_native or _load_native(), name)(a, b, out, M, N, K, dev_status, stream)
    if st is not None:
        return _check(name, st)
    fn = getattr(load_library(), name)
    st = fn(_ptr(a, torch.bfloat16, "a"), _ptr(b, torch.bfloat16, "b"), _ptr(out, torch.bfloat16, "out"), M, N, K,
            _ptr(dev_status, torch.int32, "dev_status"), _stream(stream))
    _check(name, st)


def puro_bf16_linear_fprop(x, w, y, M, N, K, dev_status=None, stream=None) -> None:
    _bf16("puro_bf16_linear_fprop", x, w, y, M, N, K, dev_status, stream)


def puro_bf16_linear_dgrad(dy, w_t, dx, M, N, K, dev_status=None, stream=None) -> None:
    _bf16("puro_bf16_linear_dgrad", dy, w_t, dx, M, N, K, dev_status, stream)


def puro_bf16_linear_wgrad(dy_t, x_t, dw, M, N, K, dev_status=None, stream=None) -> None:
    _bf16("puro_bf16_linear_wgrad", dy_t, x_t, dw, M, N, K, dev_status, stream)


# --------------------------------------------------------------------------
# Linears with an epilogue, the gated MLP's projections
# --------------------------------------------------------------------------
def puro_fp8_linear_fprop_epilogue(x: FP8Operand, w: FP8Operand, y: torch.Tensor, bias: Optional[torch.Tensor] = None,
                                   act: int = ACT_NONE, residual: Optional[torch.Tensor] = None,
                                   z: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                                   dev_status: Optional[torch.Tensor] = None, stream=None) -> None:
    """Y [M,N] = act(Z) + residual, Z = X [M,K] . W [N,K]^T + bias, all behind
    the product in the GEMM's epilogue.  bias bf16 [N]; residual bf16 [M,N]
    (rows may be strided; it may be y); z, when given, receives Z (bf16 [M,N])
    for the backward."""
    _on_current_device(x.data)
    st = (_native or _load_native()).puro_fp8_linear_fprop_epilogue(x, w, y, bias, act, residual, z, workspace, dev_status,
                                                                    stream)
    if st is not None:
        return _check("puro_fp8_linear_fprop_epilogue", st)
    _on_current_device(x.data, w.data, y, bias, residual, z, workspace, dev_status)
    cx, cw = x.as_c(), w.as_c()
    m, n, bf16 = cx.rows, cw.rows, torch.bfloat16
    res, ld = _rows_of(residual, m, n, "residual")
    st = load_library().puro_fp8_linear_fprop_epilogue(
        ctypes.byref(cx), ctypes.byref(cw), _sized(bias, bf16, n, "bias"), act, res, ld, _sized(z, bf16, m * n, "z"),
        _sized(y, bf16, m * n, "y"), *_ws(workspace), _ptr(dev_status, torch.int32, "dev_status"), _stream(stream))
    _check("puro_fp8_linear_fprop_epilogue", st)


def puro_bf16_linear_fprop_epilogue(x: torch.Tensor, w: torch.Tensor, y: torch.Tensor,
                                    bias: Optional[torch.Tensor] = None, act: int = ACT_NONE,
                                    residual: Optional[torch.Tensor] = None, z: Optional[torch.Tensor] = None,
                                    dev_status: Optional[torch.Tensor] = None, stream=None) -> None:
    """The same from BF16 x [M,K] and w [N,K]; any M, from a single token on."""
    _on_current_device(x)
    st = (_native or _load_native()).puro_bf16_linear_fprop_epilogue(x, w, y, bias, act, residual, z, dev_status, stream)
    if st is not None:
        return _check("puro_bf16_linear_fprop_epilogue", st)
    _on_current_device(x, w, y, bias, residual, z, dev_status)
    (m, k), n, bf16 = x.shape, w.shape[0], torch.bfloat16
    res, ld = _rows_of(residual, m, n, "residual")
    st = load_library().puro_bf16_linear_fprop_epilogue(
        _ptr(x, bf16, "x"), _sized(w, bf16, n * k, "w"), m, n, k, _sized(bias, bf16, n, "bias"), act, res, ld,
        _sized(z, bf16, m * n, "z"), _sized(y, bf16, m * n, "y"), _ptr(dev_status, torch.int32, "dev_status"),
        _stream(stream))
    _check("puro_bf16_linear_fprop_epilogue", st)


def puro_fp8_gated_fprop(x: FP8Operand, w: FP8Operand, act: int, fmt: int, gate_up: Optional[torch.Tensor],
                         h: Optional[torch.Tensor], hq: torch.Tensor, hq_scale: torch.Tensor,
                         hq_t: Optional[torch.Tensor] = None, hq_t_scale: Optional[torch.Tensor] = None,
                         dev_status: Optional[torch.Tensor] = None, stream=None) -> None:
    """The gated MLP's two projections, activation and product in one kernel:
    h = act(X . Wg^T) * (X . Wu^T), w = [Wg; Wu] [2F,K] quantised as one
    operand.  h is written as the FP8 copies that puro_fp8_quantize makes of
    it; gate_up (bf16 [M,2F], for the backward) and h (bf16 [M,F]) only when
    given."""
    _on_current_device(x.data)
    st = (_native or _load_native()).puro_fp8_gated_fprop(x, w, act, fmt, gate_up, h, hq, hq_scale, hq_t, hq_t_scale,
                                                          dev_status, stream)
    if st is not None:
        return _check("puro_fp8_gated_fprop", st)
    _on_current_device(x.data, w.data, gate_up, h, hq, hq_scale, hq_t, hq_t_scale, dev_status)
    cx, cw = x.as_c(), w.as_c()
    n, bf16 = cx.rows * (cw.rows // 2), torch.bfloat16
    st = load_library().puro_fp8_gated_fprop(
        ctypes.byref(cx), ctypes.byref(cw), act, fmt, _sized(gate_up, bf16, cx.rows * cw.rows, "gate_up"),
        _sized(h, bf16, n, "h"), *_copies(hq, hq_scale, hq_t, hq_t_scale, cx.rows, cw.rows // 2), _ptr(dev_status, torch.int32, "dev_status"), _stream(stream))
    _check("puro_fp8_gated_fprop", st)


def puro_bf16_gated_fprop(x: torch.Tensor, w: torch.Tensor, act: int, gate_up: Optional[torch.Tensor], h: torch.Tensor,
                          dev_status: Optional[torch.Tensor] = None, stream=None) -> None:
    """The same from BF16 x [M,K] and w [2F,K], h in BF16; any M, from a single token on."""
    _on_current_device(x)
    st = (_native or _load_native()).puro_bf16_gated_fprop(x, w, act, gate_up, h, dev_status, stream)
    if st is not None:
        return _check("puro_bf16_gated_fprop", st)
    _on_current_device(x, w, gate_up, h, dev_status)
    (m, k), n, bf16 = x.shape, w.shape[0], torch.bfloat16
    if n % 2:
        raise ValueError("w must hold the gate's and up's rows, as many of each")
    st = load_library().puro_bf16_gated_fprop(
        _ptr(x, bf16, "x"), _sized(w, bf16, n * k, "w"), m, n // 2, k, act, _sized(gate_up, bf16, m * n, "gate_up"),
        _sized(h, bf16, m * (n // 2), "h"), _ptr(dev_status, torch.int32, "dev_status"), _stream(stream))
    _check("puro_bf16_gated_fprop", st)


# --------------------------------------------------------------------------
# Backward of activations and gates
# --------------------------------------------------------------------------
def puro_act_backward_workspace_size(rows: int, cols: int) -> int:
    return int(load_library().puro_act_backward_workspace_size(rows, cols))


def puro_fp8_quantize_act_backward(dy: torch.Tensor, z: Optional[torch.Tensor], act: int, fmt: int,
                                   dz: Optional[torch.Tensor], dbias: Optional[torch.Tensor],
                                   workspace: Optional[torch.Tensor], q: torch.Tensor, scale: torch.Tensor,
                                   q_t: Optional[torch.Tensor] = None, scale_t: Optional[torch.Tensor] = None,
                                   dev_status: Optional[torch.Tensor] = None, stream=None) -> None:
    """dz = dy * act'(z) (bf16, z None without an activation) as the FP8 copies
    that puro_fp8_quantize makes of it, dbias (fp32 [cols]) its sum over the
    rows, through a workspace of puro_act_backward_workspace_size bytes; dz
    (bf16) is written only when given."""
    _on_current_device(dy)
    st = (_native or _load_native()).puro_fp8_quantize_act_backward(dy, z, act, fmt, dz, dbias, workspace, q, scale, q_t,
                                                                    scale_t, dev_status, stream)
    if st is not None:
        return _check("puro_fp8_quantize_act_backward", st)
    _on_current_device(dy, z, dz, dbias, workspace, q, scale, q_t, scale_t, dev_status)
    rows, cols = dy.shape
    n, bf16 = rows * cols, torch.bfloat16
    st = load_library().puro_fp8_quantize_act_backward(
        _ptr(dy, bf16, "dy"), _sized(z, bf16, n, "z"), rows, cols, act, fmt, _sized(dz, bf16, n, "dz"),
        _sized(dbias, torch.float32, cols, "dbias"), *_ws(workspace), *_copies(q, scale, q_t, scale_t, rows, cols),
        _ptr(dev_status, torch.int32, "dev_status"), _stream(stream))
    _check("puro_fp8_quantize_act_backward", st)


def puro_act_backward_bf16(dy: torch.Tensor, z: Optional[torch.Tensor], act: int, dz: Optional[torch.Tensor],
                           dbias: Optional[torch.Tensor], workspace: Optional[torch.Tensor] = None, stream=None) -> None:
    """The same without the quantiser: dz (bf16, may be dy) and dbias, each only when given."""
    _on_current_device(dy)
    st = (_native or _load_native()).puro_act_backward_bf16(dy, z, act, dz, dbias, workspace, stream)
    if st is not None:
        return _check("puro_act_backward_bf16", st)
    _on_current_device(dy, z, dz, dbias, workspace)
    rows, cols = dy.shape
    n, bf16 = rows * cols, torch.bfloat16
    st = load_library().puro_act_backward_bf16(
        _ptr(dy, bf16, "dy"), _sized(z, bf16, n, "z"), rows, cols, act, _sized(dz, bf16, n, "dz"),
        _sized(dbias, torch.float32, cols, "dbias"), *_ws(workspace), _stream(stream))
    _check("puro_act_backward_bf16", st)


def puro_fp8_quantize_gated_backward(dh: torch.Tensor, gate: torch.Tensor, up: torch.Tensor, act: int, fmt: int,
                                     dgate_up: Optional[torch.Tensor], q: torch.Tensor, scale: torch.Tensor,
                                     q_t: Optional[torch.Tensor] = None, scale_t: Optional[torch.Tensor] = None,
                                     dev_status: Optional[torch.Tensor] = None, stream=None) -> None:
    """[dgate, dup] = [dh * up * act'(gate), dh * act(gate)] (bf16 [rows, 2
    cols]) as the FP8 copies that puro_fp8_quantize makes of it: the output
    gradient of the fused gate/up linear, whose output gate and up are views
    of.  dgate_up (bf16) is written only when given."""
    _on_current_device(dh)
    st = (_native or _load_native()).puro_fp8_quantize_gated_backward(dh, gate, up, act, fmt, dgate_up, q, scale, q_t, scale_t,
                                                                      dev_status, stream)
    if st is not None:
        return _check("puro_fp8_quantize_gated_backward", st)
    _on_current_device(dh, gate, up, dgate_up, q, scale, q_t, scale_t, dev_status)
    g, u, rows, cols, ld = _gate_up(gate, up)
    n, bf16 = 2 * rows * cols, torch.bfloat16
    _same_shape(dh, gate, "dh")
    st = load_library().puro_fp8_quantize_gated_backward(
        _ptr(dh, bf16, "dh"), g, u, rows, cols, ld, act, fmt, _sized(dgate_up, bf16, n, "dgate_up"),
        *_copies(q, scale, q_t, scale_t, rows, 2 * cols), _ptr(dev_status, torch.int32, "dev_status"), _stream(stream))
    _check("puro_fp8_quantize_gated_backward", st)


def puro_gated_backward_bf16(dh: torch.Tensor, gate: torch.Tensor, up: torch.Tensor, act: int, dgate_up: torch.Tensor,
                             stream=None) -> None:
    """The same without the quantiser."""
    _on_current_device(dh)
    st = (_native or _load_native()).puro_gated_backward_bf16(dh, gate, up, act, dgate_up, stream)
    if st is not None:
        return _check("puro_gated_backward_bf16", st)
    _on_current_device(dh, gate, up, dgate_up)
    g, u, rows, cols, ld = _gate_up(gate, up)
    _same_shape(dh, gate, "dh")
    st = load_library().puro_gated_backward_bf16(_ptr(dh, torch.bfloat16, "dh"), g, u, rows, cols, ld, act,
                                                 _sized(dgate_up, torch.bfloat16, 2 * rows * cols, "dgate_up"),
                                                 _stream(stream))
    _check("puro_gated_backward_bf16", st)


# --------------------------------------------------------------------------
# Query and key norms with the position rotation
# --------------------------------------------------------------------------
class puro_heads_t(ctypes.Structure):
    """Mirror of the C struct puro_heads_t."""
    _fields_ = [("data", ctypes.c_void_p), ("token_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64),
                ("heads", ctypes.c_int32), ("reserved", ctypes.c_int32)]


def _heads(t: Optional[torch.Tensor], name: str, tokens: int, channels: int):
    """The C view of a bf16 [tokens, heads, channels] tensor with unit channel stride."""
    if t is None:
        return puro_heads_t()
    if not t.is_cuda or t.dtype != torch.bfloat16 or t.dim() != 3:
        raise ValueError(f"{name} must be a bf16 CUDA tensor [tokens, heads, head_dim]")
    if t.shape[0] != tokens or t.shape[2] != channels:
        raise ValueError(f"{name} is {tuple(t.shape)}, expected {tokens} tokens of {channels} channels")
    if t.numel() and t.stride(2) != 1:
        raise ValueError(f"{name} must have unit channel stride")
    return puro_heads_t(t.data_ptr() or None, t.stride(0) if t.shape[0] > 1 else 0, t.stride(1) if t.shape[1] > 1 else 0,
                        t.shape[1], 0)


def _tables(cos, sin):
    if cos is None and sin is None:
        return None, None, 0, 0
    if cos is None or sin is None or cos.dim() != 2 or cos.shape != sin.shape:
        raise ValueError("cos and sin must be two tables [positions, rot_dim / 2] of one shape")
    return (_ptr(cos, torch.float32, "cos"), _ptr(sin, torch.float32, "sin"), cos.shape[0], 2 * cos.shape[1])


def puro_qk_norm_rope(q: Optional[torch.Tensor], k: Optional[torch.Tensor], q_gain: Optional[torch.Tensor],
                      k_gain: Optional[torch.Tensor], eps: float, cos: Optional[torch.Tensor],
                      sin: Optional[torch.Tensor], positions: Optional[torch.Tensor], interleaved: bool,
                      q_out: Optional[torch.Tensor], k_out: Optional[torch.Tensor], rstd: Optional[torch.Tensor] = None,
                      dev_status: Optional[torch.Tensor] = None, stream=None) -> None:
    """RMSNorm of each query and key head (bf16 [tokens, heads, head_dim]
    views, for instance of one qkv output; optional bf16 gains) and the
    rotation by the tokens' positions (fp32 tables cos and sin [positions,
    rot_dim / 2], None for the norm alone) in one pass: q_out, k_out (which may
    be q and k) and rstd (fp32 [tokens, q heads + k heads]) for the backward.
    positions: int32 [tokens], None for 0, 1, ...; a negative one marks a
    padding row, whose output is zero."""
    _on_current_device(q if q is not None else k)
    st = (_native or _load_native()).puro_qk_norm_rope(q, k, q_gain, k_gain, eps, cos, sin, positions, interleaved, q_out,
                                                       k_out, rstd, dev_status, stream)
    if st is not None:
        return _check("puro_qk_norm_rope", st)
    _on_current_device(q, k, q_gain, k_gain, cos, sin, positions, q_out, k_out, rstd, dev_status)
    some = q if q is not None else k
    if some is None or some.dim() != 3:
        raise ValueError("q or k must be a bf16 CUDA tensor [tokens, heads, head_dim]")
    tokens, _, d = some.shape
    h = [_heads(t, n, tokens, d) for t, n in ((q, "q"), (k, "k"), (q_out, "q_out"), (k_out, "k_out"))]
    cp, sp, npos, rot = _tables(cos, sin)
    st = load_library().puro_qk_norm_rope(
        ctypes.byref(h[0]), ctypes.byref(h[1]), tokens, d, _sized(q_gain, torch.bfloat16, d, "q_gain"),
        _sized(k_gain, torch.bfloat16, d, "k_gain"), float(eps), cp, sp, npos, rot, int(bool(interleaved)),
        _sized(positions, torch.int32, tokens, "positions"), ctypes.byref(h[2]), ctypes.byref(h[3]),
        _sized(rstd, torch.float32, tokens * (h[0].heads + h[1].heads), "rstd"),
        _ptr(dev_status, torch.int32, "dev_status"), _stream(stream))
    _check("puro_qk_norm_rope", st)


def puro_qk_norm_rope_backward(dq_out: Optional[torch.Tensor], dk_out: Optional[torch.Tensor],
                               q: Optional[torch.Tensor], k: Optional[torch.Tensor], rstd: torch.Tensor,
                               q_gain: Optional[torch.Tensor], k_gain: Optional[torch.Tensor],
                               cos: Optional[torch.Tensor], sin: Optional[torch.Tensor],
                               positions: Optional[torch.Tensor], interleaved: bool, dq: Optional[torch.Tensor],
                               dk: Optional[torch.Tensor], dq_gain: Optional[torch.Tensor] = None,
                               dk_gain: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                               dev_status: Optional[torch.Tensor] = None, stream=None) -> None:
    """Backward of puro_qk_norm_rope from the gradients of its outputs, its
    inputs and rstd: dq, dk (bf16 views, which may be dq_out and dk_out) and the
    gains' gradients (fp32 [head_dim], through a workspace of
    puro_qk_norm_rope_workspace_size bytes)."""
    _on_current_device(q if q is not None else k)
    st = (_native or _load_native()).puro_qk_norm_rope_backward(dq_out, dk_out, q, k, rstd, q_gain, k_gain, cos, sin,
                                                                positions, interleaved, dq, dk, dq_gain, dk_gain, workspace,
                                                                dev_status, stream)
    if st is not None:
        return _check("puro_qk_norm_rope_backward", st)
    _on_current_device(dq_out, dk_out, q, k, rstd, q_gain, k_gain, cos, sin, positions, dq, dk, dq_gain, dk_gain,
                       workspace, dev_status)
    some = q if q is not None else k
    if some is None or some.dim() != 3:
        raise ValueError("q or k must be a bf16 CUDA tensor [tokens, heads, head_dim]")
    tokens, _, d = some.shape
    h = [_heads(t, n, tokens, d) for t, n in ((dq_out, "dq_out"), (dk_out, "dk_out"), (q, "q"), (k, "k"), (dq, "dq"),
                                              (dk, "dk"))]
    cp, sp, npos, rot = _tables(cos, sin)
    st = load_library().puro_qk_norm_rope_backward(
        *[ctypes.byref(x) for x in h[:4]], _sized(rstd, torch.float32, tokens * (h[2].heads + h[3].heads), "rstd"), tokens, d,
        _sized(q_gain, torch.bfloat16, d, "q_gain"), _sized(k_gain, torch.bfloat16, d, "k_gain"), cp, sp, npos, rot,
        int(bool(interleaved)), _sized(positions, torch.int32, tokens, "positions"), ctypes.byref(h[4]), ctypes.byref(h[5]),
        _sized(dq_gain, torch.float32, d, "dq_gain"), _sized(dk_gain, torch.float32, d, "dk_gain"),
        _ptr(workspace, None, "workspace"), workspace.numel() * workspace.element_size() if workspace is not None else 0,
        _ptr(dev_status, torch.int32, "dev_status"), _stream(stream))
    _check("puro_qk_norm_rope_backward", st)


def puro_qk_norm_rope_workspace_size(tokens: int, q_heads: int, k_heads: int, head_dim: int) -> int:
    return int(load_library().puro_qk_norm_rope_workspace_size(tokens, q_heads, k_heads, head_dim))


# --------------------------------------------------------------------------
# The position rotation without a norm
# --------------------------------------------------------------------------
def puro_rope_frequencies(rot_dim: int, base: float, scaling: int, factor: float, trained_positions: int, fast_turns: float,
                          slow_turns: float, frequencies: torch.Tensor) -> None:
    """The angle of each pair of channels per position, as 2^64ths of a turn: into
    frequencies, int64 [rot_dim / 2] on the CPU."""
    if frequencies.is_cuda or frequencies.dtype != torch.int64 or not frequencies.is_contiguous() or \
            frequencies.numel() != rot_dim // 2:
        raise ValueError(f"frequencies must be an int64 CPU tensor [{rot_dim // 2}]")
    st = load_library().puro_rope_frequencies(rot_dim, float(base), scaling, float(factor), trained_positions, float(fast_turns),
                                              float(slow_turns), frequencies.data_ptr())
    _check("puro_rope_frequencies", st)


def rope_frequencies(rot_dim: int, base: float, scaling: int = ROPE_NONE, factor: float = 1.0, trained_positions: int = 0,
                     fast_turns: float = 32.0, slow_turns: float = 1.0, device="cuda") -> torch.Tensor:
    """The frequencies that puro_rope and puro_rope_tables read (int64 [rot_dim / 2]), scaled for
    a context factor times the trained one where scaling is not ROPE_NONE."""
    f = torch.empty(max(0, rot_dim) // 2, dtype=torch.int64)
    puro_rope_frequencies(rot_dim, base, scaling, factor, trained_positions, fast_turns, slow_turns, f)
    return f.to(device)


def puro_rope_tables(frequencies: torch.Tensor, first: int, cos: torch.Tensor, sin: torch.Tensor, scale: float = 1.0,
                     stream=None) -> None:
    """cos and sin (fp32 [positions, rot_dim / 2], written) of positions first, first + 1, ..., times
    scale: the tables of puro_qk_norm_rope."""
    _on_current_device(frequencies)
    st = (_native or _load_native()).puro_rope_tables(frequencies, first, cos, sin, scale, stream)
    if st is not None:
        return _check("puro_rope_tables", st)
    _on_current_device(frequencies, cos, sin)
    cp, sp, count, rot = _tables(cos, sin)
    st = load_library().puro_rope_tables(_sized(frequencies, torch.int64, rot // 2, "frequencies"), rot, float(scale), first,
                                         count, cp, sp, _stream(stream))
    _check("puro_rope_tables", st)


def _rope(name, x, x2, frequencies, positions, interleaved, y, y2, scale, stream, names):
    _on_current_device(x if x is not None else x2)
    st = getattr(_native or _load_native(), name)(x, x2, frequencies, positions, interleaved, y, y2, scale, stream)
    if st is not None:
        return _check(name, st)
    _on_current_device(x, x2, frequencies, positions, y, y2)
    some = x if x is not None else x2
    if some is None or some.dim() != 3:
        raise ValueError(f"{names[0]} or {names[1]} must be a bf16 CUDA tensor [tokens, heads, head_dim]")
    tokens, _, d = some.shape
    h = [_heads(t, n, tokens, d) for t, n in zip((x, x2, y, y2), names)]
    st = getattr(load_library(), name)(
        ctypes.byref(h[0]), ctypes.byref(h[1]), tokens, d, _ptr(frequencies, torch.int64, "frequencies"),
        2 * frequencies.numel(), float(scale), int(bool(interleaved)), _sized(positions, torch.int32, tokens, "positions"),
        ctypes.byref(h[2]), ctypes.byref(h[3]), _stream(stream))
    _check(name, st)


def puro_rope(q: Optional[torch.Tensor], k: Optional[torch.Tensor], frequencies: torch.Tensor,
              positions: Optional[torch.Tensor], interleaved: bool, q_out: Optional[torch.Tensor],
              k_out: Optional[torch.Tensor], scale: float = 1.0, stream=None) -> None:
    """Rotate each query and key head (bf16 [tokens, heads, head_dim] views, for
    instance of one qkv output) by the tokens' positions, without a norm: q_out,
    k_out, which may be q and k.  frequencies: rope_frequencies(rot_dim, ...) on the
    device; scale multiplies the rotated channels.  positions: int32 [tokens], None
    for 0, 1, ...; a negative one marks a padding row, whose output is zero."""
    _rope("puro_rope", q, k, frequencies, positions, interleaved, q_out, k_out, scale, stream, ("q", "k", "q_out", "k_out"))


def puro_rope_backward(dq_out: Optional[torch.Tensor], dk_out: Optional[torch.Tensor], frequencies: torch.Tensor,
                       positions: Optional[torch.Tensor], interleaved: bool, dq: Optional[torch.Tensor],
                       dk: Optional[torch.Tensor], scale: float = 1.0, stream=None) -> None:
    """Backward of puro_rope: dq, dk (bf16 views, which may be dq_out and dk_out) from the gradients of its outputs."""
    _rope("puro_rope_backward", dq_out, dk_out, frequencies, positions, interleaved, dq, dk, scale, stream,
          ("dq_out", "dk_out", "dq", "dk"))


def puro_set_wait_timeout_ns(ns: int) -> None:
    load_library().puro_set_wait_timeout_ns(int(ns))


def puro_set_gemm_tile_n(tile_n: int) -> None:
    """0: per-shape choice; 224 or 256: force that block-scaled GEMM form."""
    _check("puro_set_gemm_tile_n", load_library().puro_set_gemm_tile_n(int(tile_n)))


# --------------------------------------------------------------------------
# Allocation helpers (torch allocates; the library computes)
# --------------------------------------------------------------------------
@dataclass
class Quantized:
    """Both copies produced by one quantise call."""
    rowwise: FP8Operand
    colwise: Optional[FP8Operand]
    amax: Optional[torch.Tensor] = None


def scale_vec_shape(rows: int, red: int):
    """Shape of a blockwise scale buffer for an operand [rows, red]: 512-byte
    tensor-core scale-vector chunks per 128 rows and 4 k-blocks."""
    return (rows // 128, (red // 128 + 3) // 4, 512)


def empty_scales(rows: int, red: int, scaling: int, role: int, device) -> torch.Tensor:
    if scaling == SCALE_TENSOR:
        return torch.empty(1, dtype=torch.float32, device=device)
    return torch.empty(scale_vec_shape(rows, red), dtype=torch.uint8, device=device)


def puro_fp8_scale_bytes(rows: int, red: int) -> int:
    return int(load_library().puro_fp8_scale_bytes(rows, red))


def quantize(x: torch.Tensor, fmt: int = E4M3, scaling: int = SCALE_BLOCK, role: int = ROLE_ACT,
             transpose: bool = True, out: Optional[Quantized] = None, dev_status: Optional[torch.Tensor] = None,
             stream=None) -> Quantized:
    """Quantise x [rows, cols] (bf16) into a rowwise operand [rows, cols] and,
    if ``transpose``, a columnwise operand [cols, rows]; per-tensor mode runs
    the amax kernel first."""
    rows, cols = x.shape
    dev = x.device
    if out is None:
        q = torch.empty((rows, cols), dtype=torch.uint8, device=dev)
        s = empty_scales(rows, cols, scaling, role, dev)
        colwise = None
        if transpose:
            colwise = FP8Operand(torch.empty((cols, rows), dtype=torch.uint8, device=dev),
                                 empty_scales(cols, rows, scaling, role, dev), fmt, scaling, role)
        amax = torch.zeros(1, dtype=torch.int32, device=dev) if scaling == SCALE_TENSOR else None
        out = Quantized(FP8Operand(q, s, fmt, scaling, role), colwise, amax)
    if scaling == SCALE_TENSOR:
        puro_fp8_amax(x, out.amax, stream)
    puro_fp8_quantize(x, fmt, scaling, role, out.amax if scaling == SCALE_TENSOR else None, out.rowwise.data,
                      out.rowwise.scale, out.colwise.data if out.colwise else None,
                      out.colwise.scale if out.colwise else None, dev_status=dev_status, stream=stream)
    return out


__all__ = [n for n in dir() if n.startswith("puro_")] + [
    "E4M3", "E5M2", "SCALE_TENSOR", "SCALE_BLOCK", "ROLE_ACT", "ROLE_WEIGHT", "ACT_NONE", "ACT_RELU", "ACT_SILU",
    "ACT_GELU", "ACT_GELU_TANH", "ROPE_NONE", "ROPE_LINEAR", "ROPE_BASE", "ROPE_TURNS", "ROPE_INDEX", "rope_frequencies", "MUON_STEPS", "muon_table", "PuroError", "FP8Operand",
    "Quantized", "quantize", "load_library", "empty_scales", "scale_vec_shape", "LIB_PATH", "HEADER_PATH",
]
