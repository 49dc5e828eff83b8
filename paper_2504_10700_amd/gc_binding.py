"""ctypes binding of the gradient norm and clipping (include/gc.h): same names as the C ABI, argument marshalling
only.  `make_tensors` builds the host array that gc_clip takes; a training loop whose gradients keep their buffers builds it once."""
from __future__ import annotations

import ctypes as C
from typing import Optional, Sequence

import torch

from .binding import SC_BF16, SC_F32, SC_F64, ScError, _check, _ptr, _stream, lib  # noqa: F401

GC_MAX_TENSORS = 65536

EXPORTS = ("gc_workspace_bytes", "gc_clip")

_DTYPES = {torch.float32: SC_F32, torch.float64: SC_F64, torch.bfloat16: SC_BF16}


class gc_tensor(C.Structure):
    _fields_ = [("src", C.c_void_p), ("dst", C.c_void_p), ("numel", C.c_int64), ("dtype", C.c_int32), ("reserved", C.c_int32)]


class gc_config(C.Structure):
    _fields_ = [("struct_size", C.c_int32), ("dtype", C.c_int32), ("device", C.c_int32), ("reserved", C.c_int32),
                ("max_norm", C.c_double), ("eps", C.c_double)]


def make_config(max_norm: float, eps: float = 1e-6, dtype: int = SC_F32, device: int = 0) -> gc_config:
    return gc_config(C.sizeof(gc_config), dtype, device, 0, max_norm, eps)


def make_tensors(src: Sequence[torch.Tensor], dst: Optional[Sequence[torch.Tensor]] = None):
    """The gc_tensor array of `src`, written to `dst` (None: the norm alone; `src` itself: clipped in place).  It holds
    addresses: the caller keeps the tensors alive as long as it is used."""
    if dst is not None and len(dst) != len(src):
        raise ValueError("src and dst differ in length")
    for x, y in zip(src, src if dst is None else dst):
        if x.dtype not in _DTYPES or y.dtype != x.dtype or y.numel() != x.numel() or y.device != x.device:
            raise ValueError("tensors are float32, float64 or bfloat16, and dst is of the type, size and device of src")
        if not x.is_contiguous() or not y.is_contiguous():
            raise ValueError("tensors are dense")
    return (gc_tensor * len(src))(*[gc_tensor(x.data_ptr() or None, None if dst is None else dst[i].data_ptr() or None, x.numel(),
                                              _DTYPES[x.dtype], 0) for i, x in enumerate(src)])


_vp, _i64 = C.c_void_p, C.c_int64
lib.gc_workspace_bytes.argtypes = [C.POINTER(gc_config), _i64, _vp, C.POINTER(C.c_size_t)]
lib.gc_clip.argtypes = [C.POINTER(gc_config), _i64, _vp, _vp, _vp, C.c_size_t, _vp]
for _name in EXPORTS:
    getattr(lib, _name).restype = C.c_int


def gc_workspace_bytes(cfg: gc_config, tensors) -> int:
    n = C.c_size_t()
    _check(lib.gc_workspace_bytes(C.byref(cfg), len(tensors), tensors, C.byref(n)))
    return n.value


def gc_clip(cfg: gc_config, tensors, norm_and_coefficient, workspace, workspace_bytes: int, stream=None) -> None:
    _check(lib.gc_clip(C.byref(cfg), len(tensors), tensors, _ptr(norm_and_coefficient), _ptr(workspace), workspace_bytes,
                       _stream(stream)))
