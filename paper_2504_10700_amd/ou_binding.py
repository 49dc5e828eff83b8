"""ctypes binding of the orthogonalised update (include/ou.h): same names as the C ABI, argument marshalling only.  `make_tensors` builds
the host array that ou_step takes; a training loop whose gradients keep their buffers builds it once."""
from __future__ import annotations

import ctypes as C
from typing import Optional, Sequence

import torch

from .binding import SC_BF16, SC_F32, SC_F64, ScError, _check, _ptr, _stream, lib  # noqa: F401

OU_MAX_TENSORS, OU_MAX_SIDE, OU_MAX_STEPS, OU_MAX_GROWTH = 16384, 65536, 32, 1024
OU_MAX_TILES = 8388608
OU_NESTEROV = 1

EXPORTS = ("ou_workspace_bytes", "ou_step")

_DTYPES = {torch.float32: SC_F32, torch.float64: SC_F64, torch.bfloat16: SC_BF16}


class ou_tensor(C.Structure):
    _fields_ = [("grad", C.c_void_p), ("momentum", C.c_void_p), ("weight", C.c_void_p), ("update", C.c_void_p), ("scale", C.c_double),
                ("count", C.c_int64), ("rows", C.c_int32), ("cols", C.c_int32), ("dtype", C.c_int32), ("reserved", C.c_int32)]


class ou_config(C.Structure):
    _fields_ = [("struct_size", C.c_int32), ("device", C.c_int32), ("steps", C.c_int32), ("flags", C.c_uint32), ("a", C.c_double), ("b", C.c_double),
                ("c", C.c_double), ("momentum", C.c_double), ("rate", C.c_double), ("decay", C.c_double), ("eps", C.c_double)]


def make_config(rate: float, momentum: float = 0.95, decay: float = 0.0, steps: int = 5, coefficients=(3.4445, -4.7750, 2.0315), eps: float = 1e-7,
                nesterov: bool = True, device: int = 0) -> ou_config:
    return ou_config(C.sizeof(ou_config), device, steps, OU_NESTEROV if nesterov else 0, *coefficients, momentum, rate, decay, eps)


def make_tensors(grad: Sequence[torch.Tensor], momentum: Optional[Sequence[torch.Tensor]] = None, weight: Optional[Sequence[torch.Tensor]] = None,
                 update: Optional[Sequence[torch.Tensor]] = None, scale=1.0):
    """The ou_tensor array of matrices [rows][cols] or batches [...][rows][cols].  scale: one number, or one for each tensor.  It holds
    addresses: the caller keeps the tensors alive as long as it is used."""
    n = len(grad)
    lists = [momentum, weight, update]
    scales = list(scale) if isinstance(scale, (list, tuple)) else [scale] * n
    if any(x is not None and len(x) != n for x in lists) or len(scales) != n:
        raise ValueError("the lists differ in length")
    items = []
    for i, g in enumerate(grad):
        if g.dtype not in _DTYPES or g.dim() < 2 or not g.is_contiguous():
            raise ValueError("gradients are dense matrices of float32, float64 or bfloat16, or batches of them")
        wide = torch.float32 if g.dtype == torch.bfloat16 else g.dtype
        own = [None if x is None else x[i] for x in lists]
        for x, t in zip(own, (wide, wide, g.dtype)):
            if x is not None and (x.dtype != t or x.shape != g.shape or x.device != g.device or not x.is_contiguous()):
                raise ValueError("momentum and weight are dense, of the shape and device of the gradient and of its type (float32 beside bfloat16), "
                                 "the update of its type")
        count = 1
        for s in g.shape[:-2]:
            count *= s
        items.append(ou_tensor(g.data_ptr() or None, *[None if x is None else x.data_ptr() or None for x in own], scales[i], count,
                               g.shape[-2], g.shape[-1], _DTYPES[g.dtype], 0))
    return (ou_tensor * n)(*items)


_vp, _i64 = C.c_void_p, C.c_int64
lib.ou_workspace_bytes.argtypes = [C.POINTER(ou_config), _i64, _vp, C.POINTER(C.c_size_t)]
lib.ou_step.argtypes = [C.POINTER(ou_config), _i64, _vp, _vp, C.c_size_t, _vp]
for _name in EXPORTS:
    getattr(lib, _name).restype = C.c_int


def ou_workspace_bytes(cfg: ou_config, tensors) -> int:
    n = C.c_size_t()
    _check(lib.ou_workspace_bytes(C.byref(cfg), len(tensors), tensors, C.byref(n)))
    return n.value


def ou_step(cfg: ou_config, tensors, workspace, workspace_bytes: int, stream=None) -> None:
    _check(lib.ou_step(C.byref(cfg), len(tensors), tensors, _ptr(workspace), workspace_bytes, _stream(stream)))
