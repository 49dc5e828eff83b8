"""ctypes binding of the element embedding (include/ee.h): same names as the C ABI, argument marshalling only."""
from __future__ import annotations

import ctypes as C

from .binding import SC_BF16, SC_F32, SC_F64, ScError, _check, _ptr, _stream, lib  # noqa: F401

EE_MAX_ELEMENTS, EE_MAX_CHANNELS = 1000000, 65536

EXPORTS = ("ee_forward", "ee_workspace_bytes", "ee_backward")


class ee_config(C.Structure):
    _fields_ = [("struct_size", C.c_int32), ("num_elements", C.c_int32), ("num_channels", C.c_int32), ("dtype", C.c_int32),
                ("device", C.c_int32), ("reserved", C.c_int32), ("scale", C.c_double)]


def make_config(num_elements: int, num_channels: int, scale: float = 1.0, dtype: int = SC_F32, device: int = 0) -> ee_config:
    return ee_config(C.sizeof(ee_config), num_elements, num_channels, dtype, device, 0, scale)


_vp, _i64, _cfg = C.c_void_p, C.c_int64, C.POINTER(ee_config)
lib.ee_forward.argtypes = [_cfg, _i64] + [_vp] * 4
lib.ee_workspace_bytes.argtypes = [_cfg, _i64, C.POINTER(C.c_size_t)]
lib.ee_backward.argtypes = [_cfg, _i64] + [_vp] * 4 + [C.c_size_t, _vp]
for _name in EXPORTS:
    getattr(lib, _name).restype = C.c_int


def ee_forward(cfg: ee_config, n_nodes: int, z, T, Y, stream=None) -> None:
    _check(lib.ee_forward(C.byref(cfg), n_nodes, _ptr(z), _ptr(T), _ptr(Y), _stream(stream)))


def ee_workspace_bytes(cfg: ee_config, n_nodes: int) -> int:
    n = C.c_size_t()
    _check(lib.ee_workspace_bytes(C.byref(cfg), n_nodes, C.byref(n)))
    return n.value


def ee_backward(cfg: ee_config, n_nodes: int, z, dY, dT, workspace, workspace_bytes: int, stream=None) -> None:
    _check(lib.ee_backward(C.byref(cfg), n_nodes, _ptr(z), _ptr(dY), _ptr(dT), _ptr(workspace), workspace_bytes, _stream(stream)))
