"""ctypes binding of the products by element (include/gp.h): same names as the C ABI, argument marshalling only."""
from __future__ import annotations

import ctypes as C

from .binding import SC_BF16, SC_F32, SC_F64, ScError, _check, _ptr, _stream, lib  # noqa: F401

GP_MAX_ELEMENTS, GP_MAX_WIDTH, GP_MAX_COMPONENTS, GP_MAX_STRIDE = 1024, 65536, 64, 33554432
GP_MAX_ROWS, GP_UNGROUPED = 536870912, 64

EXPORTS = ("gp_grouping_bytes", "gp_group", "gp_workspace_bytes", "gp_forward", "gp_backward")


class gp_config(C.Structure):
    _fields_ = [("struct_size", C.c_int32), ("num_elements", C.c_int32), ("k_in", C.c_int32), ("k_out", C.c_int32), ("components", C.c_int32),
                ("dtype", C.c_int32), ("device", C.c_int32), ("reserved", C.c_int32), ("ld_in", C.c_int64), ("ld_out", C.c_int64)]


def make_config(num_elements: int, k_in: int, k_out: int, components: int = 1, dtype: int = SC_F32, device: int = 0, ld_in: int = 0,
                ld_out: int = 0) -> gp_config:
    return gp_config(C.sizeof(gp_config), num_elements, k_in, k_out, components, dtype, device, 0, ld_in, ld_out)


_vp, _i64, _sz, _cfg = C.c_void_p, C.c_int64, C.c_size_t, C.POINTER(gp_config)
lib.gp_grouping_bytes.argtypes = [_cfg, _i64, C.POINTER(_sz)]
lib.gp_group.argtypes = [_cfg, _i64, _vp, _vp, _sz, _vp]
lib.gp_workspace_bytes.argtypes = [_cfg, _i64, C.POINTER(_sz)]
lib.gp_forward.argtypes = [_cfg, _i64] + [_vp] * 7 + [_sz, _vp]
lib.gp_backward.argtypes = [_cfg, _i64] + [_vp] * 8 + [_sz, _vp]
for _name in EXPORTS:
    getattr(lib, _name).restype = C.c_int


def _bytes(fn, cfg: gp_config, n_nodes: int) -> int:
    n = _sz()
    _check(fn(C.byref(cfg), n_nodes, C.byref(n)))
    return n.value


def gp_grouping_bytes(cfg: gp_config, n_nodes: int) -> int:
    return _bytes(lib.gp_grouping_bytes, cfg, n_nodes)


def gp_group(cfg: gp_config, n_nodes: int, z, grouping, grouping_bytes: int, stream=None) -> None:
    _check(lib.gp_group(C.byref(cfg), n_nodes, _ptr(z), _ptr(grouping), grouping_bytes, _stream(stream)))


def gp_workspace_bytes(cfg: gp_config, n_nodes: int) -> int:
    return _bytes(lib.gp_workspace_bytes, cfg, n_nodes)


def gp_forward(cfg: gp_config, n_nodes: int, z, grouping, X, W, residual, Y, workspace, workspace_bytes: int, stream=None) -> None:
    _check(lib.gp_forward(C.byref(cfg), n_nodes, _ptr(z), _ptr(grouping), _ptr(X), _ptr(W), _ptr(residual), _ptr(Y), _ptr(workspace),
                          workspace_bytes, _stream(stream)))


def gp_backward(cfg: gp_config, n_nodes: int, z, grouping, X, W, dY, dX, dW, workspace, workspace_bytes: int, stream=None) -> None:
    _check(lib.gp_backward(C.byref(cfg), n_nodes, _ptr(z), _ptr(grouping), _ptr(X), _ptr(W), _ptr(dY), _ptr(dX), _ptr(dW), _ptr(workspace),
                           workspace_bytes, _stream(stream)))
