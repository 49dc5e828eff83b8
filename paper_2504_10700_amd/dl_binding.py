"""ctypes binding of the dense layer (include/dl.h): same names as the C ABI, argument marshalling only."""
from __future__ import annotations

import ctypes as C

from .binding import SC_BF16, SC_F32, SC_F64, ScError, _check, _ptr, _stream, lib  # noqa: F401

DL_NONE, DL_RELU, DL_SILU, DL_GELU = 0, 1, 2, 3
DL_MAX_WIDTH, DL_MAX_STRIDE = 65536, 33554432

EXPORTS = ("dl_forward", "dl_workspace_bytes", "dl_backward", "dl_double_backward")


class dl_config(C.Structure):
    _fields_ = [("struct_size", C.c_int32), ("k_in", C.c_int32), ("k_out", C.c_int32), ("activation", C.c_int32),
                ("dtype", C.c_int32), ("device", C.c_int32), ("ld_in", C.c_int64), ("ld_out", C.c_int64)]


def make_config(k_in: int, k_out: int, activation: int = DL_NONE, dtype: int = SC_F32, device: int = 0, ld_in: int = 0,
                ld_out: int = 0) -> dl_config:
    return dl_config(C.sizeof(dl_config), k_in, k_out, activation, dtype, device, ld_in, ld_out)


_vp, _i64, _cfg = C.c_void_p, C.c_int64, C.POINTER(dl_config)
lib.dl_forward.argtypes = [_cfg, _i64] + [_vp] * 7
lib.dl_workspace_bytes.argtypes = [_cfg, _i64, C.POINTER(C.c_size_t)]
lib.dl_backward.argtypes = [_cfg, _i64] + [_vp] * 8 + [C.c_size_t, _vp]
lib.dl_double_backward.argtypes = [_cfg, _i64] + [_vp] * 10 + [C.c_size_t, _vp]
for _name in EXPORTS:
    getattr(lib, _name).restype = C.c_int


def dl_forward(cfg: dl_config, n_rows: int, X, W, b, residual, Y, Z, stream=None) -> None:
    _check(lib.dl_forward(C.byref(cfg), n_rows, _ptr(X), _ptr(W), _ptr(b), _ptr(residual), _ptr(Y), _ptr(Z), _stream(stream)))


def dl_workspace_bytes(cfg: dl_config, n_rows: int) -> int:
    n = C.c_size_t()
    _check(lib.dl_workspace_bytes(C.byref(cfg), n_rows, C.byref(n)))
    return n.value


def dl_backward(cfg: dl_config, n_rows: int, X, W, Z, dY, dX, dW, db, workspace, workspace_bytes: int, stream=None) -> None:
    _check(lib.dl_backward(C.byref(cfg), n_rows, _ptr(X), _ptr(W), _ptr(Z), _ptr(dY), _ptr(dX), _ptr(dW), _ptr(db), _ptr(workspace),
                           workspace_bytes, _stream(stream)))


def dl_double_backward(cfg: dl_config, n_rows: int, X, W, Z, dY, HX, ddY, X2, W2, b2, workspace, workspace_bytes: int,
                       stream=None) -> None:
    _check(lib.dl_double_backward(C.byref(cfg), n_rows, _ptr(X), _ptr(W), _ptr(Z), _ptr(dY), _ptr(HX), _ptr(ddY), _ptr(X2), _ptr(W2),
                                  _ptr(b2), _ptr(workspace), workspace_bytes, _stream(stream)))
