"""ctypes binding of libmgwfbp_layers.so with the names of include/mgwfbp_layers.h: the operators that make per-layer
gradients.  Argument marshalling only; device buffers are integer addresses, streams integer handles, as in binding.py.
`layers` takes torch tensors."""
from __future__ import annotations

import ctypes as C
import functools
import os
from typing import Optional, Sequence, Tuple

from .binding import BF16, F16, F32, MgwfbpError  # noqa: F401

I32, I64 = 0, 1                                             # mgwfbp_id_type
IDENTITY, GELU, GELU_TANH, SILU = range(4)                  # mgwfbp_act_kind
ACT_GROUP = 128                                             # MGWFBP_ACT_GROUP
MAX_TABLES = 4                                              # MGWFBP_MAX_TABLES

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB: Optional[C.CDLL] = None

_i32, _i64, _u64, _f32, _vp = C.c_int32, C.c_int64, C.c_uint64, C.c_float, C.c_void_p
_i64p, _u64p = C.POINTER(C.c_int64), C.POINTER(C.c_uint64)

_SIGNATURES = {
    "mgwfbp_embed": (C.c_int, [_vp, _i32, _i32, _i64, _i64, _vp, _i64, _i32, _vp]),
    "mgwfbp_embed_grad_workspace": (C.c_int, [_i64, _i64, _i64, _u64p]),
    "mgwfbp_embed_grad": (C.c_int, [_vp, _i32, _i64, _vp, _i64, _i32, _f32, _i64, _i32, _vp, _i64, _i64, _i64, _i32, _vp, _u64, _vp]),
    "mgwfbp_act_dims": (C.c_int, [_i64, _i64, _i64p, _i64p]),
    "mgwfbp_act_store": (C.c_int, [_vp, _i64, _i32, _i64, _i64, _i32, _vp, _vp, _i64, _vp, _i64, _vp]),
    "mgwfbp_act_backward": (C.c_int, [_vp, _vp, _i64, _i64, _i64, _i32, _vp, _i64, _vp, _i64, _vp, _i64, _i32, _vp]),
    "mgwfbp_act_linear_grad_workspace": (C.c_int, [_i64, _i64, _i64, _u64p]),
    "mgwfbp_act_linear_grad": (C.c_int, [_vp, _vp, _i64, _i64, _i64, _vp, _i64, _i32, _i64, _i32, _vp, _i64, _vp, _i32, _vp, _u64, _vp]),
    "mgwfbp_layers_last_hip_error": (C.c_int, []),
}


class Table(C.Structure):
    """mgwfbp_table: one table of an embedding lookup and the rows that are taken from it."""
    _fields_ = [("d_rows", _vp), ("d_ids", _vp), ("n_rows", _i64), ("row_stride", _i64), ("scale", _f32), ("id_type", _i32)]


def library_path() -> str:
    return os.environ.get("MGWFBP_LAYERS_LIBRARY", os.path.join(_HERE, "libmgwfbp_layers.so"))


def lib() -> C.CDLL:
    """The loaded library.  Raises if it is missing: there is no fallback path."""
    global _LIB
    if _LIB is None:
        path = library_path()
        if not os.path.exists(path):
            raise MgwfbpError(f"load {path} (not built; run `python -m paper_1912_09268_amd.build`)", -1)
        handle = C.CDLL(path)
        for name, (res, args) in _SIGNATURES.items():
            fn = getattr(handle, name)
            fn.restype = res
            fn.argtypes = args
        _LIB = handle
        _announce()
    return _LIB


_native = None      # the extension module of layers.py, once that is imported


def _announce() -> None:
    """Hands the loaded library's entry points to the extension module that takes the tensors of layers.py apart."""
    if _native is not None and _LIB is not None:
        _native.set_functions(_check, {name: C.cast(getattr(_LIB, name), _vp).value for name in _SIGNATURES})


def _check(fn: str, status: int) -> None:
    if status != 0:
        raise MgwfbpError(fn, status, lib().mgwfbp_layers_last_hip_error())


def embed(tables: Sequence[Table], table_dtype: int, n_tokens: int, dim: int, d_out: int, out_stride: int, out_dtype: int,
          stream: int = 0) -> None:
    """mgwfbp_embed."""
    _check("mgwfbp_embed", lib().mgwfbp_embed((Table * len(tables))(*tables), len(tables), table_dtype, n_tokens, dim, d_out, out_stride,
                                              out_dtype, stream))


@functools.lru_cache(maxsize=1024)
def embed_grad_workspace(n_tokens: int, n_rows: int, dim: int) -> int:
    """mgwfbp_embed_grad_workspace: bytes."""
    out = C.c_uint64()
    _check("mgwfbp_embed_grad_workspace", lib().mgwfbp_embed_grad_workspace(n_tokens, n_rows, dim, C.byref(out)))
    return out.value


def embed_grad(d_ids: int, id_type: int, n_tokens: int, d_dy: int, dy_stride: int, dy_dtype: int, scale: float, padding_row: int,
               accumulate: bool, d_grad: int, n_rows: int, dim: int, grad_stride: int, grad_dtype: int, d_workspace: int,
               workspace_bytes: int, stream: int = 0) -> None:
    """mgwfbp_embed_grad."""
    _check("mgwfbp_embed_grad", lib().mgwfbp_embed_grad(d_ids, id_type, n_tokens, d_dy, dy_stride, dy_dtype, scale, padding_row,
                                                        bool(accumulate), d_grad, n_rows, dim, grad_stride, grad_dtype, d_workspace,
                                                        workspace_bytes, stream))


@functools.lru_cache(maxsize=1024)
def act_dims(n_tokens: int, n_channels: int) -> Tuple[int, int]:
    """mgwfbp_act_dims -> (ld, n_groups)."""
    ld, groups = C.c_int64(), C.c_int64()
    _check("mgwfbp_act_dims", lib().mgwfbp_act_dims(n_tokens, n_channels, C.byref(ld), C.byref(groups)))
    return ld.value, groups.value


def act_store(d_x: int, x_stride: int, dtype: int, n_tokens: int, n_channels: int, kind: int, d_q: int, d_scale: int, ld: int, d_y: int,
              y_stride: int, stream: int = 0) -> None:
    """mgwfbp_act_store."""
    _check("mgwfbp_act_store", lib().mgwfbp_act_store(d_x, x_stride, dtype, n_tokens, n_channels, kind, d_q, d_scale, ld, d_y, y_stride,
                                                      stream))


def act_backward(d_q: int, d_scale: int, ld: int, n_tokens: int, n_channels: int, kind: int, d_dy: int, dy_stride: int, d_dx: int,
                 dx_stride: int, d_y: int, y_stride: int, dtype: int, stream: int = 0) -> None:
    """mgwfbp_act_backward."""
    _check("mgwfbp_act_backward", lib().mgwfbp_act_backward(d_q, d_scale, ld, n_tokens, n_channels, kind, d_dy, dy_stride, d_dx, dx_stride,
                                                            d_y, y_stride, dtype, stream))


@functools.lru_cache(maxsize=1024)
def act_linear_grad_workspace(n_tokens: int, n_channels: int, n_outputs: int) -> int:
    """mgwfbp_act_linear_grad_workspace: bytes."""
    out = C.c_uint64()
    _check("mgwfbp_act_linear_grad_workspace", lib().mgwfbp_act_linear_grad_workspace(n_tokens, n_channels, n_outputs, C.byref(out)))
    return out.value


def act_linear_grad(d_q: int, d_scale: int, ld: int, n_tokens: int, n_channels: int, d_dy: int, dy_stride: int, dy_dtype: int,
                    n_outputs: int, accumulate: bool, d_dw: int, dw_stride: int, d_db: int, grad_dtype: int, d_workspace: int,
                    workspace_bytes: int, stream: int = 0) -> None:
    """mgwfbp_act_linear_grad."""
    _check("mgwfbp_act_linear_grad", lib().mgwfbp_act_linear_grad(d_q, d_scale, ld, n_tokens, n_channels, d_dy, dy_stride, dy_dtype, n_outputs,
                                                                  bool(accumulate), d_dw, dw_stride, d_db, grad_dtype, d_workspace,
                                                                  workspace_bytes, stream))
