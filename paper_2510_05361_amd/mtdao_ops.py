"""ctypes binding of include/mtdao_ops.h (argument marshalling only).

As in ``mtdao.py``: function names match the C entry points, device buffers
are raw pointers, streams raw HIP stream handles, and errors raise
``MtdaoError``.
"""

from __future__ import annotations

import ctypes
import struct
from typing import Optional, Sequence

from . import mtdao as abi

MTDAO_BLOCK8 = 128
MTDAO_NORM_RMS, MTDAO_NORM_LAYER = 0, 1
MTDAO_PERI_MAX_D = 8192

_VP, _I32, _I64, _F32, _F64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_double


class AdamwTensor(ctypes.Structure):
    _fields_ = [("p", _VP), ("g", _VP), ("m", _VP), ("v", _VP), ("m_scale", _VP), ("v_scale", _VP), ("numel", _I64),
                ("weight_decay", _F64)]


class AdamwConfig(ctypes.Structure):
    _fields_ = [("param_dtype", _I32), ("grad_dtype", _I32), ("state_bits", _I32), ("n_tensors", _I32), ("beta1", _F64),
                ("beta2", _F64), ("eps", _F64), ("max_norm", _F64), ("start_step", _I64)]


class PeriNormArgs(ctypes.Structure):
    _fields_ = [("rows", _I64), ("d", _I64), ("kind", _I32), ("stream_dtype", _I32), ("branch_dtype", _I32),
                ("weight_dtype", _I32), ("eps", _F32), ("scale", _F32), ("rows_per_gate", _I64), ("ld_x", _I64),
                ("ld_f", _I64), ("ld_d_out", _I64), ("ld_dn", _I64), ("x", _VP), ("f", _VP), ("w_post", _VP),
                ("w_pre", _VP), ("gate", _VP), ("d_out", _VP), ("dn", _VP), ("x_out", _VP), ("n_out", _VP), ("df", _VP),
                ("d_w_post", _VP), ("d_w_pre", _VP), ("d_gate", _VP)]


class Matrix8(ctypes.Structure):
    _fields_ = [("codes", _VP), ("scales", _VP), ("rows", _I64), ("cols", _I64), ("ld", _I64), ("scale_ld", _I64),
                ("scale_rows", _I32)]


_lib = None


def lib() -> ctypes.CDLL:
    global _lib
    if _lib is None:
        L = abi.lib()
        P, SZ = ctypes.POINTER, ctypes.c_size_t
        for name, args, res in (
                ("mtdao_adamw_workspace_bytes", [P(AdamwConfig), P(AdamwTensor), P(SZ)], _I32),
                ("mtdao_adamw_init", [P(AdamwConfig), P(AdamwTensor), _VP, SZ, _VP, P(_VP)], _I32),
                ("mtdao_adamw_set_grads", [_VP, P(_VP), _VP], _I32),
                ("mtdao_adamw_step", [_VP, _F64, _VP], _I32),
                ("mtdao_adamw_step_count", [_VP], _I64),
                ("mtdao_adamw_last_error", [_VP], ctypes.c_char_p),
                ("mtdao_adamw_destroy", [_VP], None),
                ("mtdao_peri_norm", [_VP, _VP], _I32),
                ("mtdao_peri_norm_backward_workspace_bytes", [_VP, P(SZ)], _I32),
                ("mtdao_peri_norm_backward", [_VP, _VP, SZ, _VP], _I32),
                ("mtdao_quantize8", [_VP, _I32, _I64, P(Matrix8), P(Matrix8), _VP], _I32),
                ("mtdao_product8_workspace_bytes", [_I64, _I64, _I64, P(SZ)], _I32),
                ("mtdao_product8", [P(Matrix8), P(Matrix8), _VP, _I32, _I64, _I32, _VP, SZ, _VP], _I32),
                ("mtdao_linear8_workspace_bytes", [_I64, _I64, _I64, P(SZ), P(SZ)], _I32),
                ("mtdao_linear8", [_VP, _I32, _I64, _I64, _VP, _VP, _I32, _I64, _VP, SZ, _VP], _I32),
                ("mtdao_linear8_backward", [_VP, _VP, _I32, _I64, _I64, _I64, _VP, _VP, _I64, _VP, _I64, _I32, _VP, SZ, _VP],
                 _I32)):
            fn = getattr(L, name)
            fn.argtypes, fn.restype = args, res
        _lib = L
    return _lib


def _check(code: int) -> None:
    if code != abi.MTDAO_OK:
        raise abi.MtdaoError(code, lib().mtdao_last_error(None).decode())


def _check_adamw(code: int, h) -> None:
    if code != abi.MTDAO_OK:
        raise abi.MtdaoError(code, lib().mtdao_adamw_last_error(h).decode())


def mtdao_adamw_workspace_bytes(cfg: AdamwConfig, tensors) -> int:
    out = ctypes.c_size_t(0)
    _check(lib().mtdao_adamw_workspace_bytes(ctypes.byref(cfg), tensors, ctypes.byref(out)))
    return int(out.value)


def mtdao_adamw_init(cfg: AdamwConfig, tensors, workspace: Optional[int], workspace_bytes: int,
                     stream: Optional[int]) -> int:
    h = _VP()
    _check(lib().mtdao_adamw_init(ctypes.byref(cfg), tensors, workspace, int(workspace_bytes), stream, ctypes.byref(h)))
    return int(h.value)


def mtdao_adamw_set_grads(h: int, grads: Sequence[Optional[int]], stream: Optional[int]) -> None:
    arr = (_VP * len(grads))(*grads)
    _check_adamw(lib().mtdao_adamw_set_grads(h, arr, stream), h)


def mtdao_adamw_step(h: int, lr: float, stream: Optional[int]) -> None:
    _check_adamw(lib().mtdao_adamw_step(h, float(lr), stream), h)


def mtdao_adamw_step_count(h: int) -> int:
    return int(lib().mtdao_adamw_step_count(h))


def mtdao_adamw_destroy(h: Optional[int]) -> None:
    lib().mtdao_adamw_destroy(h)


#: An mtdao_peri_norm_args as bytes (PACKED_ARGS.pack(fields in order)), which
#: the calls below take like the structure: filled in one call, it costs a
#: fifth of setting 26 fields.
PACKED_ARGS = struct.Struct("=qqiiiiffqqqqq13Q")


def _args(args):
    return args if isinstance(args, bytes) else ctypes.byref(args)


def mtdao_peri_norm(args, stream: Optional[int]) -> None:
    _check((_lib or lib()).mtdao_peri_norm(_args(args), stream))


def mtdao_peri_norm_backward_workspace_bytes(args) -> int:
    out = ctypes.c_size_t(0)
    _check(lib().mtdao_peri_norm_backward_workspace_bytes(_args(args), ctypes.byref(out)))
    return int(out.value)


def mtdao_peri_norm_backward(args, workspace: Optional[int], workspace_bytes: int, stream: Optional[int]) -> None:
    _check((_lib or lib()).mtdao_peri_norm_backward(_args(args), workspace, workspace_bytes, stream))


def mtdao_quantize8(x: Optional[int], dtype: int, ld: int, q: Optional[Matrix8], qt: Optional[Matrix8],
                    stream: Optional[int]) -> None:
    _check(lib().mtdao_quantize8(x, dtype, int(ld), ctypes.byref(q) if q is not None else None,
                                 ctypes.byref(qt) if qt is not None else None, stream))


def mtdao_product8_workspace_bytes(m: int, n: int, k: int) -> int:
    out = ctypes.c_size_t(0)
    _check(lib().mtdao_product8_workspace_bytes(int(m), int(n), int(k), ctypes.byref(out)))
    return int(out.value)


def mtdao_product8(a: Matrix8, b: Matrix8, c: Optional[int], c_dtype: int, ldc: int, accumulate: bool,
                   workspace: Optional[int], workspace_bytes: int, stream: Optional[int]) -> None:
    _check(lib().mtdao_product8(ctypes.byref(a), ctypes.byref(b), c, c_dtype, int(ldc), int(accumulate), workspace,
                                int(workspace_bytes), stream))


def mtdao_linear8_workspace_bytes(m: int, n: int, k: int):
    """(forward, backward) bytes."""
    f, b = ctypes.c_size_t(0), ctypes.c_size_t(0)
    _check(lib().mtdao_linear8_workspace_bytes(int(m), int(n), int(k), ctypes.byref(f), ctypes.byref(b)))
    return int(f.value), int(b.value)


def mtdao_linear8(x: Optional[int], dtype: int, rows: int, ld: int, w: Matrix8, y: Optional[int], y_dtype: int, ldy: int,
                  workspace: Optional[int], workspace_bytes: int, stream: Optional[int]) -> None:
    _check((_lib or lib()).mtdao_linear8(x, dtype, rows, ld, ctypes.byref(w), y, y_dtype, ldy, workspace, workspace_bytes,
                                         stream))


def mtdao_linear8_backward(dy: Optional[int], x: Optional[int], dtype: int, rows: int, ld_dy: int, ld_x: int, wt: Matrix8,
                           dx: Optional[int], ld_dx: int, dw: Optional[int], ld_dw: int, accumulate: bool,
                           workspace: Optional[int], workspace_bytes: int, stream: Optional[int]) -> None:
    _check((_lib or lib()).mtdao_linear8_backward(dy, x, dtype, rows, ld_dy, ld_x, ctypes.byref(wt), dx, ld_dx, dw, ld_dw,
                                                  accumulate, workspace, workspace_bytes, stream))
