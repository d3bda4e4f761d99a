"""Binding of the orthogonalised update (include/axo_update.h): argument marshalling only, same names and argument order as the C functions, matrices as raw device
addresses, streams as raw `hipStream_t` values.  The coefficients, which the C function reads in host memory, are a sequence of numbers."""
from __future__ import annotations

import ctypes
from typing import Optional, Sequence

from .binding import Problem, _check, library

AXO_ORTHO_MOST_STEPS = 64

_ready = None


def _lib():
    global _ready
    if _ready is None:
        L = library()
        vp, i64, i32, sz, fl = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_size_t, ctypes.c_float
        L.axo_ortho.argtypes = [ctypes.POINTER(Problem), vp, i64, i32, i32, ctypes.POINTER(fl), fl, vp, i64, vp, sz, vp]
        L.axo_ortho.restype = i32
        L.axo_ortho_workspace_bytes.argtypes = [ctypes.POINTER(Problem)]
        L.axo_ortho_workspace_bytes.restype = sz
        _ready = L
    return _ready


def _ref(p: Optional[Problem]):
    return ctypes.byref(p) if p is not None else None


def axo_ortho_workspace_bytes(p: Problem) -> int:
    return int(_lib().axo_ortho_workspace_bytes(_ref(p)))


def axo_ortho(p: Problem, G: int, ldg: int, type: int, steps: int, abc: Optional[Sequence[float]], eps: float, O: int, ldo: int, ws: Optional[int] = None,
              ws_bytes: int = 0, stream: Optional[int] = None, check: bool = True) -> int:
    """abc: None, or the 3 * steps coefficients (ValueError for another number of them)."""
    if abc is not None:
        if len(abc) != 3 * steps:
            raise ValueError(f"{len(abc)} coefficients for {steps} steps: three a step")
        abc = (ctypes.c_float * max(1, len(abc)))(*abc)
    rc = _lib().axo_ortho(_ref(p), G, ldg, type, steps, abc, eps, O, ldo, ws, ws_bytes, stream)
    return _check(rc, "axo_ortho", check)
