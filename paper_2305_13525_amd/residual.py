"""Binding of the residual addition's operators (include/axo_residual.h): argument marshalling only, same names and argument order as the C functions,
matrices as raw device addresses, streams as raw `hipStream_t` values.  By ctypes, and through the extension module _calls, whose functions stand in for
the wrappers below and call them for all but plain arguments."""
from __future__ import annotations

import ctypes
from typing import Optional

from .binding import Problem, _calls, _check, library
from .block import _KINDS, _ref

AXO_NORM_NONE, AXO_NORM_LAYER, AXO_NORM_RMS = 0, 1, 2

# kinds of arguments as in block.py
_SIGNATURES = {
    "axo_fc_add": "pvlvlvivlifvlvlvzv",
    "axo_fc_add_dact": "pvlivlifvlv",
    "axo_resnorm_fwd": "pvlvliivvvfivvfvlvlvv",
    "axo_resnorm_bwd": "pvlvlvlvliivvvfivvvlvlvvvvvivzv",
}

_quick = _calls if hasattr(_calls, "bind_residual") else None  # a module of an older build, or none, has not these functions
_ready = None


def _lib():
    global _ready
    if _ready is None:
        L = library()
        for name, kinds in _SIGNATURES.items():
            getattr(L, name).argtypes = [_KINDS[k] for k in kinds]
            getattr(L, name).restype = ctypes.c_int
        for name in ("axo_fc_add_workspace_bytes", "axo_resnorm_workspace_bytes"):
            getattr(L, name).argtypes = [_KINDS["p"]]
            getattr(L, name).restype = ctypes.c_size_t
        if _quick is not None:
            _quick.bind_residual({name: ctypes.cast(getattr(L, name), ctypes.c_void_p).value for name in _SIGNATURES}, L.axo_version())
        _ready = L
    return _ready


def axo_fc_add_workspace_bytes(p: Problem) -> int:
    return int(_lib().axo_fc_add_workspace_bytes(_ref(p)))


def axo_resnorm_workspace_bytes(p: Problem) -> int:
    return int(_lib().axo_resnorm_workspace_bytes(_ref(p)))


def axo_fc_add(p: Problem, X: int, ldx: int, W: int, ldw: int, bias: Optional[int], epilogue: int, R: Optional[int], ldr: int, type: int, scale: float,
               Z: Optional[int], ldz: int, Y: int, ldy: int, ws: Optional[int] = None, ws_bytes: int = 0, stream: Optional[int] = None,
               check: bool = True) -> int:
    rc = _lib().axo_fc_add(_ref(p), X, ldx, W, ldw, bias, epilogue, R, ldr, type, scale, Z, ldz, Y, ldy, ws, ws_bytes, stream)
    return _check(rc, "axo_fc_add", check)


def axo_fc_add_dact(p: Problem, dY: int, lddy: int, type: int, Z: Optional[int], ldz: int, epilogue: int, scale: float, dZ: int, lddz: int,
                    stream: Optional[int] = None, check: bool = True) -> int:
    rc = _lib().axo_fc_add_dact(_ref(p), dY, lddy, type, Z, ldz, epilogue, scale, dZ, lddz, stream)
    return _check(rc, "axo_fc_add_dact", check)


def axo_resnorm_fwd(p: Problem, B: int, ldb: int, X: int, ldx: int, type: int, norm_a: int, gamma_a: Optional[int], beta_a: Optional[int],
                    gate: Optional[int], scale: float, norm_b: int, gamma_b: Optional[int], beta_b: Optional[int], eps: float, S: int, lds: int, Y: int,
                    ldy: int, stats: Optional[int], stream: Optional[int] = None, check: bool = True) -> int:
    rc = _lib().axo_resnorm_fwd(_ref(p), B, ldb, X, ldx, type, norm_a, gamma_a, beta_a, gate, scale, norm_b, gamma_b, beta_b, eps, S, lds, Y, ldy, stats, stream)
    return _check(rc, "axo_resnorm_fwd", check)


def axo_resnorm_bwd(p: Problem, dY: int, lddy: int, dS: Optional[int], ldds: int, B: int, ldb: int, S: int, lds: int, type: int, norm_a: int,
                    gamma_a: Optional[int], beta_a: Optional[int], gate: Optional[int], scale: float, norm_b: int, gamma_b: Optional[int], stats: int,
                    dX: int, lddx: int, dB: int, lddb: int, dgamma_a: Optional[int], dbeta_a: Optional[int], dgate: Optional[int],
                    dgamma_b: Optional[int], dbeta_b: Optional[int], accumulate: int = 0, ws: Optional[int] = None, ws_bytes: int = 0,
                    stream: Optional[int] = None, check: bool = True) -> int:
    rc = _lib().axo_resnorm_bwd(_ref(p), dY, lddy, dS, ldds, B, ldb, S, lds, type, norm_a, gamma_a, beta_a, gate, scale, norm_b, gamma_b, stats, dX, lddx, dB, lddb,
                                dgamma_a, dbeta_a, dgate, dgamma_b, dbeta_b, accumulate, ws, ws_bytes, stream)
    return _check(rc, "axo_resnorm_bwd", check)


_WRAPPERS = {name: globals()[name] for name in _SIGNATURES}
if _quick is not None:
    _quick.set_up_residual(Problem, _WRAPPERS, _check)
    globals().update({name: getattr(_quick, name) for name in _SIGNATURES})
