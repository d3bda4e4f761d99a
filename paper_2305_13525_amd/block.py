"""Binding of layer norm and the gated feed-forward block (include/axo_block.h): argument marshalling only, same names and argument order as
the C functions, matrices as raw device addresses, streams as raw `hipStream_t` values.  By ctypes, and through the extension module _calls,
whose functions stand in for the wrappers below and call them for all but plain arguments."""
from __future__ import annotations

import ctypes
from typing import Optional, Tuple

from .binding import Problem, _calls, _check, library

AXO_TYPE_BF16, AXO_TYPE_F32 = 0, 1
AXO_GATE_SILU, AXO_GATE_GELU_TANH, AXO_GATE_GELU_ERF = 0, 1, 2
AXO_GATED_OP_FWD, AXO_GATED_OP_DGRAD_ACT, AXO_GATED_OP_DGRAD, AXO_GATED_OP_WGRAD = 0, 1, 2, 3

# kinds of arguments: p problem, v pointer, l int64_t, i int, f float, z size_t
_SIGNATURES = {
    "axo_norm_fwd": "pvlvlivvfvlvlvv",
    "axo_norm_part": "pvlvlivlvv",
    "axo_norm_apply": "pvlivivvfvlvv",
    "axo_norm_bwd": "pvlvlvlivvvlvvivzv",
    "axo_norm_bwd_part": "pvlvlivvvvvivzv",
    "axo_norm_bwd_apply": "pvlvlvlivvvvlv",
    "axo_gated_fwd": "pvlvvlvvivvlvlvzv",
    "axo_gated_act": "pvvlivlv",
    "axo_gated_dact": "pvlvvlivvlv",
    "axo_gated_dgrad_act": "pvlvlvvlivvlvzv",
    "axo_gated_dgrad": "pvvlvvlvlvzv",
    "axo_gated_wgrad": "pvlvvlvvlvzv",
    "axo_gated_wgrad_acc": "pvlvvlvvlvzv",
}
_KINDS = {"p": ctypes.POINTER(Problem), "v": ctypes.c_void_p, "l": ctypes.c_int64, "i": ctypes.c_int, "f": ctypes.c_float, "z": ctypes.c_size_t}

_quick = _calls if hasattr(_calls, "bind_block") else None  # a module of an older build, or none, has not these functions
_ready = None


def _lib():
    global _ready
    if _ready is None:
        L = library()
        for name, kinds in _SIGNATURES.items():
            getattr(L, name).argtypes = [_KINDS[k] for k in kinds]
            getattr(L, name).restype = ctypes.c_int
        for name in ("axo_norm_workspace_bytes", "axo_gated_workspace_bytes"):
            getattr(L, name).argtypes = [_KINDS["p"]]
            getattr(L, name).restype = ctypes.c_size_t
        L.axo_gated_tiles.argtypes = [_KINDS["p"], ctypes.c_int] + 3 * [ctypes.POINTER(ctypes.c_int)]
        L.axo_gated_tiles.restype = ctypes.c_int
        if _quick is not None:
            _quick.bind_block({name: ctypes.cast(getattr(L, name), ctypes.c_void_p).value for name in _SIGNATURES}, L.axo_version())
        _ready = L
    return _ready


def _ref(p: Optional[Problem]):
    return ctypes.byref(p) if p is not None else None


def axo_norm_workspace_bytes(p: Problem) -> int:
    return int(_lib().axo_norm_workspace_bytes(_ref(p)))


def axo_gated_workspace_bytes(p: Problem) -> int:
    return int(_lib().axo_gated_workspace_bytes(_ref(p)))


def axo_gated_tiles(p: Problem, op: int, check: bool = True) -> Tuple[int, Tuple[int, int, int]]:
    """(status, (rows, columns, workgroups per tile)) of the tiles that a product runs on."""
    out = [ctypes.c_int(0) for _ in range(3)]
    rc = _lib().axo_gated_tiles(_ref(p), op, *[ctypes.byref(o) for o in out])
    return _check(rc, "axo_gated_tiles", check), tuple(o.value for o in out)


def axo_norm_fwd(p: Problem, X: int, ldx: int, R: Optional[int], ldr: int, type: int, gamma: Optional[int], beta: Optional[int], eps: float,
                 S: Optional[int], lds: int, Y: int, ldy: int, stats: Optional[int], stream: Optional[int] = None, check: bool = True) -> int:
    rc = _lib().axo_norm_fwd(_ref(p), X, ldx, R, ldr, type, gamma, beta, eps, S, lds, Y, ldy, stats, stream)
    return _check(rc, "axo_norm_fwd", check)


def axo_norm_part(p: Problem, X: int, ldx: int, R: Optional[int], ldr: int, type: int, S: Optional[int], lds: int, part: int,
                  stream: Optional[int] = None, check: bool = True) -> int:
    rc = _lib().axo_norm_part(_ref(p), X, ldx, R, ldr, type, S, lds, part, stream)
    return _check(rc, "axo_norm_part", check)


def axo_norm_apply(p: Problem, S: int, lds: int, type: int, parts: int, n_parts: int, gamma: Optional[int], beta: Optional[int], eps: float,
                   Y: int, ldy: int, stats: Optional[int], stream: Optional[int] = None, check: bool = True) -> int:
    rc = _lib().axo_norm_apply(_ref(p), S, lds, type, parts, n_parts, gamma, beta, eps, Y, ldy, stats, stream)
    return _check(rc, "axo_norm_apply", check)


def axo_norm_bwd(p: Problem, dY: int, lddy: int, S: int, lds: int, R: Optional[int], ldr: int, type: int, gamma: Optional[int], stats: int,
                 dX: int, lddx: int, dgamma: Optional[int], dbeta: Optional[int], accumulate: int = 0, ws: Optional[int] = None,
                 ws_bytes: int = 0, stream: Optional[int] = None, check: bool = True) -> int:
    rc = _lib().axo_norm_bwd(_ref(p), dY, lddy, S, lds, R, ldr, type, gamma, stats, dX, lddx, dgamma, dbeta, accumulate, ws, ws_bytes, stream)
    return _check(rc, "axo_norm_bwd", check)


def axo_norm_bwd_part(p: Problem, dY: int, lddy: int, S: int, lds: int, type: int, gamma: Optional[int], stats: int, sums: int,
                      dgamma: Optional[int], dbeta: Optional[int], accumulate: int = 0, ws: Optional[int] = None, ws_bytes: int = 0,
                      stream: Optional[int] = None, check: bool = True) -> int:
    rc = _lib().axo_norm_bwd_part(_ref(p), dY, lddy, S, lds, type, gamma, stats, sums, dgamma, dbeta, accumulate, ws, ws_bytes, stream)
    return _check(rc, "axo_norm_bwd_part", check)


def axo_norm_bwd_apply(p: Problem, dY: int, lddy: int, S: int, lds: int, R: Optional[int], ldr: int, type: int, gamma: Optional[int],
                       stats: int, sums: int, dX: int, lddx: int, stream: Optional[int] = None, check: bool = True) -> int:
    rc = _lib().axo_norm_bwd_apply(_ref(p), dY, lddy, S, lds, R, ldr, type, gamma, stats, sums, dX, lddx, stream)
    return _check(rc, "axo_norm_bwd_apply", check)


def axo_gated_fwd(p: Problem, X: int, ldx: int, Wg: int, Wu: int, ldw: int, bg: Optional[int], bu: Optional[int], gate: int,
                  G: Optional[int], U: Optional[int], ldz: int, H: int, ldh: int, ws: Optional[int] = None, ws_bytes: int = 0,
                  stream: Optional[int] = None, check: bool = True) -> int:
    rc = _lib().axo_gated_fwd(_ref(p), X, ldx, Wg, Wu, ldw, bg, bu, gate, G, U, ldz, H, ldh, ws, ws_bytes, stream)
    return _check(rc, "axo_gated_fwd", check)


def axo_gated_act(p: Problem, G: int, U: int, ldz: int, gate: int, H: int, ldh: int, stream: Optional[int] = None, check: bool = True) -> int:
    rc = _lib().axo_gated_act(_ref(p), G, U, ldz, gate, H, ldh, stream)
    return _check(rc, "axo_gated_act", check)


def axo_gated_dact(p: Problem, dH: int, lddh: int, G: int, U: int, ldz: int, gate: int, dG: int, dU: int, lddz: int,
                   stream: Optional[int] = None, check: bool = True) -> int:
    rc = _lib().axo_gated_dact(_ref(p), dH, lddh, G, U, ldz, gate, dG, dU, lddz, stream)
    return _check(rc, "axo_gated_dact", check)


def axo_gated_dgrad_act(p: Problem, dY: int, lddy: int, W: int, ldw: int, G: int, U: int, ldz: int, gate: int, dG: int, dU: int, lddz: int,
                        ws: Optional[int] = None, ws_bytes: int = 0, stream: Optional[int] = None, check: bool = True) -> int:
    rc = _lib().axo_gated_dgrad_act(_ref(p), dY, lddy, W, ldw, G, U, ldz, gate, dG, dU, lddz, ws, ws_bytes, stream)
    return _check(rc, "axo_gated_dgrad_act", check)


def axo_gated_dgrad(p: Problem, dG: int, dU: int, lddz: int, Wg: int, Wu: int, ldw: int, dX: int, lddx: int, ws: Optional[int] = None,
                    ws_bytes: int = 0, stream: Optional[int] = None, check: bool = True) -> int:
    rc = _lib().axo_gated_dgrad(_ref(p), dG, dU, lddz, Wg, Wu, ldw, dX, lddx, ws, ws_bytes, stream)
    return _check(rc, "axo_gated_dgrad", check)


def axo_gated_wgrad(p: Problem, X: int, ldx: int, dG: int, dU: int, lddz: int, dWg: int, dWu: int, lddw: int, ws: Optional[int] = None,
                    ws_bytes: int = 0, stream: Optional[int] = None, check: bool = True) -> int:
    rc = _lib().axo_gated_wgrad(_ref(p), X, ldx, dG, dU, lddz, dWg, dWu, lddw, ws, ws_bytes, stream)
    return _check(rc, "axo_gated_wgrad", check)


def axo_gated_wgrad_acc(p: Problem, X: int, ldx: int, dG: int, dU: int, lddz: int, dWg: int, dWu: int, lddw: int, ws: Optional[int] = None,
                        ws_bytes: int = 0, stream: Optional[int] = None, check: bool = True) -> int:
    rc = _lib().axo_gated_wgrad_acc(_ref(p), X, ldx, dG, dU, lddz, dWg, dWu, lddw, ws, ws_bytes, stream)
    return _check(rc, "axo_gated_wgrad_acc", check)


_WRAPPERS = {name: globals()[name] for name in _SIGNATURES}
if _quick is not None:
    _quick.set_up_block(Problem, _WRAPPERS, _check)
    globals().update({name: getattr(_quick, name) for name in _SIGNATURES})
