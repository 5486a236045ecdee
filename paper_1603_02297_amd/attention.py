"""ctypes binding of the heads and the attention: the same names as the C ABI in include/ttc_attention.h, argument marshalling only.
Tensors are passed as device addresses (tensor.data_ptr(), 0 or None where the C side takes NULL), streams as hipStream_t integers; the
caller keeps every tensor alive until the stream has run."""
from __future__ import annotations

import ctypes
from typing import Optional, Sequence

from . import binding
from .binding import TtcError, lib, ttc_last_status
from .moves import _Address, _checked, _failed, _fast as _moves_fast, _size

TTC_HEADS_MAX_DIM, TTC_HEADS_MAX_ROTATED, TTC_ATTEND_MAX_DIM = 512, 256, 256

ATTENTION_EXPORTS = (
    "ttc_heads_create", "ttc_heads_destroy", "ttc_heads_rotate", "ttc_heads_workspace", "ttc_heads_rotate_grad", "ttc_pages_append",
    "ttc_attend_create", "ttc_attend_destroy", "ttc_attend_workspace", "ttc_attend_pages",
)

__all__ = [*ATTENTION_EXPORTS, "ATTENTION_EXPORTS", "TTC_HEADS_MAX_DIM", "TTC_HEADS_MAX_ROTATED", "TTC_ATTEND_MAX_DIM"]

# the calls that enqueue work, by their numbers in the CPython form's table
_CALLS = {"ttc_heads_rotate": 7, "ttc_heads_rotate_grad": 8, "ttc_pages_append": 9, "ttc_attend_pages": 10}
_fast = _moves_fast if all(hasattr(_moves_fast, name) for name in _CALLS) else None      # not built, or of an older source


def _declare(L: ctypes.CDLL) -> None:
    vp, ret, i, n, f = _Address, ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_float
    for name, restype, argtypes in (
            ("ttc_heads_create", ret, [i, n, n, n, n, i, ctypes.POINTER(ctypes.c_double), i, f]), ("ttc_heads_destroy", i, [vp]),
            ("ttc_heads_rotate", i, [vp, n, vp, vp, n, vp, n, vp, vp, vp, n, vp, n, vp]),
            ("ttc_heads_workspace", n, [vp, n]),
            ("ttc_heads_rotate_grad", i, [vp, n, vp, vp, n, vp, n, vp, n, vp, n, vp, vp, vp, n, vp, n, vp, vp, vp, vp]),
            ("ttc_pages_append", i, [vp, vp, n, vp, vp, vp, n, vp, n, vp, n, vp, vp, vp, n, vp, vp, vp, vp, vp]),
            ("ttc_attend_create", ret, [vp, n, ctypes.c_double, n]), ("ttc_attend_destroy", i, [vp]),
            ("ttc_attend_workspace", n, [vp, n, n, n]),
            ("ttc_attend_pages", i, [vp, n, n, vp, n, vp, vp, vp, n, vp, vp, vp, vp, vp, n, vp, vp, vp])):
        g = getattr(L, name)
        g.restype, g.argtypes = restype, argtypes
    if _fast is not None:
        for name, k in _CALLS.items():
            _fast.bind_move(k, ctypes.cast(getattr(L, name), ret).value)


binding._on_load.append(_declare)


def ttc_heads_create(dtype: int, q_heads: int, kv_heads: int, dim: int, rotated: int = 0, paired: int = 0, angles: Optional[Sequence[float]] = None,
                     norm: int = 0, eps: float = 1e-6) -> int:
    """Returns the handle (an integer address).  angles: radians for each position, rotated/2 of them.  Raises TtcError when the library refuses."""
    if angles is not None and len(angles) != int(rotated) // 2:
        raise ValueError(f"{len(angles)} angles for {rotated} rotated elements: one for each two of them")
    a = None if angles is None else (ctypes.c_double * max(len(angles), 1))(*[float(x) for x in angles])
    h = lib().ttc_heads_create(int(dtype), int(q_heads), int(kv_heads), int(dim), int(rotated), int(paired), a, int(norm), float(eps))
    if not h:
        raise TtcError(ttc_last_status(), "ttc_heads_create")
    return h


def ttc_heads_destroy(heads: Optional[int]) -> None:
    lib().ttc_heads_destroy(heads)


def ttc_heads_rotate(heads: int, tokens: int, positions: Optional[int], q: Optional[int], ldq: int, k: Optional[int], ldk: int, q_weight: Optional[int],
                     k_weight: Optional[int], q_out: Optional[int], ld_qo: int, k_out: Optional[int], ld_ko: int, stream: Optional[int] = None) -> None:
    """Norms of queries and keys for each head, and their rotation by position."""
    _checked(lib().ttc_heads_rotate(heads, tokens, positions, q, ldq, k, ldk, q_weight, k_weight, q_out, ld_qo, k_out, ld_ko, stream or None), "ttc_heads_rotate")


def ttc_heads_workspace(heads: int, tokens: int) -> int:
    """Bytes of workspace for ttc_heads_rotate_grad."""
    return _size(lib().ttc_heads_workspace(heads, int(tokens)), "ttc_heads_workspace")


def ttc_heads_rotate_grad(heads: int, tokens: int, positions: Optional[int], dq_out: Optional[int], ld_dqo: int, dk_out: Optional[int], ld_dko: int,
                          q: Optional[int], ldq: int, k: Optional[int], ldk: int, q_weight: Optional[int], k_weight: Optional[int], dq: Optional[int], ld_dq: int,
                          dk: Optional[int], ld_dk: int, dq_weight: Optional[int], dk_weight: Optional[int], workspace: Optional[int],
                          stream: Optional[int] = None) -> None:
    """Gradients of ttc_heads_rotate with respect to queries, keys and both weights."""
    _checked(lib().ttc_heads_rotate_grad(heads, tokens, positions, dq_out, ld_dqo, dk_out, ld_dko, q, ldq, k, ldk, q_weight, k_weight, dq, ld_dq, dk, ld_dk,
                                         dq_weight, dk_weight, workspace, stream or None), "ttc_heads_rotate_grad")


def ttc_pages_append(pages: int, heads: int, tokens: int, slots: int, positions: Optional[int], q: Optional[int], ldq: int, k: int, ldk: int, v: int, ldv: int,
                     q_weight: Optional[int], k_weight: Optional[int], q_out: Optional[int], ld_qo: int, k_cache: int, v_cache: int,
                     k_scale: Optional[int] = None, v_scale: Optional[int] = None, stream: Optional[int] = None) -> None:
    """The same on the way into the cache, values with the keys."""
    _checked(lib().ttc_pages_append(pages, heads, tokens, slots, positions, q, ldq, k, ldk, v, ldv, q_weight, k_weight, q_out, ld_qo, k_cache, v_cache,
                                    k_scale, v_scale, stream or None), "ttc_pages_append")


def ttc_attend_create(pages: int, q_heads: int, scale: float, window: int = 0) -> int:
    """Returns the handle.  window: positions that a query sees, its own among them; 0: all before it."""
    h = lib().ttc_attend_create(pages, int(q_heads), float(scale), int(window))
    if not h:
        raise TtcError(ttc_last_status(), "ttc_attend_create")
    return h


def ttc_attend_destroy(attend: Optional[int]) -> None:
    lib().ttc_attend_destroy(attend)


def ttc_attend_workspace(attend: int, requests: int, tokens: int, ld_table: int) -> int:
    """Bytes of workspace for ttc_attend_pages."""
    return _size(lib().ttc_attend_workspace(attend, int(requests), int(tokens), int(ld_table)), "ttc_attend_workspace")


def ttc_attend_pages(attend: int, requests: int, tokens: int, q: int, ldq: int, starts: int, cached: int, table: int, ld_table: int, k_cache: int, v_cache: int,
                     k_scale: Optional[int], v_scale: Optional[int], out: int, ldo: int, lse: Optional[int], workspace: Optional[int],
                     stream: Optional[int] = None) -> None:
    """Attention of packed new tokens over the pages of their requests."""
    _checked(lib().ttc_attend_pages(attend, requests, tokens, q, ldq, starts, cached, table, ld_table, k_cache, v_cache, k_scale, v_scale, out, ldo, lse,
                                    workspace, stream or None), "ttc_attend_pages")


_ctypes_forms = {name: globals()[name] for name in _CALLS}

if _fast is not None:                       # the same without ctypes' conversions: plain ints go straight to the library, the rest as above
    for _name, _k in _CALLS.items():
        _fast.bind_move(_k, _ctypes_forms[_name], _failed(_name))
        globals()[_name] = getattr(_fast, _name)
