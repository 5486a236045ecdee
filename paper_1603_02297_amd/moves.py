"""ctypes binding of the moves whose index map is data: the same names as the C ABI in include/ttc_moves.h, argument
marshalling only.  Tensors are passed as device addresses (tensor.data_ptr(), 0 or None where the C side takes NULL), streams as
hipStream_t integers; the caller keeps every tensor alive until the stream has run."""
from __future__ import annotations

import ctypes
from typing import Optional, Sequence

from . import binding
from .binding import TTC_OK, TtcError, lib, ttc_last_status

TTC_BF16, TTC_F16, TTC_F8 = 8, 9, 10
TTC_ROUTE_MAX_EXPERTS, TTC_ROUTE_MAX_TOPK, TTC_ROUTE_MAX_ALIGN = 1024, 64, 65536

MOVE_EXPORTS = (
    "ttc_route_create", "ttc_route_destroy", "ttc_route_rows", "ttc_route_workspace", "ttc_route_sort", "ttc_route_gather",
    "ttc_route_combine", "ttc_route_combine_grad", "ttc_pages_create", "ttc_pages_destroy", "ttc_pages_map", "ttc_pages_write",
    "ttc_pages_read",
)

__all__ = [*MOVE_EXPORTS, "MOVE_EXPORTS", "TTC_BF16", "TTC_F16", "TTC_F8", "TTC_ROUTE_MAX_EXPERTS", "TTC_ROUTE_MAX_TOPK", "TTC_ROUTE_MAX_ALIGN"]

# the calls that enqueue work, in the order of the CPython form's table
_MOVES = ("ttc_route_sort", "ttc_route_gather", "ttc_route_combine", "ttc_route_combine_grad", "ttc_pages_map", "ttc_pages_write", "ttc_pages_read")


class _Address(ctypes.c_void_p):
    """An address: an int, None, a c_void_p, or an object whose _as_parameter_ is one.  ctypes by itself would also take a str, bytes or an array for one and hand on where those lie in
    host memory, which no check of the library can tell from a device address."""

    @classmethod
    def from_param(cls, value):
        value = getattr(value, "_as_parameter_", value)
        if value is None or isinstance(value, (int, ctypes.c_void_p)):
            return ctypes.c_void_p.from_param(value)
        raise TypeError(f"an address is an int or None, not {type(value).__name__}")


def _declare(L: ctypes.CDLL) -> None:
    vp, ret, i, n = _Address, ctypes.c_void_p, ctypes.c_int, ctypes.c_int64
    fp, np = ctypes.POINTER(ctypes.c_float), ctypes.POINTER(ctypes.c_int64)
    for name, restype, argtypes in (
            ("ttc_route_create", ret, [i, n, i, i, n, i, i, fp, fp]), ("ttc_route_destroy", i, [vp]),
            ("ttc_route_rows", n, [vp, n]), ("ttc_route_workspace", n, [vp, n]),
            ("ttc_route_sort", i, [vp, n, vp, n, vp, vp, vp, vp, vp, vp]),
            ("ttc_route_gather", i, [vp, n, vp, n, vp, vp, vp, vp, vp, n, vp]),
            ("ttc_route_combine", i, [vp, n, vp, n, vp, vp, vp, n, vp]),
            ("ttc_route_combine_grad", i, [vp, n, vp, n, vp, n, vp, vp, vp, vp, vp, n, vp, vp]),
            ("ttc_pages_create", ret, [i, i, n, n, n, n, np]), ("ttc_pages_destroy", i, [vp]),
            ("ttc_pages_map", i, [vp, n, vp, vp, vp, vp, n, vp, n, n, vp, vp, vp, vp, vp, vp]),
            ("ttc_pages_write", i, [vp, n, vp, vp, n, vp, n, vp, vp, vp, vp, vp]),
            ("ttc_pages_read", i, [vp, n, vp, vp, vp, vp, vp, vp, n, vp, n, vp])):
        f = getattr(L, name)
        f.restype, f.argtypes = restype, argtypes
    if _fast is not None:
        for k, name in enumerate(_MOVES):
            _fast.bind_move(k, ctypes.cast(getattr(L, name), ret).value)


binding._on_load.append(_declare)
_fast = binding._call if hasattr(binding._call, "bind_move") else None      # not built, or of an older source


def _checked(status: int, where: str) -> None:
    if status != TTC_OK:
        raise TtcError(status, where)


def _size(value: int, where: str) -> int:
    if value < 0:
        raise TtcError(-value, where)
    return value


def ttc_route_create(dtype: int, width: int, topk: int, experts: int, first: int = 0, align: int = 1, id_bytes: int = 8,
                     alpha: Optional[float] = None, beta: Optional[float] = None) -> int:
    """Returns the handle (an integer address).  Raises TtcError when the library refuses."""
    a, b = (None if s is None else ctypes.byref(ctypes.c_float(float(s))) for s in (alpha, beta))
    h = lib().ttc_route_create(int(dtype), int(width), int(topk), int(experts), int(first), int(align), int(id_bytes), a, b)
    if not h:
        raise TtcError(ttc_last_status(), "ttc_route_create")
    return h


def ttc_route_destroy(route: Optional[int]) -> None:
    lib().ttc_route_destroy(route)


def ttc_route_rows(route: int, tokens: int) -> int:
    """Rows of a sorted tensor that suffice for `tokens` tokens."""
    return _size(lib().ttc_route_rows(route, int(tokens)), "ttc_route_rows")


def ttc_route_workspace(route: int, tokens: int) -> int:
    """Bytes of workspace for ttc_route_sort."""
    return _size(lib().ttc_route_workspace(route, int(tokens)), "ttc_route_workspace")


def ttc_route_sort(route: int, tokens: int, ids: int, ld_ids: int, offsets: int, counts: int, position: int, source: Optional[int],
                   workspace: Optional[int], stream: Optional[int] = None) -> None:
    """Ids of the chosen experts -> offsets, counts, position, source (device addresses, int32)."""
    _checked(lib().ttc_route_sort(route, tokens, ids, ld_ids, offsets, counts, position, source, workspace, stream or None), "ttc_route_sort")


def ttc_route_gather(route: int, tokens: int, x: int, ldx: int, weights: Optional[int], position: int, offsets: Optional[int],
                     counts: Optional[int], rows: int, ld_rows: int, stream: Optional[int] = None) -> None:
    """Tokens to their rows, times their weights if there are any."""
    _checked(lib().ttc_route_gather(route, tokens, x, ldx, weights, position, offsets, counts, rows, ld_rows, stream or None), "ttc_route_gather")


def ttc_route_combine(route: int, tokens: int, rows: int, ld_rows: int, weights: Optional[int], position: int, y: int, ldy: int,
                      stream: Optional[int] = None) -> None:
    """Rows back to their tokens, weighted and added up: y <- alpha * sum + beta * y."""
    _checked(lib().ttc_route_combine(route, tokens, rows, ld_rows, weights, position, y, ldy, stream or None), "ttc_route_combine")


def ttc_route_combine_grad(route: int, tokens: int, dy: int, ld_dy: int, rows: Optional[int], ld_rows: int, weights: Optional[int],
                           position: int, offsets: Optional[int], counts: Optional[int], drows: Optional[int], ld_drows: int,
                           dweights: Optional[int], stream: Optional[int] = None) -> None:
    """Gradients of ttc_route_combine with respect to the rows and the weights."""
    _checked(lib().ttc_route_combine_grad(route, tokens, dy, ld_dy, rows, ld_rows, weights, position, offsets, counts, drows, ld_drows,
                                          dweights, stream or None), "ttc_route_combine_grad")


def ttc_pages_create(dtype: int, cache_dtype: int, heads: int, dim: int, page: int, pages: int, strides: Optional[Sequence[int]] = None) -> int:
    """Returns the handle.  strides: elements between neighbouring heads, slots and pages of the cache; None: [dim, heads, page, pages] dense."""
    if strides is not None and len(strides) != 3:
        raise ValueError("strides are three: of a head, of a slot, of a page")
    s = None if strides is None else (ctypes.c_int64 * 3)(*[int(x) for x in strides])
    h = lib().ttc_pages_create(int(dtype), int(cache_dtype), int(heads), int(dim), int(page), int(pages), s)
    if not h:
        raise TtcError(ttc_last_status(), "ttc_pages_create")
    return h


def ttc_pages_destroy(pages: Optional[int]) -> None:
    lib().ttc_pages_destroy(pages)


def ttc_pages_map(pages: int, requests: int, first: Optional[int], cached: int, fresh: int, table: int, ld_table: int, free_list: int,
                  free_count: int, tokens: int, starts: int, page_starts: int, slots: int, positions: Optional[int], owner: Optional[int],
                  stream: Optional[int] = None) -> None:
    """Block tables, packed offsets and slots from request lengths."""
    _checked(lib().ttc_pages_map(pages, requests, first, cached, fresh, table, ld_table, free_list, free_count, tokens, starts, page_starts,
                                 slots, positions, owner, stream or None), "ttc_pages_map")


def ttc_pages_write(pages: int, tokens: int, slots: int, k: int, ldk: int, v: Optional[int], ldv: int, k_cache: int, v_cache: Optional[int],
                    k_scale: Optional[int] = None, v_scale: Optional[int] = None, stream: Optional[int] = None) -> None:
    """Keys and values into their slots of the cache."""
    _checked(lib().ttc_pages_write(pages, tokens, slots, k, ldk, v, ldv, k_cache, v_cache, k_scale, v_scale, stream or None), "ttc_pages_write")


def ttc_pages_read(pages: int, tokens: int, slots: int, k_cache: int, v_cache: Optional[int], k_scale: Optional[int], v_scale: Optional[int],
                   k: int, ldk: int, v: Optional[int], ldv: int, stream: Optional[int] = None) -> None:
    """Keys and values out of their slots of the cache."""
    _checked(lib().ttc_pages_read(pages, tokens, slots, k_cache, v_cache, k_scale, v_scale, k, ldk, v, ldv, stream or None), "ttc_pages_read")


_ctypes_forms = {name: globals()[name] for name in _MOVES}


def _failed(name: str):
    def fail(status: int) -> None:
        raise TtcError(status, name)
    return fail


if _fast is not None:                       # the same without ctypes' conversions: plain ints go straight to the library, the rest as above
    for _k, _name in enumerate(_MOVES):
        _fast.bind_move(_k, _ctypes_forms[_name], _failed(_name))
        globals()[_name] = getattr(_fast, _name)
