"""Addresses of the moves by data: what is no address is refused by the binding, before the library sees it."""
import ctypes
import inspect

import pytest

import paper_1603_02297_amd as ttc
from paper_1603_02297_amd import moves

NUMBERS = {"tokens", "requests", "free_count"}


def addresses(name):
    """The positions of a move's arguments that are addresses: all but counts and leading dimensions."""
    names = list(inspect.signature(moves._ctypes_forms[name]).parameters)
    return names, [k for k, p in enumerate(names) if p not in NUMBERS and not p.startswith("ld")]


@pytest.mark.parametrize("name", moves._MOVES)
def test_only_integers_are_addresses(monkeypatch, name):
    """Every address argument in turn, in both forms; the library's function is never reached."""
    names, places = addresses(name)
    assert len(places) >= 6
    reached = []
    real = getattr(ttc.lib(), name)
    stand_in = ctypes.CFUNCTYPE(ctypes.c_int, *real.argtypes)(lambda *args: reached.append(args) or 0)
    stand_in.argtypes = real.argtypes
    monkeypatch.setattr(ttc.lib(), name, stand_in)
    buffer = ctypes.create_string_buffer(8)
    for form in (moves._ctypes_forms[name], getattr(ttc, name)):
        for place in places:
            for bad in ("x", b"x", buffer, bytearray(b"x"), 1.5, (ctypes.c_int * 3)(), ctypes.byref(buffer)):
                args = [16 * (k + 1) for k in range(len(names))]
                args[place] = bad
                with pytest.raises((TypeError, ctypes.ArgumentError)):
                    form(*args)
    assert not reached


class Tensor:
    _as_parameter_ = 8192


def test_what_was_an_address_still_is():
    for good, value in ((Tensor(), 8192), (None, None), (0, None), (4096, 4096), (True, 1), (ctypes.c_void_p(64), 64), (2 ** 64 - 16, 2 ** 64 - 16)):
        f = ctypes.CFUNCTYPE(ctypes.c_void_p, ctypes.c_void_p)(lambda p: p)
        f.argtypes = [moves._Address]
        assert f(good) == value
    h = ttc.ttc_route_create(ttc.TTC_BF16, 64, 2, 8)
    for form in (moves._ctypes_forms["ttc_route_gather"], ttc.ttc_route_gather):
        with pytest.raises(ttc.TtcError) as e:
            form(ctypes.c_void_p(h), 10, ctypes.c_void_p(64), 63, None, 4096, None, 0, 8192, 64, None)
        assert e.value.status == ttc.TTC_ERR_INVALID_VALUE
        form(h, 0, None, 64, None, None, None, None, None, 64)
    ttc.ttc_route_destroy(ctypes.c_void_p(h))
