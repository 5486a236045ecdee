"""include/ttc_attention.h, the library and its binding: the same functions and constants, and the CPython forms refuse as the ctypes forms do."""
import ctypes
import inspect
import os
import re
import shutil
import subprocess
import sysconfig

import pytest

import paper_1603_02297_amd as ttc
from paper_1603_02297_amd import attention, binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "ttc_attention.h")
NUMBERS = {"tokens", "requests"}


def declared():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    return sorted(set(re.findall(r"\b(ttc_[a-z_0-9]+)\s*\(", text)))


def test_the_header_is_exported_and_bound():
    assert sorted(ttc.ATTENTION_EXPORTS) == declared()
    lib = ctypes.CDLL(binding.LIB_PATH)
    for name in declared():
        assert hasattr(lib, name) and callable(getattr(ttc, name))


def test_constants_match_the_header():
    text = open(HEADER).read()
    names = re.findall(r"\b(TTC_[A-Z_]+) = (\d+)", text)
    assert names and all(int(value) == getattr(ttc, name) for name, value in names)
    moves = open(os.path.join(ROOT, "include", "ttc_moves.h")).read()
    assert int(re.search(r"\bTTC_Q4 = (\d+)", moves).group(1)) == ttc.TTC_Q4


def test_the_header_is_plain_c(tmp_path):
    if shutil.which("gcc") is None:
        pytest.skip("no C compiler")
    source = tmp_path / "use.c"
    source.write_text('#include "ttc_attention.h"\nint main(void) { return ttc_heads_destroy(0); }\n')
    subprocess.run(["gcc", "-std=c99", "-pedantic", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), "-c", str(source), "-o", str(tmp_path / "use.o")], check=True)


def test_the_cpython_forms_are_the_ones_in_use():
    if not os.path.exists(os.path.join(sysconfig.get_paths()["include"], "Python.h")) or shutil.which("gcc") is None:
        pytest.skip("no Python headers or no C compiler")
    for name in attention._CALLS:
        assert getattr(ttc, name) is getattr(binding._call, name)


@pytest.mark.parametrize("name", list(attention._CALLS))
def test_arguments_arrive_in_their_places(monkeypatch, name):
    """Both forms hand every argument on as it is; anything but integers, None and addresses never arrives."""
    form = attention._ctypes_forms[name]
    names = list(inspect.signature(form).parameters)
    real = getattr(ttc.lib(), name)
    reached = []
    stand_in = ctypes.CFUNCTYPE(ctypes.c_int, *real.argtypes)(lambda *args: reached.append([getattr(a, "value", a) for a in args]) or 0)
    stand_in.argtypes = real.argtypes
    monkeypatch.setattr(ttc.lib(), name, stand_in)
    args = [16 * (k + 1) for k in range(len(names))]
    fast = getattr(ttc, name)
    if fast is not form:
        attention._fast.bind_move(attention._CALLS[name], ctypes.cast(stand_in, ctypes.c_void_p).value)
    try:
        for f in (form, fast):
            f(*args)
            assert reached.pop() == args
            f(*args[:-1])
            assert [x or 0 for x in reached.pop()] == [*args[:-1], 0]
            for place, p in enumerate(names):
                if p in NUMBERS or p.startswith("ld"):
                    continue
                for bad in ("x", b"x", bytearray(b"x"), 1.5):
                    wrong = list(args)
                    wrong[place] = bad
                    with pytest.raises((TypeError, ctypes.ArgumentError)):
                        f(*wrong)
            with pytest.raises(TypeError):
                f(*args[:3])
        assert not reached
    finally:
        if fast is not form:
            attention._fast.bind_move(attention._CALLS[name], ctypes.cast(real, ctypes.c_void_p).value)
