"""include/ttc_moves.h, the library and its binding: the same functions, and the CPython forms refuse as the ctypes forms do."""
import ctypes
import os
import re
import shutil
import sysconfig

import pytest

import paper_1603_02297_amd as ttc
from paper_1603_02297_amd import binding, moves

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def declared():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "ttc_moves.h")).read(), flags=re.S)
    return sorted(set(re.findall(r"\b(ttc_[a-z_0-9]+)\s*\(", text)))


def test_the_header_is_exported_and_bound():
    assert sorted(ttc.MOVE_EXPORTS) == declared() and len(declared()) == 13
    lib = ctypes.CDLL(binding.LIB_PATH)
    for name in declared():
        assert hasattr(lib, name) and callable(getattr(ttc, name))


def test_constants_match_the_header():
    text = open(os.path.join(ROOT, "include", "ttc_moves.h")).read()
    for name in ("TTC_BF16", "TTC_F16", "TTC_F8", "TTC_ROUTE_MAX_EXPERTS", "TTC_ROUTE_MAX_TOPK", "TTC_ROUTE_MAX_ALIGN"):
        assert int(re.search(rf"\b{name} = (\d+)", text).group(1)) == getattr(ttc, name)


def test_the_header_is_plain_c(tmp_path):
    if shutil.which("gcc") is None:
        pytest.skip("no C compiler")
    import subprocess
    source = tmp_path / "use.c"
    source.write_text('#include "ttc_moves.h"\nint main(void) { return ttc_route_destroy(0) + ttc_pages_destroy(0); }\n')
    subprocess.run(["gcc", "-std=c99", "-pedantic", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), "-c", str(source), "-o", str(tmp_path / "use.o")], check=True)


def test_the_cpython_forms_are_the_ones_in_use():
    include = sysconfig.get_paths()["include"]
    if not os.path.exists(os.path.join(include, "Python.h")) or shutil.which("gcc") is None:
        pytest.skip("no Python headers or no C compiler")
    for name in moves._MOVES:
        assert getattr(ttc, name) is getattr(binding._call, name)


@pytest.mark.parametrize("args,kwargs", [
    ((None, 10, 64, 64, 0, 4096, 0, 0, 8192, 64, 0), {}), (("h", 10, 0, 64, 0, 4096, 0, 0, 8192, 64), {}), (("h", 10, 64, 64, 0, 4096, 0, 0, 66, 64, None), {}),
    (("h", 10, 64, 63, 0, 4096, 0, 0, 1 << 20, 64), {}), (("h", 10, 64), {}), ((7,), {}), (("h", 10, 64, 64, 0, 4096, 0, 0, 1 << 20, 64, 0, 0), {}), (("h", 1.5, 64, 64, 0, 4096, 0, 0, 1 << 20, 64), {}),
    (("h", "x", 64, 64, 0, 4096, 0, 0, 1 << 20, 64), {}), (("h", -1, 64, 64, None, 4096, None, None, 1 << 20, 64), {}), (("h",), {"tokens": -1, "x": 0, "ldx": 64, "weights": 0, "position": 0, "offsets": 0,
                                                                                                                             "counts": 0, "rows": 0, "ld_rows": 64})])
def test_the_cpython_form_and_the_ctypes_form_refuse_alike(args, kwargs):
    h = ttc.ttc_route_create(ttc.TTC_BF16, 64, 2, 8)
    seen = []
    for f in (ttc.ttc_route_gather, moves._ctypes_forms["ttc_route_gather"]):
        try:
            f(*[h if a == "h" else a for a in args], **kwargs)
            seen.append(None)
        except Exception as e:                      # noqa: BLE001: the type is what is compared
            seen.append((type(e), str(e)))
    assert seen[0] is not None and seen[0] == seen[1]
    assert "HIP" not in seen[0][1]                  # refused by a check of the arguments, not by a launch
    ttc.ttc_route_destroy(h)
