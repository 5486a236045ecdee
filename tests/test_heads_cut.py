"""How heads are cut into lanes' units (ttc_attention.cpp, cut_heads), on the CPU through tests/heads_cut_driver.cpp."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_1603_02297_amd", "csrc")


def test_lanes_have_what_the_kernels_take_as_theirs(tmp_path):
    exe = str(tmp_path / "heads_cut_driver")
    sources = [os.path.join(ROOT, "tests", "heads_cut_driver.cpp"), *(os.path.join(CSRC, s) for s in ("ttc_attention.cpp", "ttc_moves.cpp", "ttc_plan.cpp", "ttc_cache.cpp"))]
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Wno-unused-function", "-Wno-unknown-pragmas", "-O2", "-I", os.path.join(ROOT, "include"), "-I", CSRC, *sources, "-o", exe], check=True)
    done = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert done.returncode == 0, done.stdout[-3000:] + done.stderr[-3000:]
    assert "heads cut ok" in done.stdout
