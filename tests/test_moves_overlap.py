"""Which overlaps of tensors the host checks of the moves by data refuse (ttc_moves.cpp, no HIP, no GPU), against every element of small ones:
tests/moves_overlap_driver.cpp, under AddressSanitizer and UndefinedBehaviorSanitizer."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_1603_02297_amd", "csrc")


def test_overlaps_are_refused_where_elements_are_shared(tmp_path):
    exe = str(tmp_path / "overlap_driver")
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Wno-unused-function", "-Wno-unknown-pragmas", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-O0",
                    "-I", os.path.join(ROOT, "include"), "-I", CSRC, os.path.join(ROOT, "tests", "moves_overlap_driver.cpp"),
                    os.path.join(CSRC, "ttc_moves.cpp"), os.path.join(CSRC, "ttc_plan.cpp"), os.path.join(CSRC, "ttc_cache.cpp"), "-static-libasan", "-o", exe], check=True)
    done = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert done.returncode == 0, done.stdout[-3000:] + done.stderr[-3000:]
    assert "overlap driver ok" in done.stdout
