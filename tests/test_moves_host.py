"""The host part of the moves by data (ttc_moves.cpp) built with AddressSanitizer and UndefinedBehaviorSanitizer, no HIP, no GPU, and run
through tests/moves_driver.cpp: sizes at the ends of their types, and what the checks let through."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_1603_02297_amd", "csrc")


def test_host_checks_are_clean_under_asan_and_ubsan(tmp_path):
    exe = str(tmp_path / "moves_driver")
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Wno-unused-function", "-Wno-unknown-pragmas", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
                    "-fno-omit-frame-pointer", "-g", "-O1", "-I", os.path.join(ROOT, "include"), "-I", CSRC, os.path.join(ROOT, "tests", "moves_driver.cpp"),
                    os.path.join(CSRC, "ttc_moves.cpp"), os.path.join(CSRC, "ttc_plan.cpp"), os.path.join(CSRC, "ttc_cache.cpp"), "-static-libasan", "-o", exe], check=True)
    done = subprocess.run([exe], capture_output=True, text=True, timeout=300, env=dict(os.environ, ASAN_OPTIONS="detect_leaks=1", UBSAN_OPTIONS="print_stacktrace=1"))
    assert done.returncode == 0, done.stdout[-3000:] + done.stderr[-3000:]
    assert "moves driver ok" in done.stdout
