"""Device code of the moves by data that has to be right at every level of optimisation, compiled here and looked at."""
import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")


@pytest.mark.skipif(shutil.which(HIPCC) is None, reason="no hipcc")
@pytest.mark.parametrize("level", ["-O0", "-O3"])
def test_arguments_are_touched_where_the_launch_put_them(tmp_path, level):
    """touch() reads a kernel's arguments by scalar loads: from the segment that the launch filled, never through the address of a private copy, which is
    what the parameter's own address is until the compiler has dropped the copy."""
    text = open(os.path.join(ROOT, "paper_1603_02297_amd", "csrc", "ttc_moves_device.h")).read()
    call = "touch<Args>()" if re.search(r"void touch\(\)", text) else "touch(a)"
    source = tmp_path / "touched.hip"
    source.write_text('#include "ttc_moves_device.h"\nstruct Args { unsigned w[40]; };\n'
                      "__global__ void touched(Args a, unsigned* out) { ttc::%s; if (threadIdx.x == 0) *out = 1; }\n" % call)
    made = tmp_path / "touched.ll"
    subprocess.run([HIPCC, "--offload-arch=gfx950", level, "-std=c++17", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-I", os.path.join(ROOT, "include"),
                    "-I", os.path.join(ROOT, "paper_1603_02297_amd", "csrc"), "-S", "-emit-llvm", "--cuda-device-only", "-x", "hip", str(source), "-o", str(made)],
                   check=True, capture_output=True, timeout=200)
    code = made.read_text()
    assert "asm sideeffect" in code
    assert not re.search(r"addrspacecast .* to ptr addrspace\(4\)", code)
    assert "@llvm.amdgcn.kernarg.segment.ptr()" in code
