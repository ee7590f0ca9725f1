"""The blocks of instructions in csrc/tkv_prefill.hip that write M0, which the compiler may have set for instructions of its own, tell it so."""
import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")


@pytest.mark.skipif(shutil.which(HIPCC) is None, reason="no hipcc")
def test_blocks_that_write_m0_say_so(tmp_path):
    csrc, to = os.path.join(ROOT, "paper_2605_17170_amd", "csrc"), str(tmp_path / "prefill.ll")
    subprocess.run([HIPCC, "-x", "hip", "--cuda-device-only", "-S", "-emit-llvm", os.path.join(csrc, "tkv_prefill.hip"), "-o", to, "-O1", "-std=c++17",
                    "--offload-arch=gfx950", "-I", os.path.join(ROOT, "include"), "-I", csrc], check=True, capture_output=True, text=True)
    blocks = [m for m in re.findall(r'asm sideeffect "([^"]*)", "([^"]*)"', open(to).read()) if re.search(r"s_\w+ m0,", m[0])]
    assert blocks
    for text, constraints in blocks:
        assert "~{m0}" in constraints, text
