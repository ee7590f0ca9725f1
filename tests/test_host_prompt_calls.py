"""What tkv_prefill_attention, tkv_quantize_rows and tkv_head_distortion launch and refuse, under AddressSanitizer and
UndefinedBehaviorSanitizer: csrc/tkv_host_prompt.cpp with tests/host_prompt_calls_driver.cpp by the host compiler, launchers stubbed out."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.skipif(shutil.which("g++") is None, reason="no host compiler")
def test_calls_are_launched_or_refused(tmp_path):
    exe = str(tmp_path / "host_prompt_calls")
    csrc = os.path.join(ROOT, "paper_2605_17170_amd", "csrc")
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-static-libasan", "-Wall",
           "-I", os.path.join(ROOT, "include"), "-I", csrc, os.path.join(ROOT, "tests", "host_prompt_calls_driver.cpp"),
           os.path.join(csrc, "tkv_host_prompt.cpp"), "-o", exe]
    subprocess.run(cmd, check=True, capture_output=True, text=True)
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:verify_asan_link_order=0", UBSAN_OPTIONS="print_stacktrace=1")
    res = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=120)
    assert res.returncode == 0, res.stdout + res.stderr
    assert "host prompt calls ok" in res.stdout
