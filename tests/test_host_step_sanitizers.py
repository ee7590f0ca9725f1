"""csrc/tkv_host_step.cpp (rotation table, plan of shared prefixes, argument checks) under AddressSanitizer and
UndefinedBehaviorSanitizer: compiled with tests/host_step_sanitize_driver.cpp by the host compiler, launchers stubbed out."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.skipif(shutil.which("g++") is None, reason="no host compiler")
def test_host_step_code_runs_clean_under_asan_and_ubsan(tmp_path):
    exe = str(tmp_path / "host_step_sanitize")
    csrc = os.path.join(ROOT, "paper_2605_17170_amd", "csrc")
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-static-libasan", "-Wall",
           "-I", os.path.join(ROOT, "include"), "-I", csrc, os.path.join(ROOT, "tests", "host_step_sanitize_driver.cpp"),
           os.path.join(csrc, "tkv_host.cpp"), os.path.join(csrc, "tkv_host_step.cpp"), "-o", exe]
    subprocess.run(cmd, check=True, capture_output=True, text=True)
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:verify_asan_link_order=0", UBSAN_OPTIONS="print_stacktrace=1")
    res = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=120)
    assert res.returncode == 0, res.stdout + res.stderr
    assert "host step sanitizer run ok" in res.stdout
