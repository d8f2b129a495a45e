"""Calls without tokens, on the CPU (tests/c/empty_check.cpp)."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2607_20125_amd", "csrc")
HIP = "/opt/rocm/include"


def test_calls_without_tokens(tmp_path):
    if shutil.which("g++") is None or not os.path.isdir(HIP):
        pytest.skip("g++ or the HIP headers are not available")
    exe = tmp_path / "empty_check"
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-Wall", "-Wextra", "-Werror", "-fsanitize=address,undefined",
           "-fno-sanitize-recover=all", "-D__HIP_PLATFORM_AMD__", "-isystem", HIP, "-I", CSRC, "-I", os.path.join(ROOT, "include"),
           os.path.join(ROOT, "tests", "c", "empty_check.cpp")]
    cmd += [os.path.join(CSRC, f) for f in ("hc_ops.cpp", "hc_window.cpp", "hc_runtime.cpp")] + ["-o", str(exe)]
    res = subprocess.run(cmd, capture_output=True, text=True)
    assert res.returncode == 0, res.stderr
    run = subprocess.run([str(exe)], capture_output=True, text=True, timeout=120, env=dict(os.environ, ASAN_OPTIONS="detect_leaks=0"))
    assert run.returncode == 0 and run.stdout == "ok\n", run.stdout + run.stderr
