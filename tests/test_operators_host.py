"""The entry points beside the routed attention (paper_2607_20125_amd/csrc/hc_ops.cpp) on the CPU:
tests/c/ops_check.cpp compiles them against a HIP runtime in host memory (tests/c/fake_hip.h) and
checks what they refuse and what they hand to the kernels; and the refusals of the Python binding."""
import ctypes
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2607_20125_amd", "csrc")
HIP = "/opt/rocm/include"


@pytest.fixture(scope="module")
def ops_check(tmp_path_factory):
    if shutil.which("g++") is None or not os.path.isdir(HIP):
        pytest.skip("g++ or the HIP headers are not available")
    exe = tmp_path_factory.mktemp("ops") / "ops_check"
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-Wall", "-Wextra", "-Werror",
           "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
           "-D__HIP_PLATFORM_AMD__", "-isystem", HIP, "-I", CSRC, "-I", os.path.join(ROOT, "include"),
           os.path.join(ROOT, "tests", "c", "ops_check.cpp"), os.path.join(CSRC, "hc_ops.cpp"),
           os.path.join(CSRC, "hc_runtime.cpp"), "-o", str(exe)]
    res = subprocess.run(cmd, capture_output=True, text=True)
    assert res.returncode == 0, res.stderr
    return str(exe)


@pytest.mark.parametrize("check", ["rotate_refusals", "packed_refusals", "cache_refusals", "unit_rooms", "devices"])
def test_entry_points(ops_check, check):
    run = subprocess.run([ops_check, check], capture_output=True, text=True, timeout=120,
                         env=dict(os.environ, ASAN_OPTIONS="detect_leaks=0"))
    assert run.returncode == 0, run.stdout + run.stderr
    assert f"{check}: ok" in run.stdout


def test_structures_match_the_header(tmp_path):
    """Sizes and the last field's offset of every argument structure, from a C compiler."""
    from paper_2607_20125_amd import headcast as hc
    pairs = {"hc_rotate_tensor": hc.HCRotateTensor, "hc_rotate_args": hc.HCRotateArgs,
             "hc_packed_args": hc.HCPackedArgs, "hc_qcache": hc.HCQCache,
             "hc_qcache_rows": hc.HCQCacheRows, "hc_qcache_attention_args": hc.HCQCacheAttentionArgs}
    lines, want = [], []
    for name, kind in pairs.items():
        lines.append(f'printf("{name} %zu\\n", sizeof({name}));')
        want.append(f"{name} {ctypes.sizeof(kind)}")
        for field, _ in kind._fields_:
            lines.append(f'printf("{name}.{field} %zu\\n", offsetof({name}, {field}));')
            want.append(f"{name}.{field} {getattr(kind, field).offset}")
    src = tmp_path / "sizes.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "headcast.h"\nint main(void) {\n'
                   + "\n".join(lines) + "\nreturn 0;\n}\n")
    exe = tmp_path / "sizes"
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    got = subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split("\n")
    assert got[:-1] == want


def test_binding_refuses_tensors_that_do_not_fit():
    import torch
    from paper_2607_20125_amd import headcast as hc
    ctx = hc.Context.__new__(hc.Context)          # no device is needed for these
    ctx._h, ctx.device, ctx.cfg = ctypes.c_void_p(), 0, hc.default_config()
    x = torch.zeros(4, 2, 64, dtype=torch.bfloat16)
    cu = torch.tensor([0, 4], dtype=torch.int32)
    with pytest.raises(ValueError, match="on cuda:0"):
        ctx.rotate(x, axis_dims=(24, 20, 20))
    with pytest.raises(ValueError, match="on cuda:0"):
        ctx.packed_attention(x, x, x, cu)
    with pytest.raises(ValueError, match="one tensor or a pair"):
        ctx.rotate((x, x, x), axis_dims=(64,))
    with pytest.raises(ValueError, match="axis_dims"):
        ctx.rotate(x, axis_dims=())
    with pytest.raises(ValueError, match="capacity"):
        hc.QCache(1, 1, 64, 0, "cpu")
    with pytest.raises(hc.HeadCastError):
        hc.QCache(1, 1, 96, 10, "cpu")
    cache = hc.QCache(2, 3, 64, 65, "cpu")
    assert cache.data.numel() == 2 * 3 * 2 * 64 * 2 * 34
