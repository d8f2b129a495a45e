"""The entry points of a model with a sliding window (paper_2607_20125_amd/csrc/hc_window.cpp) on the CPU:
tests/c/window_check.cpp compiles them against a HIP runtime in host memory and checks what they refuse and what they
hand to the kernels; and the refusals and structures of the Python binding."""
import ctypes
import os
import shutil
import subprocess

import pytest
import torch

from paper_2607_20125_amd import headcast as hc

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2607_20125_amd", "csrc")
HIP = "/opt/rocm/include"


@pytest.fixture(scope="module")
def window_check(tmp_path_factory):
    if shutil.which("g++") is None or not os.path.isdir(HIP):
        pytest.skip("g++ or the HIP headers are not available")
    exe = tmp_path_factory.mktemp("window") / "window_check"
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-Wall", "-Wextra", "-Werror",
           "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
           "-D__HIP_PLATFORM_AMD__", "-isystem", HIP, "-I", CSRC, "-I", os.path.join(ROOT, "include"),
           os.path.join(ROOT, "tests", "c", "window_check.cpp"), os.path.join(CSRC, "hc_window.cpp"),
           os.path.join(CSRC, "hc_runtime.cpp"), "-o", str(exe)]
    res = subprocess.run(cmd, capture_output=True, text=True)
    assert res.returncode == 0, res.stderr
    return str(exe)


@pytest.mark.parametrize("check", ["norm_refusals", "paged_refusals", "window_refusals", "rooms", "call_devices"])
def test_entry_points(window_check, check):
    run = subprocess.run([window_check, check], capture_output=True, text=True, timeout=120,
                         env=dict(os.environ, ASAN_OPTIONS="detect_leaks=0"))
    assert run.returncode == 0, run.stdout + run.stderr
    assert f"{check}: ok" in run.stdout


def test_structures_match_the_header(tmp_path):
    """Sizes and field offsets of every argument structure, from a C compiler."""
    pairs = {"hc_norm_tensor": hc.HCNormTensor, "hc_norm_args": hc.HCNormArgs, "hc_norm_grad_tensor": hc.HCNormGradTensor,
             "hc_pages": hc.HCPages, "hc_page_table": hc.HCPageTable, "hc_paged_args": hc.HCPagedArgs,
             "hc_window_args": hc.HCWindowArgs, "hc_window_grad_args": hc.HCWindowGradArgs}
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


# --- the binding ------------------------------------------------------------------------------------

@pytest.fixture
def ctx(monkeypatch):
    """A context without a device: its tensors are the CPU's, and a call that is not refused gets as far as the
    library, which has no context and says so."""
    hc._use_torch()
    monkeypatch.setattr(hc, "_raw_stream", lambda device: 0)
    c = hc.Context.__new__(hc.Context)
    c._h, c.device, c.cfg, c._need = ctypes.c_void_p(), -1, hc.default_config(), ctypes.c_int64()
    return c


def rows(n, heads=2, d=64, dtype=torch.bfloat16):
    return torch.zeros(n, heads, d, dtype=dtype)


def ints(*shape):
    return torch.zeros(*shape, dtype=torch.int32)


def taken(call):
    """The call passes the binding's checks and reaches the library."""
    with pytest.raises(hc.HeadCastError):
        call()


def pages(n=3, tokens=16, heads=2, d=64):
    return hc.Pages(*(torch.zeros(n, tokens, heads, d, dtype=torch.bfloat16) for _ in range(2)))


def test_norm_refusals(ctx):
    q, k, o, p = (rows(4) for _ in range(4))
    w = torch.ones(64)
    kw = dict(axis_dims=(64,), positions=ints(1, 4))
    taken(lambda: ctx.norm_rotate(q, w, **kw))
    taken(lambda: ctx.norm_rotate(q, None, **kw))
    taken(lambda: ctx.norm_rotate((q, k), (w, w), (q, k), **kw))
    for weight in (torch.ones(65), torch.ones(64, dtype=torch.float16), torch.ones(128)[::2], torch.ones(1, 64)):
        with pytest.raises(ValueError, match="weight"):
            ctx.norm_rotate(q, weight, **kw)
    with pytest.raises(ValueError, match="weight"):              # of two types
        ctx.norm_rotate((q, k), (w, w.bfloat16()), **kw)
    with pytest.raises(ValueError, match="as many weights"):
        ctx.norm_rotate((q, k), (w,), **kw)
    with pytest.raises(ValueError, match="pair"):
        ctx.norm_rotate((q, rows(5)), (w, w), **kw)
    for xs, outs in (((q, q), (q, q)), ((q, k), (k, q)), ((q, k), (o, o)), ((q, k), (o, q))):
        with pytest.raises(ValueError, match="overlap"):
            ctx.norm_rotate(xs, (w, w), outs, **kw)
    with pytest.raises(ValueError, match="requires a gradient"):
        ctx.norm_rotate(q, w.clone().requires_grad_(), **kw)
    with pytest.raises(ValueError, match="requires a gradient"):
        ctx.norm_rotate(rows(4, dtype=torch.float32).requires_grad_(), w, **kw)


def test_norm_backward_refusals(ctx):
    q, k, o, p, a, b = (rows(4) for _ in range(6))
    w, v, d, e = (torch.ones(64) for _ in range(4))
    kw = dict(axis_dims=(64,), positions=ints(1, 4))
    taken(lambda: ctx.norm_rotate_backward(q, w, o, **kw))
    taken(lambda: ctx.norm_rotate_backward(q, w, o, q, **kw))           # dx may be x or dout
    taken(lambda: ctx.norm_rotate_backward(q, w, o, o, **kw))
    taken(lambda: ctx.norm_rotate_backward((q, k), (w, w), (o, p), (o, p), (d, e), **kw))
    for dx, dw in (((a, a), (d, e)), ((a, b), (d, d)), ((k, b), (d, e)), ((a, o), (d, e)), ((p, a), (d, e)), ((a, b), (w, e)), ((a, b), (d, v))):
        with pytest.raises(ValueError, match="overlap"):
            ctx.norm_rotate_backward((q, k), (w, v), (o, p), dx, dw, **kw)
    for dw in (torch.ones(63), torch.ones(64, dtype=torch.bfloat16), torch.ones(128)[::2]):
        with pytest.raises(ValueError, match="dweight"):
            ctx.norm_rotate_backward(q, w, o, None, dw, **kw)
    with pytest.raises(ValueError, match="as many dx"):
        ctx.norm_rotate_backward((q, k), (w, v), (o, p), (a,), **kw)


def test_pages_refusals(ctx):
    good = torch.zeros(3, 16, 2, 64, dtype=torch.bfloat16)
    for k, v in ((good, good), (good, good[:2].clone()), (good.float(), good.float()), (good.flatten(1, 2), good.flatten(1, 2)),
                 (good, torch.zeros(3, 16, 64, 2, dtype=torch.bfloat16).transpose(2, 3)), (good, good.clone().requires_grad_()),
                 (good[:0], good[:0])):
        with pytest.raises(ValueError):
            hc.Pages(k, v)
    q, k, table = rows(4, 4), rows(4), ints(2, 3)
    p = pages()
    taken(lambda: ctx.paged_append(p, table, k, rows(4), ints(2)))
    taken(lambda: ctx.paged_attention(p, table, q, ints(2)))
    taken(lambda: ctx.paged_attention(p, table, q, ints(2), out=q, window=3, sinks=1))
    for bad in (ints(2, 3).long(), ints(6), ints(3, 2).t(), ints(2, 6)[:, ::2]):
        with pytest.raises(ValueError, match="table"):
            ctx.paged_append(p, bad, k, rows(4), ints(2))
        with pytest.raises(ValueError, match="table"):
            ctx.paged_attention(p, bad, q, ints(2))
    taken(lambda: ctx.paged_append(p, ints(2, 9)[:, 2:5], k, rows(4), ints(2)))          # rows apart
    with pytest.raises(ValueError, match="start"):
        ctx.paged_append(p, table, k, rows(4), ints(3))
    with pytest.raises(ValueError, match="kv_len"):
        ctx.paged_attention(p, table, q, ints(3))
    with pytest.raises(ValueError, match="cu_seqlens"):
        ctx.paged_attention(p, table, q, ints(2), ints(2))
    with pytest.raises(ValueError, match="expected shape"):
        ctx.paged_append(p, table, rows(4, 3), rows(4, 3), ints(2))
    with pytest.raises(ValueError, match="heads of 64"):
        ctx.paged_attention(p, table, rows(4, 4, 128), ints(2))
    with pytest.raises(ValueError, match="overlap"):
        ctx.paged_append(p, table, p.k[0, :4], rows(4), ints(2))
    with pytest.raises(ValueError, match="overlap"):
        ctx.paged_attention(p, table, q, ints(2), out=q.as_strided(q.shape, (64, 256, 1)))
    with pytest.raises(ValueError, match="overlap"):
        ctx.paged_attention(p, table, rows(4), ints(2), out=p.v[0, :4])
    p.device = 3
    with pytest.raises(ValueError, match="pages are on"):
        ctx.paged_attention(p, table, q, ints(2))


def test_window_refusals(ctx):
    q, k, v, o, g, a, b, c = (rows(4) for _ in range(8))
    lse = torch.zeros(2, 4)
    taken(lambda: ctx.window_attention(q, k, v, out=q, lse=lse))
    taken(lambda: ctx.window_attention_backward(q, k, v, o, lse, g))
    for out in (k, v):
        with pytest.raises(ValueError, match="overlap"):
            ctx.window_attention(q, k, v, out=out)
    for bad in (torch.zeros(4, 2), torch.zeros(2, 4).double(), torch.zeros(4, 2).t()):
        with pytest.raises(ValueError, match="lse"):
            ctx.window_attention(q, k, v, lse=bad)
        with pytest.raises(ValueError, match="lse"):
            ctx.window_attention_backward(q, k, v, o, bad, g)
    for grads in ((a, a, c), (q, b, c), (a, k, c), (a, b, v), (o, b, c), (a, g, c), (a, b, b)):
        with pytest.raises(ValueError, match="overlap"):
            ctx.window_attention_backward(q, k, v, o, lse, g, None, None, *grads)
    with pytest.raises(ValueError, match="dout"):
        ctx.window_attention_backward(q, k, v, o, lse, rows(3))
    with pytest.raises(ValueError, match="dk"):
        ctx.window_attention_backward(q, k, v, o, lse, g, None, None, a, rows(5), c)
    # (a half-precision leaf cannot be made on its own: views of a float one stand for it)
    leaf = torch.zeros(4, 2, 64, requires_grad=True).bfloat16()
    with pytest.raises(ValueError, match="requires a gradient"):
        ctx.window_attention(leaf, k, v)
    with torch.no_grad():
        taken(lambda: ctx.window_attention(leaf, k, v))


def test_no_positions_of_no_tokens(window_check):
    """An empty tensor of positions has no address, which stands for the grid where there are tokens."""
    run = subprocess.run([window_check, "no_tokens"], capture_output=True, text=True, timeout=60,
                         env=dict(os.environ, ASAN_OPTIONS="detect_leaks=0"))
    assert run.returncode == 0, run.stdout + run.stderr
