"""What the Python binding does on the host alone."""
import ctypes
import os
import subprocess
import sys

import pytest
import torch

from paper_2607_20125_amd import headcast as hc

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

WITHOUT_TORCH = """
import sys
sys.modules["torch"] = None                  # as where it is not installed
from paper_2607_20125_amd import headcast as hc
cfg = hc.make_config(n_layers=2)
assert hc.validate_config(cfg) == hc.HC_OK and hc.default_config().n_heads > 0
assert 0 <= hc.ring_slot(9, 7) < 7
assert hc.status_string(hc.HC_E_INVAL)
try:
    hc.QCache(1, 1, 64, 10, "cpu")
except ImportError:
    print("fine")
"""


def test_host_functions_need_no_torch():
    run = subprocess.run([sys.executable, "-c", WITHOUT_TORCH], cwd=ROOT, capture_output=True, text=True, timeout=120)
    assert run.returncode == 0, run.stderr
    assert run.stdout == "fine\n"


# --- tensors that a call writes -----------------------------------------------------------------

@pytest.fixture
def ctx():
    """A context without a device: its tensors are the CPU's, and a call that is not refused gets as far as the
    library, which has no context and says so."""
    c = hc.Context.__new__(hc.Context)
    c._h, c.device, c.cfg, c._need = ctypes.c_void_p(), -1, hc.default_config(), ctypes.c_int64()
    return c


def rows(n, heads=2, d=64):
    return torch.zeros(n, heads, d, dtype=torch.bfloat16)


@pytest.fixture(autouse=True)
def no_stream(monkeypatch):
    hc._use_torch()
    monkeypatch.setattr(hc, "_raw_stream", lambda device: 0)


def taken(call):
    """The call passes the binding's checks and reaches the library."""
    with pytest.raises(hc.HeadCastError):
        call()


def test_a_pair_writes_no_tensor_of_the_other(ctx):
    q, k, o, p = (rows(4) for _ in range(4))
    kw = dict(axis_dims=(64,), positions=torch.zeros(1, 4, dtype=torch.int32))
    for xs, outs in (((q, q), (q, q)), ((q, k), (k, q)), ((q, k), (o, o)), ((q, k), (o, q)), ((q, k), (k, o))):
        with pytest.raises(ValueError, match="overlap"):
            ctx.rotate(xs, outs, **kw)
    for xs, outs in (((q, k), (q, k)), ((q, k), (o, p)), ((q, q), (o, p)), ((q, k), None)):
        taken(lambda: ctx.rotate(xs, outs, **kw))
    none = rows(0)
    taken(lambda: ctx.rotate((none, none), (none, none), axis_dims=(64,), positions=torch.zeros(1, 0, dtype=torch.int32)))


def test_attention_writes_no_key_and_no_value(ctx):
    q, k, v = (rows(4) for _ in range(3))
    for out in (k, v):
        with pytest.raises(ValueError, match="overlap"):
            ctx.packed_attention(q, k, v, out=out)
    cu = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError, match="overlap"):     # the queries' memory in another order
        ctx.packed_attention(q[:2], k, v, cu, cu, out=q[:2].transpose(0, 1))
    taken(lambda: ctx.packed_attention(q, k, k, out=q))
    taken(lambda: ctx.packed_attention(q, q, q))
    one = rows(1)
    taken(lambda: ctx.packed_attention(one, k, v, cu, cu, out=one.as_strided((1, 2, 64), (1, 64, 1))))
    none = q[:0]
    taken(lambda: ctx.packed_attention(none, none, none, out=none))
    cache = hc.QCache(1, 2, 64, 10, "cpu")
    n = torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError, match="overlap"):
        ctx.qcache_attention(cache, q[:2], n, out=q[:2].transpose(0, 1))
    taken(lambda: ctx.qcache_attention(cache, q, n, out=q))


def test_reading_a_cache_needs_two_tensors(ctx):
    cache, k, n = hc.QCache(1, 2, 64, 10, "cpu"), rows(4), torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError, match="overlap"):
        ctx.qcache_read(cache, k, k, n)
    taken(lambda: ctx.qcache_read(cache, k[:0], k[:0], n))
    taken(lambda: ctx.qcache_read(cache, k, rows(4), n))
    taken(lambda: ctx.qcache_append(cache, k, k, n))


# --- gradients -----------------------------------------------------------------------------------

def test_no_gradient_is_dropped_in_silence(ctx):
    """The methods record none: a tensor that requires one is refused where gradients are recorded."""
    kw = dict(axis_dims=(64,), positions=torch.zeros(1, 4, dtype=torch.int32))
    cache, n = hc.QCache(1, 2, 64, 10, "cpu"), torch.zeros(1, dtype=torch.int32)
    calls = (lambda x, y: ctx.rotate(x, **kw), lambda x, y: ctx.rotate((y, x), **kw), lambda x, y: ctx.rotate(y, x, **kw),
             lambda x, y: ctx.packed_attention(x, y, y), lambda x, y: ctx.packed_attention(y, x, y),
             lambda x, y: ctx.packed_attention(y, y, x), lambda x, y: ctx.qcache_append(cache, x, y, n),
             lambda x, y: ctx.qcache_append(cache, y, x, n), lambda x, y: ctx.qcache_attention(cache, x, n))
    for call in calls:
        x = rows(4).requires_grad_()
        with pytest.raises(ValueError, match="gradient"):
            call(x, rows(4))
        taken(lambda: call(x.detach(), rows(4)))
        with torch.no_grad():
            taken(lambda: call(x, rows(4)))
        with torch.inference_mode():
            taken(lambda: call(x, rows(4)))
