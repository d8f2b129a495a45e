"""What the Python binding does on the host alone."""
import os
import subprocess
import sys

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
