"""The library and its ctypes calls do not need torch; the torch functions of the routed experts say that they do."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PROGRAM = """
import sys
sys.modules["torch"] = None
from paper_2608_27888_gb300 import build
assert build.build().endswith("libntc.so")
from paper_2608_27888_gb300 import ntc
assert ntc._lib.ntc_status_string(0)
assert ntc.ntc_expert_order_workspace(1 << 20, 64) > 0
try:
    ntc.route
    raise SystemExit("route came without torch")
except ImportError as e:
    assert "torch" in str(e)
"""


def test_build_and_calls_without_torch():
    r = subprocess.run([sys.executable, "-c", PROGRAM], cwd=ROOT, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
