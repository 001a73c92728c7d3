"""What the routed-expert functions say about inputs that require a gradient."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PROGRAM = """
import warnings
import torch
from paper_2608_27888_gb300 import build as B
B.build()
from paper_2608_27888_gb300 import ntc
x, w, i = torch.zeros(2, 8), torch.zeros(4, 8), torch.zeros(2, 1, dtype=torch.int32)
p = torch.nn.Parameter(w)
def heard(call):
    with warnings.catch_warnings(record=True) as seen:
        warnings.simplefilter("always")
        try:
            call()
        except ValueError as e:
            assert "CUDA tensor" in str(e)  # the tensors are the host's: nothing is launched
    return [str(m.message) for m in seen]
assert not heard(lambda: ntc.linear(x, w)) and not heard(lambda: ntc.route(x, 1)) and not heard(lambda: ntc.combine(x, i))
with torch.no_grad():
    assert not heard(lambda: ntc.linear(x, p))
assert not heard(lambda: ntc.linear_backward(x, x, p))
said = heard(lambda: CALL)
assert len(said) == 1 and "no gradient" in said[0], said
assert not heard(lambda: CALL)
"""


def check(call):
    r = subprocess.run([sys.executable, "-c", PROGRAM.replace("CALL", call)], cwd=ROOT, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr


def test_a_weight_that_requires_a_gradient_draws_one_warning():
    check("ntc.linear(x, p)")


def test_so_do_logits_and_rows():
    check("ntc.route(p, 1)")
    check("ntc.combine(p, i)")
