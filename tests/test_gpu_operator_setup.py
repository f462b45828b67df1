"""What the operators' calls set up on their first use, in a process of its own: a first call inside a stream capture."""
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

CODE = """
import torch
from paper_2603_06626_b200 import binding as B
x, W = torch.ones(8, 64, device="cuda:0").bfloat16(), torch.ones(64, 64, device="cuda:0").bfloat16()
graph = torch.cuda.CUDAGraph()
try:
    with torch.cuda.graph(graph):
        B.linear(x, W)
    print("captured")
except RuntimeError as e:
    print("refused" if "outside a stream capture" in str(e) else repr(e))
status = torch.zeros(1, dtype=torch.int32, device="cuda:0")
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    y, _ = B.linear(x, W, status=status)          # with a word of its own a first call can be captured
graph.replay()
torch.cuda.synchronize()
print(float(y.sum()), int(status))
B.linear(x, W)
B.check_status()
print("usable")
"""


def test_a_first_call_inside_a_capture():
    r = subprocess.run([sys.executable, "-c", CODE], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
    assert r.stdout.split() == ["refused", str(64.0 * 8 * 64), "0", "usable"]
