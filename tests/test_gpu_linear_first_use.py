"""The first linear product of a process, recorded into a graph with a plan that was made for execute."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CHILD = """
import torch
import paper_2512_22142_amd as cleave
A, B, bias = (torch.randn(*s, device="cuda").bfloat16() for s in ((512, 256), (256, 512), (1, 512)))
bias = bias[0].float()
C = torch.zeros(512, 512, dtype=torch.bfloat16, device="cuda")
plan = cleave.plan_uniform(512, 512, 256, 256, 256, 1)
plan.upload()
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    cleave.linear(plan, A, B, C, bias=bias, act="relu")
for _ in range(3):
    C.zero_()
    graph.replay()
    torch.cuda.synchronize()
    got = C.clone()
    cleave.linear(plan, A, B, C, bias=bias, act="relu")
    assert torch.equal(got, C) and bool((got > 0).any())
print("same", plan.last_kernel)
"""


def test_first_use_in_a_graph():
    done = subprocess.run([sys.executable, "-c", CHILD], cwd=ROOT, capture_output=True, text=True, timeout=100)
    assert done.returncode == 0, done.stdout + done.stderr
    assert "same linear_direct" in done.stdout
