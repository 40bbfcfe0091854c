"""The first gated product, and the first gradient of one, of a process: recorded into a graph, with a plan that was only uploaded."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
START = """
import torch
import paper_2512_22142_amd as cleave
M, K, N = {M}, {K}, {N}
def randn(*s):
    return torch.randn(*s, device="cuda").bfloat16()
def empty():
    return torch.zeros(M, N, dtype=torch.bfloat16, device="cuda")
A, B, U, g, u, C, D = randn(M, K), randn(K, N), randn(K, N), randn(M, N), randn(M, N), empty(), empty()
"""
GATED = """
plan = cleave.plan_gated(M, N, K, torch.bfloat16)
ws = torch.empty(max(1, cleave.gated_workspace(plan)), device="cuda")
def call():
    cleave.linear_gated(plan, A, B, U, C, partials=ws)
"""
GRAD = """
plan = cleave.plan_linear(M, N, K, torch.bfloat16)
ws = torch.empty(max(1, cleave.gated_grad_workspace(plan)), device="cuda")
def call():
    cleave.linear_gated_grad(plan, A, B, g, u, C, D, partials=ws)
"""
END = """
plan.upload()
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    call()
for _ in range(3):
    C.zero_()
    D.zero_()
    graph.replay()
    torch.cuda.synchronize()
    got, second = C.clone(), D.clone()
    call()
    assert torch.equal(got, C) and torch.equal(second, D) and bool((got != 0).any())
print("same", plan.last_kernel)
"""


@pytest.mark.parametrize("M,K,N", [(512, 256, 512), (900, 250, 300), (40, 250, 300), (4, 4096, 512), (4, 1024, 512)])
@pytest.mark.parametrize("what", [GATED, GRAD])
def test_first_use_in_a_graph(what, M, K, N):
    child = START.format(M=M, K=K, N=N) + what + END
    done = subprocess.run([sys.executable, "-c", child], cwd=ROOT, capture_output=True, text=True, timeout=100)
    assert done.returncode == 0, done.stdout + done.stderr
    assert "same " in done.stdout
