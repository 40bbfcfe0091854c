"""The example block: its gradients against fp64, its loss falls, its served token is the trained block's."""
import os
import sys

import numpy as np
import pytest
import torch

from oracle import operators as oo

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


def f64(t):
    return t.double().cpu().numpy()


def rel(got, want):
    return np.linalg.norm(got - want) / np.linalg.norm(want)


@pytest.mark.parametrize("tokens,width,inner", [(192, 256, 384), (100, 72, 200), (7, 64, 96)])
def test_gradients(tokens, width, inner):
    import mlp_block
    block = mlp_block.MlpBlock(tokens, width, inner, seed=3)
    g = torch.Generator().manual_seed(5)
    x, r, dy = (torch.randn(tokens, width, generator=g).to(torch.bfloat16).cuda() for _ in range(3))
    block.w["b1"].normal_()
    y = block.forward(x, r)
    dx = block.backward(dy)
    w = {n: f64(block.copy[n] if n in ("w1", "w2") else block.w[n]) for n in block.NAMES}
    n, h, inv = oo.rms_norm(f64(x), w["norm"], 1e-5, f64(r))
    a, z = oo.linear(n, w["w1"], w["b1"], "gelu_tanh")
    want_y, _ = oo.linear(a, w["w2"], w["b2"], residual=h)
    dz = (f64(dy) @ w["w2"].T) * oo.act_grad(z, "gelu_tanh")
    want_dx, want_dn = oo.rms_norm_backward(dz @ w["w1"].T, h, w["norm"], inv, f64(dy))
    want = dict(w2=a.T @ f64(dy), b2=f64(dy).sum(axis=0), w1=n.T @ dz, b1=dz.sum(axis=0), norm=want_dn)
    # every tensor between two operators is rounded to bf16 (2^-9 rms of its values), a handful of them on each way
    assert rel(f64(y), want_y) < 6 * 2.0 ** -9 and rel(f64(dx), want_dx) < 6 * 2.0 ** -9
    for name in block.NAMES:
        assert rel(f64(block.grad[name]), want[name]) < 8 * 2.0 ** -9, name


@pytest.mark.parametrize("states_8bit", [True, False])
def test_training_and_serving(states_8bit):
    import mlp_block
    block = mlp_block.MlpBlock(256, 128, 256, states_8bit=states_8bit)
    losses = mlp_block.train(block, 60)
    assert all(np.isfinite(losses)) and losses[-1] < 0.9 * losses[0]
    for n, t in block.w.items():
        assert torch.equal(block.copy[n], t.to(torch.bfloat16)), n
    x, r = (torch.randn(256, 128, device="cuda").to(torch.bfloat16) for _ in range(2))
    y = f64(block.forward(x, r))
    for rows in (1, 5, 40):
        # e4m3 rounds the norm's rows and the weight by 2^-4 at most, 2^-5.3 rms, in one of the sum's two terms
        assert rel(f64(mlp_block.ServedBlock(block, rows)(x[:rows], r[:rows])), y[:rows]) < 0.08
