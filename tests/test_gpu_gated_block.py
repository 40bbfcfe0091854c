"""The example of a gated block and its head: it runs, its gradients against fp64, its step in a graph, its served tokens."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


def rel(got, want):
    return float((got.double() - want).norm() / want.norm())


def norm(h, w, b):
    d = h - h.mean(dim=1, keepdim=True)
    return d / (d.square().mean(dim=1, keepdim=True) + 1e-5).sqrt() * w + b


@pytest.mark.parametrize("tokens,width,inner,vocabulary", [(192, 256, 384, 1000), (100, 72, 200, 333), (7, 64, 96, 50), (400, 130, 77, 501)])
def test_gradients(tokens, width, inner, vocabulary):
    import gated_block
    block = gated_block.GatedBlock(tokens, width, inner, vocabulary, seed=3)
    for n in ("bias1", "bias2"):
        block.w[n].normal_()
    for n in ("w", "wd", "we"):
        block.copy[n].copy_(block.w[n].mul_(4))
    x, r, ids = next(gated_block.batches(block, 5))
    ids[::5] = -1
    logp = block.forward(x, r, ids).clone()
    entropy = block.entropy.clone()
    dx = block.backward(ids)
    w = {n: (block.copy[n] if n in ("w", "wd", "we") else block.w[n]).double().requires_grad_() for n in block.NAMES}
    x64 = x.double().requires_grad_()
    h = x64 + r.double()
    z = norm(h, w["norm1"], w["bias1"]) @ w["w"]
    g, u = z[:, :inner], z[:, inner:]
    y = (g * torch.sigmoid(g) * u) @ w["wd"] + h
    all_logp = torch.log_softmax(norm(y, w["norm2"], w["bias2"]) @ w["we"], dim=1)
    given = ids >= 0
    want = torch.where(given, all_logp.gather(1, ids.clamp_min(0)[:, None])[:, 0], torch.zeros_like(all_logp[:, 0]))
    ent = -(all_logp.exp() * all_logp).sum(dim=1)
    (-(want + gated_block.BONUS * ent).sum() / tokens).backward()
    # every tensor between two operators is rounded to bf16 (2^-9 rms of its values), a handful of them on each way; the log
    # probabilities are sums of as many rounded logits of a size of some units
    assert rel(logp, want.detach()) < 6 * 2.0 ** -9 and rel(entropy, ent.detach()) < 6 * 2.0 ** -9
    assert rel(dx, x64.grad) < 8 * 2.0 ** -9
    for n in block.NAMES:
        assert rel(block.grad[n], w[n].grad) < 8 * 2.0 ** -9, n


def test_a_step_in_a_graph_is_the_step():
    import gated_block
    sizes = (256, 128, 256, 1000)
    block = gated_block.GatedBlock(*sizes)
    x, r, ids = next(gated_block.batches(block))
    block.forward(x, r, ids)
    want = [block.backward(ids).clone()] + [block.grad[n].clone() for n in block.NAMES] + [block.logp.clone()]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        block.forward(x, r, ids)
        block.backward(ids)
    for _ in range(3):
        for t in (block.dx, block.logp, *block.grad.values()):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = [block.dx] + [block.grad[n] for n in block.NAMES] + [block.logp]
        assert all(torch.equal(a, b) for a, b in zip(want, got))
        other = gated_block.GatedBlock(*sizes, seed=1)      # the program's own eager work between the replays
        other.forward(x, r, ids)
        other.backward(ids)


def test_training_and_serving():
    import gated_block
    block = gated_block.GatedBlock(256, 128, 256, 500)
    losses = gated_block.train(block, 10)
    assert all(x == x and x < 100 for x in losses)
    for n, t in block.w.items():
        assert torch.equal(block.copy[n], t.to(torch.bfloat16)), n
    x, r, ids = next(gated_block.batches(block, 7))
    block.forward(x, r, ids)
    logits = block.logits.double()
    for rows in (1, 5, 40):
        served = gated_block.ServedBlock(block, rows, top=5)
        top, top_logp = served(x[:rows], r[:rows])
        # e4m3 rounds the norm's rows and both weights by 2^-4 at most, 2^-5.3 rms, in one of the sum's two terms
        assert rel(served.logits, logits[:rows]) < 0.1
        own = torch.log_softmax(served.logits.double(), dim=1)
        assert torch.equal(top, torch.sort(own, dim=1, descending=True, stable=True)[1][:, :5])
        assert rel(top_logp, own.gather(1, top)) < 1e-5
