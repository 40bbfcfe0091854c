"""A gated feed-forward block and a language model's head on the package's operators: training steps, then a served token.

    python examples/gated_block.py [--tokens 4096 --width 4096 --inner 11008 --vocabulary 32000 --steps 20]

The block is  h = x + r;  y = Wd (silu(Wg n) * (Wu n)) + h, n = norm1(h);  its head  logits = We norm2(y).  It is trained to name, for each
row of x, the token whose embedding x is.  Forward: layer_norm (residual added on the way), linear_gated, linear with residual,
layer_norm, linear, log_probs.  Backward: log_probs_backward (over the logits), linear_gated_grad in the product with Wd^T, one
product each for the gradients of n and of both weights, which lie side by side, the norms' gradients.  Update: one adamw call.
Serving: the first norm leaves e4m3 rows for linear_gated with weights laid out once in e4m3; log_probs gives the most
likely tokens.  Every buffer is made once; a step allocates nothing.
"""
import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

import paper_2512_22142_amd as cleave  # noqa: E402

BF16, F32, E4M3, I64 = torch.bfloat16, torch.float32, torch.float8_e4m3fn, torch.int64
ADAM = dict(lr=1e-3, beta1=0.9, beta2=0.95, eps=1e-8, weight_decay=0.01)
BONUS = 0.01     # of the entropy, in the loss


def _empty(*shape, dtype=F32):
    return torch.empty(shape, dtype=dtype, device="cuda")


class GatedBlock:
    NAMES = ("norm1", "bias1", "w", "wd", "norm2", "bias2", "we")

    def __init__(self, tokens, width, inner, vocabulary, seed=0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        T, h, F, V = self.sizes = tokens, width, inner, vocabulary
        # w: gate's columns, then up's
        shapes = dict(norm1=(h,), bias1=(h,), w=(h, 2 * F), wd=(F, h), norm2=(h,), bias2=(h,), we=(h, V))
        self.w = {n: torch.randn(s, generator=g, device="cuda").mul_(0.02) for n, s in shapes.items()}
        for n in ("norm1", "norm2"):
            self.w[n].fill_(1.0)
        self.copy = {n: t.to(BF16) for n, t in self.w.items()}
        self.grad = {n: torch.zeros_like(t) for n, t in self.w.items()}
        self.m, self.v = ({n: torch.zeros_like(t) for n, t in self.w.items()} for _ in range(2))
        self.steps = 0
        # activations and their gradients
        self.h, self.n, self.y, self.f, self.dn, self.dy, self.dx = (_empty(T, h, dtype=BF16) for _ in range(7))
        self.zg, self.zu, self.a = (_empty(T, F, dtype=BF16) for _ in range(3))
        self.dz, self.logits = _empty(T, 2 * F, dtype=BF16), _empty(T, V, dtype=BF16)
        self.stats = [(_empty(T), _empty(T)) for _ in range(2)]
        self.logp, self.lse, self.entropy = (_empty(T) for _ in range(3))
        # gradients of the loss, the mean of -logp - BONUS entropy
        self.dlogp, self.dentropy = torch.full((T,), -1.0 / T, device="cuda"), torch.full((T,), -BONUS / T, device="cuda")
        self.gated = cleave.plan_gated(T, F, h, BF16)
        # one plan per product: M, N, K
        self.plans = {name: cleave.plan_linear(*mnk, BF16) for name, mnk in dict(
            down=(T, h, F), head=(T, V, h), dwe=(h, V, T), df=(T, h, V), dz=(T, F, h), dwd=(F, h, T), dn=(T, h, 2 * F),
            dw=(h, 2 * F, T)).items()}
        for plan in (self.gated, *self.plans.values()):
            plan.upload()
        self.ws = _empty(max([1, cleave.gated_workspace(self.gated), cleave.gated_grad_workspace(self.plans["dz"]),
                              cleave.layer_norm_workspace(T, h), cleave.log_probs_workspace(T, V)] +
                             [p.linear_workspace for p in self.plans.values()]))

    def forward(self, x, r, tokens):
        """Log probabilities of the rows' tokens."""
        p, ws, c, F = self.plans, self.ws, self.copy, self.sizes[2]
        cleave.layer_norm(x, self.w["norm1"], self.n, bias=self.w["bias1"], residual=r, sum_out=self.h, mean=self.stats[0][0],
                          inv_std=self.stats[0][1])
        cleave.linear_gated(self.gated, self.n, c["w"][:, :F], c["w"][:, F:], self.a, act="silu", gate=self.zg, up=self.zu, partials=ws)
        cleave.linear(p["down"], self.a, c["wd"], self.y, residual=self.h, partials=ws)
        cleave.layer_norm(self.y, self.w["norm2"], self.f, bias=self.w["bias2"], mean=self.stats[1][0], inv_std=self.stats[1][1])
        cleave.linear(p["head"], self.f, c["we"], self.logits, partials=ws)
        cleave.log_probs(self.logits, tokens, self.logp, lse=self.lse, entropy=self.entropy, workspace=ws)
        return self.logp

    def backward(self, tokens):
        """Gradients of the parameters into self.grad; returns that of x (and of r).  The logits give way to their gradient."""
        p, ws, c, grad, F = self.plans, self.ws, self.copy, self.grad, self.sizes[2]
        cleave.log_probs_backward(self.logits, self.lse, self.logits, ids=tokens, dlogp=self.dlogp, entropy=self.entropy,
                                  dentropy=self.dentropy)
        cleave.linear(p["dwe"], self.f, self.logits, grad["we"], transA=1, partials=ws)
        cleave.linear(p["df"], self.logits, c["we"], self.dn, transB=1, partials=ws)
        cleave.layer_norm_backward(self.dn, self.y, self.w["norm2"], *self.stats[1], self.dy, grad["norm2"], ws, dbias=grad["bias2"])
        cleave.linear_gated_grad(p["dz"], self.dy, c["wd"], self.zg, self.zu, self.dz[:, :F], self.dz[:, F:], transB=1, act="silu",
                                 partials=ws)
        cleave.linear(p["dwd"], self.a, self.dy, grad["wd"], transA=1, partials=ws)
        cleave.linear(p["dn"], self.dz, c["w"], self.dn, transB=1, partials=ws)
        cleave.linear(p["dw"], self.n, self.dz, grad["w"], transA=1, partials=ws)
        cleave.layer_norm_backward(self.dn, self.h, self.w["norm1"], *self.stats[0], self.dx, grad["norm1"], ws, dbias=grad["bias1"],
                                   dsum=self.dy)
        return self.dx

    def update(self):
        self.steps += 1
        lists = lambda d: [d[n] for n in self.NAMES]   # noqa: E731
        cleave.adamw(lists(self.w), lists(self.grad), lists(self.m), lists(self.v), copies=lists(self.copy), step=self.steps, **ADAM)


class ServedBlock:
    """The trained block for `rows` tokens at a time, gate and up in 8 bits."""

    def __init__(self, block, rows, top=5):
        _, h, F, V = block.sizes
        w = block.w["w"].t().contiguous()                    # out x in, as 8-bit products read it
        scale = w.abs().amax(dim=1) / 448
        self.wide, self.scales = (w / scale[:, None]).to(E4M3), scale
        self.block, self.F = block, F
        self.n, self.row_scales = _empty(rows, h, dtype=E4M3), _empty(rows)
        self.h, self.y, self.f = (_empty(rows, h, dtype=BF16) for _ in range(3))
        self.a, self.logits = _empty(rows, F, dtype=BF16), _empty(rows, V)
        self.top, self.top_logp = _empty(rows, top, dtype=I64), _empty(rows, top)
        self.gated = cleave.plan_gated(rows, F, h, E4M3)
        self.down, self.head = cleave.plan_linear(rows, h, F, BF16), cleave.plan_linear(rows, V, h, BF16)
        self.ws = _empty(max(1, cleave.gated_workspace(self.gated), self.down.linear_workspace, self.head.linear_workspace,
                             cleave.log_probs_workspace(rows, V, top)))

    def __call__(self, x, r):
        """The most likely tokens and their log probabilities."""
        b, F, ws = self.block, self.F, self.ws
        cleave.layer_norm(x, b.w["norm1"], self.n, bias=b.w["bias1"], residual=r, sum_out=self.h, scales=self.row_scales)
        cleave.linear_gated(self.gated, self.n, self.wide[:F], self.wide[F:], self.a, transB=1, act="silu", scale_a=self.row_scales,
                            scale_gate=self.scales[:F], scale_up=self.scales[F:], partials=ws)
        cleave.linear(self.down, self.a, b.copy["wd"], self.y, residual=self.h, partials=ws)
        cleave.layer_norm(self.y, b.w["norm2"], self.f, bias=b.w["bias2"])
        cleave.linear(self.head, self.f, b.copy["we"], self.logits, partials=ws)
        cleave.log_probs(self.logits, top_ids=self.top, top_logp=self.top_logp, workspace=ws)
        return self.top, self.top_logp


def batches(block, seed=1):
    """Endless (x, r, tokens): x the embeddings of random tokens, r noise."""
    T, h, _, V = block.sizes
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    table = torch.randn(V, h, generator=g, device="cuda").to(BF16)
    while True:
        tokens = torch.randint(0, V, (T,), generator=g, device="cuda")
        yield table[tokens], torch.randn(T, h, generator=g, device="cuda").mul_(0.1).to(BF16), tokens


def train(block, steps, seed=1):
    """The mean negative log probability before each step."""
    losses = []
    for _, (x, r, tokens) in zip(range(steps), batches(block, seed)):
        losses.append(-block.forward(x, r, tokens).mean())
        block.backward(tokens)
        block.update()
    return [float(x) for x in losses]


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--tokens", type=int, default=4096)
    ap.add_argument("--width", type=int, default=4096)
    ap.add_argument("--inner", type=int, default=11008)
    ap.add_argument("--vocabulary", type=int, default=32000)
    ap.add_argument("--steps", type=int, default=20)
    a = ap.parse_args()
    block = GatedBlock(a.tokens, a.width, a.inner, a.vocabulary)
    losses = train(block, a.steps)
    print("negative log probability: %.4f at the start, %.4f after %d steps" % (losses[0], losses[-1], a.steps))
    x, r, tokens = next(batches(block))
    logp = block.forward(x, r, tokens)[:1].clone()
    top, top_logp = ServedBlock(block, 1)(x[:1], r[:1])
    print("token %d: log probability %.3f; served in 8 bits, most likely %s (%s)" % (
        int(tokens[0]), float(logp), top[0].tolist(), ", ".join("%.3f" % v for v in top_logp[0].tolist())))


if __name__ == "__main__":
    main()
