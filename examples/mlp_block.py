"""A transformer layer's MLP block on the package's operators: training steps, then a served token.

    python examples/mlp_block.py [--tokens 4096 --width 4096 --inner 11008 --steps 20]

The block is  h = x + r;  y = W2 gelu(W1 norm(h) + b1) + b2 + h,  trained towards a fixed random map of its
input.  Forward: rms_norm (residual added on the way), linear with bias and gelu, linear with bias and
residual.  Backward: the gradient of gelu's input out of the product with W2^T, weight gradients, bias
gradients, the norm's gradient.  Update: one adamw call for all five tensors, states in 8 bits.
Serving: the same norm leaves e4m3 rows for a product with the weight laid out once in e4m3.
Every buffer is made once; a step allocates nothing.
"""
import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

import paper_2512_22142_amd as cleave  # noqa: E402

BF16, F32, E4M3 = torch.bfloat16, torch.float32, torch.float8_e4m3fn
ADAM = dict(lr=1e-3, beta1=0.9, beta2=0.95, eps=1e-8, weight_decay=0.01)


def _empty(*shape, dtype=F32):
    return torch.empty(shape, dtype=dtype, device="cuda")


class MlpBlock:
    NAMES = ("norm", "w1", "b1", "w2", "b2")

    def __init__(self, tokens, width, inner, states_8bit=True, seed=0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        T, h, F = self.sizes = tokens, width, inner
        shapes = dict(norm=(h,), w1=(h, F), b1=(F,), w2=(F, h), b2=(h,))
        # fp32 masters, bf16 copies of them for the products, gradients, optimizer states
        self.w = {n: torch.randn(s, generator=g, device="cuda").mul_(0.02) for n, s in shapes.items()}
        self.w["norm"].fill_(1.0)
        self.copy = {n: t.to(BF16) for n, t in self.w.items()}
        self.grad = {n: torch.zeros_like(t) for n, t in self.w.items()}
        state = E4M3 if states_8bit else F32
        self.m, self.v = ({n: torch.zeros(t.shape, dtype=state, device="cuda") for n, t in self.w.items()} for _ in range(2))
        scales = {n: torch.zeros(-(-t.numel() // 256), device="cuda") for n, t in self.w.items()} if states_8bit else None
        self.m_scale, self.v_scale = scales, scales and {n: s.clone() for n, s in scales.items()}
        self.steps = 0
        # activations and their gradients
        self.h, self.n, self.y, self.dn, self.dx = (_empty(T, h, dtype=BF16) for _ in range(5))
        self.z, self.a, self.dz = (_empty(T, F, dtype=BF16) for _ in range(3))
        self.inv_rms = _empty(T)
        # one plan per product: M, N, K
        self.plans = {name: cleave.plan_linear(*mnk, BF16) for name, mnk in dict(
            up=(T, F, h), down=(T, h, F), dz=(T, F, h), dw2=(F, h, T), dn=(T, h, F), dw1=(h, F, T)).items()}
        for plan in self.plans.values():
            plan.upload()
        self.ws = _empty(max([1, cleave.rms_norm_workspace(T, h), cleave.bias_grad_workspace(T, F),
                              cleave.bias_grad_workspace(T, h)] + [p.linear_workspace for p in self.plans.values()]))

    def forward(self, x, r):
        p, ws = self.plans, self.ws
        cleave.rms_norm(x, self.w["norm"], self.n, residual=r, sum_out=self.h, inv_rms=self.inv_rms)
        cleave.linear(p["up"], self.n, self.copy["w1"], self.a, bias=self.w["b1"], act="gelu_tanh", preact=self.z, partials=ws)
        cleave.linear(p["down"], self.a, self.copy["w2"], self.y, bias=self.w["b2"], residual=self.h, partials=ws)
        return self.y

    def backward(self, dy):
        """Gradients of the parameters into self.grad; returns that of x (and of r)."""
        p, ws, grad = self.plans, self.ws, self.grad
        cleave.linear(p["dz"], dy, self.copy["w2"], self.dz, transB=1, act_grad="gelu_tanh", preact=self.z, partials=ws)
        cleave.linear(p["dw2"], self.a, dy, grad["w2"], transA=1, partials=ws)
        cleave.bias_grad(dy, grad["b2"], ws)
        cleave.linear(p["dn"], self.dz, self.copy["w1"], self.dn, transB=1, partials=ws)
        cleave.linear(p["dw1"], self.n, self.dz, grad["w1"], transA=1, partials=ws)
        cleave.bias_grad(self.dz, grad["b1"], ws)
        cleave.rms_norm_backward(self.dn, self.h, self.w["norm"], self.inv_rms, self.dx, grad["norm"], ws, dsum=dy)
        return self.dx

    def update(self, grad_scale=None):
        self.steps += 1
        lists = lambda d: d and [d[n] for n in self.NAMES]   # noqa: E731
        cleave.adamw(lists(self.w), lists(self.grad), lists(self.m), lists(self.v), m_scales=lists(self.m_scale),
                     v_scales=lists(self.v_scale), copies=lists(self.copy), step=self.steps, grad_scale=grad_scale, **ADAM)


class ServedBlock:
    """The trained block for `rows` tokens at a time; the up projection in 8 bits."""

    def __init__(self, block, rows):
        _, h, F = block.sizes
        w1 = block.w["w1"].t().contiguous()                  # out x in, as the 8-bit product reads it
        self.w1_scale = w1.abs().amax(dim=1) / 448
        self.w1 = (w1 / self.w1_scale[:, None]).to(E4M3)
        self.block = block
        self.n, self.scales = _empty(rows, h, dtype=E4M3), _empty(rows)
        self.h, self.y, self.a = _empty(rows, h, dtype=BF16), _empty(rows, h, dtype=BF16), _empty(rows, F, dtype=BF16)
        self.up, self.down = cleave.plan_linear(rows, F, h, E4M3), cleave.plan_linear(rows, h, F, BF16)
        self.ws = _empty(max(1, self.up.linear_workspace, self.down.linear_workspace))

    def __call__(self, x, r):
        b = self.block
        cleave.rms_norm(x, b.w["norm"], self.n, residual=r, sum_out=self.h, scales=self.scales)
        cleave.linear(self.up, self.n, self.w1, self.a, transB=1, scale_a=self.scales, scale_b=self.w1_scale, bias=b.w["b1"],
                      act="gelu_tanh", partials=self.ws)
        cleave.linear(self.down, self.a, b.copy["w2"], self.y, bias=b.w["b2"], residual=self.h, partials=self.ws)
        return self.y


def train(block, steps, seed=1):
    """Mean squared error before each step, towards a permutation of the input's columns."""
    T, h, _ = block.sizes
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    order = torch.randperm(h, generator=g, device="cuda")
    losses = []
    for _ in range(steps):
        x, r = (torch.randn(T, h, generator=g, device="cuda").to(BF16) for _ in range(2))
        target = (x + r)[:, order]
        error = block.forward(x, r).float() - target.float()
        losses.append(error.square().mean())
        block.backward((error * (2.0 / error.numel())).to(BF16))
        norm = torch.stack([t.square().sum() for t in block.grad.values()]).sum().sqrt()
        block.update((1.0 / norm).clamp_max(1.0).reshape(1))  # gradients of norm 1 at most, without a host round trip
    return [float(x) for x in losses]


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--tokens", type=int, default=4096)
    ap.add_argument("--width", type=int, default=4096)
    ap.add_argument("--inner", type=int, default=11008)
    ap.add_argument("--steps", type=int, default=20)
    a = ap.parse_args()
    block = MlpBlock(a.tokens, a.width, a.inner)
    losses = train(block, a.steps)
    print("mean squared error: %.4f at the start, %.4f after %d steps" % (losses[0], losses[-1], a.steps))
    x, r = (torch.randn(a.tokens, a.width, device="cuda").to(BF16) for _ in range(2))
    y = block.forward(x, r)[:1].float().clone()
    served = ServedBlock(block, 1)(x[:1], r[:1]).float()
    print("one token, up projection in 8 bits: %.2e relative to the trained block" % float((served - y).norm() / y.norm()))


if __name__ == "__main__":
    main()
