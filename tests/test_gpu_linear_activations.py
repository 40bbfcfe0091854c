"""Activations and their slopes in fp32, relative to their own size down to the smallest."""
import numpy as np
import pytest
import torch

import paper_2512_22142_amd as cleave
from oracle import operators as oo

pytestmark = pytest.mark.gpu

F32 = torch.float32
U32 = 2.0 ** -24
LEAST = 2.0 ** -120   # the hardware's reciprocal and exponential may leave zero below 2^-126


def values(M, N):
    """z = a b with b a power of two: the product of one k is exact."""
    g = torch.Generator().manual_seed(M)
    a = (torch.rand(M, 1, generator=g) * 174 - 87).to(F32)
    b = torch.exp2(-(torch.arange(N) % 10).float()).view(1, N)
    return a.cuda(), b.cuda(), (a.double() * b.double()).numpy()


def sigmoid_argument(z, act):
    return z if act == "silu" else 2 * (2 / np.pi) ** 0.5 * (z + 0.044715 * z ** 3)


def logistic(u):
    with np.errstate(over="ignore"):
        return 1 / (1 + np.exp(-u))


def p_error(u, p, act):
    """Of a sigmoid p of u: the exponential's ulp, its argument's rest, an addition, the reciprocal's ulp; with tanh-gelu the
    roundings of the argument itself, five and a constant's."""
    return p * U32 * (8 + (6 * np.abs(u) * (1 - p) if act == "gelu_tanh" else 0))


@pytest.mark.parametrize("M,N", [(2000, 40), (16, 700), (40, 33)])
@pytest.mark.parametrize("act", ["silu", "gelu_tanh"])
def test_activation(M, N, act):
    a, b, z = values(M, N)
    y = torch.empty(M, N, device="cuda")
    plan = cleave.plan_linear(M, N, 1, F32)
    cleave.linear(plan, a, b, y, act=act, partials=torch.empty(max(1, plan.linear_workspace), device="cuda"))
    u = sigmoid_argument(z, act)
    p = logistic(u)
    bad = np.abs(y.double().cpu().numpy() - z * p) - (np.abs(z) * (p_error(u, p, act) + 2 * U32 * p) + np.abs(z) * LEAST)
    assert np.all(bad <= 0), z.flat[np.argmax(bad)]


@pytest.mark.parametrize("M,N", [(2000, 40), (16, 700), (40, 33)])
@pytest.mark.parametrize("act", ["silu", "gelu_tanh"])
def test_slope(M, N, act):
    _, _, z = values(M, N)
    a, b = torch.ones(M, 1, device="cuda"), torch.ones(1, N, device="cuda")
    y = torch.empty(M, N, device="cuda")
    plan = cleave.plan_linear(M, N, 1, F32)
    cleave.linear(plan, a, b, y, act_grad=act, preact=torch.from_numpy(z).float().cuda(),
                  partials=torch.empty(max(1, plan.linear_workspace), device="cuda"))
    u = sigmoid_argument(z, act)
    p, q = logistic(u), logistic(u) * logistic(-u)
    inner = np.abs(z) * (1 if act == "silu" else 2 * (2 / np.pi) ** 0.5 * (1 + 3 * 0.044715 * z * z))   # |z u'(z)|
    # p + z u' p (1 - p): p's error in both terms, 1 - p's rounding, a few more of the products and the sum
    dp = p_error(u, p, act)
    bad = np.abs(y.double().cpu().numpy() - (p + np.sign(z) * inner * q)) - (dp + 2 * inner * dp + 8 * U32 * (p + inner * q)
                                                                            + (1 + inner) * LEAST)
    assert np.all(bad <= 0), z.flat[np.argmax(bad)]


def test_oracle_agrees():
    _, _, z = values(40, 33)
    z = np.clip(z, -20, 20)
    for act in ("silu", "gelu_tanh"):
        u = sigmoid_argument(z, act)
        assert np.allclose(oo.act(z, act), z * logistic(u), rtol=1e-9, atol=1e-12)
        assert np.allclose(oo.act_grad(z, act), logistic(u) + z * logistic(u) * logistic(-u) *
                           (1 if act == "silu" else 2 * (2 / np.pi) ** 0.5 * (1 + 3 * 0.044715 * z * z)), rtol=1e-9, atol=1e-12)
