"""Outputs in an input's place, where they may be: the bits of the same call with an output of its own."""
import pytest
import torch

import paper_2512_22142_amd as cleave

pytestmark = pytest.mark.gpu

F32, BF16, E4M3 = torch.float32, torch.bfloat16, torch.float8_e4m3fn


def randn(*shape, dtype, seed):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()


# few rows, in chunks and whole; parts, chunks of parts; large tiles, several to a workgroup; ragged
LINEAR = [(3, 4096, 4096), (9, 260, 64), (70, 64, 8192), (300, 520, 200), (37, 53, 71), (4608, 4352, 128), (700, 300, 100)]


@pytest.mark.parametrize("M,N,K", LINEAR)
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("transB", [0, 1])
def test_a_products_argument_and_residual(M, N, K, dtype, transB):
    A, B = randn(M, K, dtype=dtype, seed=1), randn(*((N, K) if transB else (K, N)), dtype=dtype, seed=2)
    z = randn(M, N, dtype=dtype, seed=3)
    plan = cleave.plan_linear(M, N, K, dtype)
    ws = torch.empty(max(1, plan.linear_workspace), device="cuda")
    want, place = torch.empty_like(z), z.clone()
    cleave.linear(plan, A, B, want, transB=transB, act_grad="gelu_tanh", preact=z, partials=ws)
    cleave.linear(plan, A, B, place, transB=transB, act_grad="gelu_tanh", preact=place, partials=ws)
    assert torch.equal(want, place)
    cleave.linear(plan, A, B, want, transB=transB, act="silu", residual=z, partials=ws)
    cleave.linear(plan, A, B, z, transB=transB, act="silu", residual=z, partials=ws)
    assert torch.equal(want, z)


NORM = [(7, 100), (2000, 700), (300, 4096), (5, 16384), (3, 40000)]


@pytest.mark.parametrize("rows,cols", NORM)
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_norm(rows, cols, dtype):
    x, r, w = randn(rows, cols, dtype=dtype, seed=1), randn(rows, cols, dtype=dtype, seed=2), randn(cols, dtype=F32, seed=3)
    y, h = torch.empty_like(x), torch.empty_like(x)
    cleave.rms_norm(x, w, y, residual=r, sum_out=h)
    for y_at, h_at in ((0, 1), (1, 0)):
        place = [x.clone(), r.clone()]
        cleave.rms_norm(place[0], w, place[y_at], residual=place[1], sum_out=place[h_at])
        assert torch.equal(place[y_at], y) and torch.equal(place[h_at], h)


@pytest.mark.parametrize("rows,cols", NORM)
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_norms_gradient(rows, cols, dtype):
    named = dict(dy=randn(rows, cols, dtype=dtype, seed=1), h=randn(rows, cols, dtype=dtype, seed=2),
                 dsum=randn(rows, cols, dtype=dtype, seed=3))
    w, inv = randn(cols, dtype=F32, seed=4), torch.rsqrt(named["h"].float().square().mean(dim=1) + 1e-5)
    ws = torch.empty(cleave.rms_norm_workspace(rows, cols), device="cuda")

    def run(dx, dw, dy, h, dsum):
        cleave.rms_norm_backward(dy, h, w, inv, dx, dw, ws, dsum=dsum)

    dx, dw = torch.empty_like(named["dy"]), torch.empty(cols, device="cuda")
    run(dx, dw, **named)
    for name in named:
        at, dw2 = {k: t.clone() for k, t in named.items()}, torch.empty_like(dw)
        run(at[name], dw2, **at)
        assert torch.equal(at[name], dx) and torch.equal(dw, dw2), name
