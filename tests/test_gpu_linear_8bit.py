"""Sums of 8-bit products are fp32 sums: outliers that cancel, sums of one sign, random values; every shape of the kernel."""
import numpy as np
import pytest
import torch

import paper_2512_22142_amd as cleave

pytestmark = pytest.mark.gpu

F32, BF16, E4M3 = torch.float32, torch.bfloat16, torch.float8_e4m3fn
U32, U16 = 2.0 ** -24, 2.0 ** -8   # unit roundoffs: 24 and 8 bits of significand

# few rows; 64 x 64 parts; one 128 x 128 item per CU; a few per workgroup, whole and clipped
SIZES = [(16, 200), (17, 200), (130, 264), (1500, 1500), (2304, 2304), (3000, 3100)]


def product(A, B, out, preact=None, **kw):
    M, K = A.shape
    N = B.shape[0]
    plan = cleave.plan_linear(M, N, K, E4M3)
    C = torch.empty(M, N, dtype=out, device="cuda")
    ws = torch.full((max(1, plan.linear_workspace),), float("nan"), device="cuda")
    ones = dict(scale_a=torch.ones(M, device="cuda"), scale_b=torch.ones(N, device="cuda"))
    cleave.linear(plan, A, B, C, transB=1, preact=preact, partials=ws, **ones, **kw)
    return C


def sampled(A, B, seed=0):
    """Rows of op(A) op(B) in fp64, the sums of the products' magnitudes, and which rows."""
    rows = np.unique(np.random.default_rng(seed).integers(0, A.shape[0], 48))
    a, b = A.float().cpu().double().numpy()[rows], B.float().cpu().double().numpy()
    return a @ b.T, np.abs(a) @ np.abs(b).T, rows


def of_rows(C, rows):
    return C.float().cpu().double().numpy()[rows]


def within_fp32_sums(got, want, magnitudes, K, out):
    # K additions in fp32, in any order and rounded to either side: an ulp of the largest partial sum each
    bound = 2 * K * U32 * magnitudes
    assert np.all(np.abs(got - want) <= bound + (U16 if out == BF16 else U32) * (np.abs(want) + bound))


@pytest.mark.parametrize("M,N", SIZES)
@pytest.mark.parametrize("out", [BF16, F32])
def test_outliers_that_cancel(M, N, out):
    """Two products of 448 * 448 of opposite signs in every eight, the others 2^-14 of them and less."""
    K = 256
    g = torch.Generator().manual_seed(M)
    A, B = (torch.randint(lo, hi, s, generator=g).float() for lo, hi, s in ((2, 5, (M, K)), (1, 4, (N, K))))
    A[:, 0::8] = A[:, 1::8] = 448.0
    B[:, 0::8], B[:, 1::8] = 448.0, -448.0
    A, B = A.to(E4M3).cuda(), B.to(E4M3).cuda()
    want, magnitudes, rows = sampled(A, B)
    z = torch.empty(M, N, dtype=out, device="cuda")
    C = product(A, B, out, preact=z, act="relu")
    within_fp32_sums(of_rows(C, rows), want, magnitudes, K, out)
    within_fp32_sums(of_rows(z, rows), want, magnitudes, K, out)


@pytest.mark.parametrize("M,N", SIZES)
@pytest.mark.parametrize("out", [BF16, F32])
def test_products_of_one_sign(M, N, out):
    K = 512
    g = torch.Generator().manual_seed(M)
    A, B = ((torch.randn(n, K, generator=g).abs() * 60).to(E4M3).cuda() for n in (M, N))
    want, magnitudes, rows = sampled(A, B)
    got = of_rows(product(A, B, out), rows)
    within_fp32_sums(got, want, magnitudes, K, out)
    # the output's roundings go to either side: six standard deviations of their mean
    u = U16 if out == BF16 else U32
    assert abs(np.mean((got - want) / want)) <= 2 * K * U32 + 6 * u / (3 * got.size) ** 0.5


@pytest.mark.parametrize("M,N", SIZES)
def test_bf16_outputs_are_the_rounded_sums(M, N):
    """But for those within an fp32 sum's error of the middle between two bf16 values."""
    K = 512
    g = torch.Generator().manual_seed(M)
    A, B = ((torch.randn(n, K, generator=g) * 50).to(E4M3).cuda() for n in (M, N))
    want, _, rows = sampled(A, B)
    got = of_rows(product(A, B, BF16), rows)
    rounded = torch.from_numpy(want).to(BF16).double().numpy()
    # a random walk of K roundings: sqrt(K) 2^-24 of the values' size; values are 2^-8 of themselves apart or more, so
    # that share of them, twice for those below the rms, is an ulp (2^-7 at most) off
    off = 2 * K ** 0.5 * U32 / U16
    assert np.linalg.norm(got - rounded) <= 2.0 ** -7 * off ** 0.5 * np.linalg.norm(rounded)


@pytest.mark.parametrize("rows,N", [(16, 40), (256, 24), (4096, 1200)])
def test_every_8_bit_value(rows, N):
    """Each times one, and one times each: the value itself, NaN of both signs among them."""
    every = torch.arange(rows, device="cuda", dtype=torch.int32) % 256
    A = torch.zeros(rows, 256, device="cuda").to(E4M3)
    at = torch.arange(rows, device="cuda")
    A.view(torch.uint8)[at, at % 256] = every.to(torch.uint8)
    B = torch.ones(N, 256, device="cuda").to(E4M3)
    want = every.to(torch.uint8).view(E4M3).float()[:, None].expand(rows, N)
    nan = want.isnan()
    for out in (BF16, F32):
        got = product(A, B, out).float()
        assert torch.equal(got.isnan(), nan) and torch.equal(got[~nan], want[~nan])
        if N > 16:
            got = product(B, A, out).float()
            assert torch.equal(got.isnan(), nan.t()) and torch.equal(got[~nan.t()], want.t()[~nan.t()])
