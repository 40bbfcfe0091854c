"""The gradient of the logits where tokens are masked: in rows that have no token left, whatever the scale makes of their logits, and beside
gradients near fp32's largest value."""
import math

import pytest
import torch

import paper_2512_22142_amd as cleave

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
U32, U16 = 2.0 ** -24, 2.0 ** -8   # unit roundoffs: 24 and 8 bits of significand
INF = math.inf


def logits_of(rows, cols, dtype, offset=0.0):
    g = torch.Generator(device="cuda").manual_seed(1)
    return (torch.randn(rows, cols, generator=g, device="cuda") * 2.5 + offset).to(dtype)


def gradient(x, ids, scale, d):
    lse, ent = torch.empty(len(x), device="cuda"), torch.empty(len(x), device="cuda")
    cleave.log_probs(x, lse=lse, entropy=ent, scale=scale)
    dx = torch.empty_like(x)
    cleave.log_probs_backward(x, lse, dx, ids=ids, dlogp=d, entropy=ent, dentropy=d, scale=scale)
    return dx


@pytest.mark.parametrize("scale", [1e-37, 1e-30, 1e-20, 1e-9, 1.0, 300.0, 1e30])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("cols", [40, 1000, 5000, 20003])
def test_rows_of_masked_tokens_at_any_scale(scale, dtype, cols):
    """By the lowest value, by minus infinity, by both, by values between that and -1e30: zeros, but for a token beyond the row."""
    x = logits_of(6, cols, dtype)
    x[0], x[1], x[2], x[4] = torch.finfo(dtype).min, -INF, -INF, torch.finfo(dtype).min
    x[2, ::3] = torch.finfo(dtype).min
    x[3] = -2e30
    x[3, 1::2] = -1e38
    ids = torch.tensor([3, 4, 6, 7, cols, 8], device="cuda")
    dx = gradient(x, ids, scale, torch.ones(6, device="cuda"))
    assert torch.all(dx[:4] == 0) and torch.all(dx[4].isnan()) and not torch.any(dx[5].isnan())


@pytest.mark.parametrize("value,scale", [(-1e29, 1.0), (-1e29, 1e12), (-1e29, 1e-25), (-1e20, 1e-30), (-1e4, 1e-37)])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("cols", [40, 1000, 5000, 20003])
def test_rows_of_equal_logits_above_the_masked_ones(value, scale, dtype, cols):
    """All equal: d (1[j = id] - 1/n), and nothing of the entropy, whose largest value this is."""
    x = torch.full((3, cols), value, device="cuda", dtype=dtype)
    ids = torch.tensor([0, cols - 1, -1], device="cuda")
    scale = float(torch.tensor(scale))
    dx = gradient(x, ids, scale, torch.full((3,), 1.0 / scale, device="cuda"))
    want = torch.full((3, cols), -1.0 / cols, dtype=torch.float64, device="cuda")
    want[2] = 0
    want[0, 0] += 1
    want[1, cols - 1] += 1
    # the sum of n ones, its logarithm (of at most 10) and the exponential's argument, and the entropy's, for d and dent; scale twice
    n_err = (cols / 256 + 32 + 64) * U32
    half = U16 if dtype == BF16 else U32
    bad = (dx.double() - want).abs() - 4 * n_err / cols - (1.01 * half + 8 * U32) * want.abs()
    assert bad.max() <= 0, float(bad.max())


@pytest.mark.parametrize("mask", [-INF, -3e38])
@pytest.mark.parametrize("offset", [0.0, 1e4])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("cols", [1000, 20003])
def test_masked_tokens_beside_the_largest_gradients(mask, offset, dtype, cols):
    x = logits_of(3, cols, dtype, offset)
    x[:, 100:900] = mask
    ids = torch.tensor([3, 950, -1], device="cuda")
    lse, ent = torch.empty(3, device="cuda"), torch.empty(3, device="cuda")
    cleave.log_probs(x, lse=lse, entropy=ent)
    t = x.double() - x.double().amax(dim=1, keepdim=True)
    t = t - t.exp().sum(dim=1, keepdim=True).log()
    p = t.exp()
    for given in (1e20, 3e34, 3e38):
        d = torch.full((3,), given, device="cuda")
        dx = torch.empty_like(x)
        cleave.log_probs_backward(x, lse, dx, entropy=ent, dentropy=d)
        assert torch.all(dx[:, 100:900] == 0) and not torch.any(dx.isnan())
        want = -d.double()[:, None] * p * (torch.where(p > 0, t, torch.zeros_like(t)) + ent.double()[:, None])
        fits = want.abs() < 3.3e38      # (what the type holds)
        # log p of |t| + the distance's roundings and those of a near row's sum of exponentials (15 in size); p from it; three products
        far = t.abs().clamp_max(1e4)
        t_err = U32 * (cols / 256 + 32 + 64 + 8 * far)
        err = d.double()[:, None] * p * (t_err * (1 + (t + ent.double()[:, None]).abs().clamp_max(1e4)) + 8 * U32 * far)
        half = U16 if dtype == BF16 else U32
        bad = ((dx.double() - want).abs() - err - 1.01 * half * (want.abs() + err) - 2.0 ** -126 * given)[fits]
        assert bad.max() <= 0, float(bad.max() / given)
        cleave.log_probs_backward(x, lse, dx, ids=ids, dlogp=d)
        assert torch.all(dx[:, 100:900] == 0) and torch.all(dx.isfinite())
        d.fill_(torch.finfo(F32).max)
        cleave.log_probs_backward(x, lse, dx, ids=ids, dlogp=d, entropy=ent, dentropy=torch.full((3,), -1e30, device="cuda"))
        assert torch.all(dx[:, 100:900] == 0) and not torch.any(dx.isnan())


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("cols", [1000, 20003])
def test_rows_without_a_token_left_beside_the_largest_gradients(dtype, cols):
    x = logits_of(3, cols, dtype)
    x[0], x[1] = -INF, torch.finfo(dtype).min
    dx = gradient(x, torch.tensor([3, 4, 5], device="cuda"), 1.0, torch.full((3,), 3e38, device="cuda"))
    assert torch.all(dx[:2] == 0)


def test_infinite_and_nan_gradients_stay_visible():
    """No token is masked: the row shows what it was given; the others are what they are alone."""
    for dtype in (BF16, F32):
        for cols in (1000, 20003):
            x = logits_of(5, cols, dtype)
            ids = torch.arange(5, device="cuda")
            plain = gradient(x, ids, 1.0, torch.ones(5, device="cuda"))
            d = torch.tensor([1.0, INF, -INF, float("nan"), 1.0], device="cuda")
            dx = gradient(x, ids, 1.0, d)
            assert torch.equal(dx[0], plain[0]) and torch.equal(dx[4], plain[4]) and not torch.any(dx[1:4].isfinite())
