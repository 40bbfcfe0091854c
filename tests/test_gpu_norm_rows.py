"""Norm and its gradient with rows enough for every kernel, nothing written beside the outputs; 8-bit rows beyond fp32's range."""
import pytest
import torch

import paper_2512_22142_amd as cleave

pytestmark = pytest.mark.gpu

F32, BF16, E4M3 = torch.float32, torch.bfloat16, torch.float8_e4m3fn
U32, U16 = 2.0 ** -24, 2.0 ** -8   # unit roundoffs: 24 and 8 bits of significand
SPARE = 70                         # sevens behind every output


def matrix(rows, cols, dtype, seed, pad=0, std=1.0):
    """A rows x cols view with a leading dimension of cols + pad in a buffer of sevens that is longer than it, and the buffer."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    flat = torch.full((rows * (cols + pad) + SPARE,), 7.0, device="cuda").to(dtype)
    view = flat[:rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    if std is not None:
        view.copy_((torch.randn(rows, cols, generator=g, device="cuda") * std).to(dtype))
    return view, flat


def floats(n, value=7.0):
    flat = torch.full((n + SPARE,), value, device="cuda")
    return flat[:n], flat


def beside(whole, view):
    """Nothing is written beside the view."""
    keep = view.clone()
    view.fill_(7.0)
    assert torch.all(whole.float() == 7.0)
    view.copy_(keep)


def near(got, want, dtype, slack, what):
    bad = (got.double() - want).abs() - (want.abs() * (U16 if dtype == BF16 else U32) * 1.01 + slack)
    assert bad.max() <= 0, (what, float(bad.max()))


def check_norm(rows, cols, dtype, out, pad):
    x, r = matrix(rows, cols, dtype, 1, pad, 2.0)[0], matrix(rows, cols, dtype, 2, pad)[0]
    w = matrix(1, cols, F32, 3)[0][0] + 1
    (y, y_whole), (s, s_whole) = matrix(rows, cols, out, 0, pad, None), matrix(rows, cols, dtype, 0, pad, None)
    (inv, inv_whole), (scales, scales_whole) = floats(rows), floats(rows)
    cleave.rms_norm(x, w, y, residual=r, sum_out=s, inv_rms=inv, scales=scales if out == E4M3 else None)
    h = x.double() + r.double()
    want_inv = 1 / (h.square().mean(dim=1) + 1e-5).sqrt()
    want = h * want_inv[:, None] * w.double()
    # a sum of n squares in any tree: n rounding errors at most, in practice the depth; half of it under the root
    n_err = (cols / 64 + 16) * U32
    near(inv, want_inv, F32, n_err * want_inv, "1 / rms")
    near(s, h, dtype, 2 * U32 * h.abs(), "sum")
    if out == E4M3:
        want_scale = want.abs().amax(dim=1) / 448
        near(scales, want_scale, F32, (n_err + 8 * U32) * want_scale, "scales")
        q = want / want_scale[:, None]
        # half a step: 2^-4 of the value, 2^-10 below the normal numbers
        bound = torch.maximum(q.abs() * 2.0 ** -4, torch.full_like(q, 2.0 ** -10)) * 1.001 + q.abs() * (n_err + 8 * U32)
        assert torch.all((y.float().double() - q).abs() <= bound)
        beside(scales_whole, scales)
    else:
        near(y, want, dtype, want.abs() * (n_err + 4 * U32), "y")
    for whole, view in ((y_whole, y), (s_whole, s), (inv_whole, inv)):
        beside(whole, view)


def around(*most):
    """Columns at and beside those that the groups of sixteen bytes of some threads hold."""
    return [n + d for n in most for d in (-1, 0, 1)]


# a wave to a row with one to four groups to a lane (more than 1024 rows), 256 threads with one to eight (more than 256), 1024 below
WAVE, WIDE = (64, 128, 192, 256), (512, 768, 1024, 1280, 1536, 1792, 2048)


@pytest.mark.parametrize("pad", [0, 5])
@pytest.mark.parametrize("dtype,out", [(BF16, BF16), (BF16, E4M3), (F32, F32), (F32, E4M3)])
@pytest.mark.parametrize("rows,groups", [(1025, g) for g in WAVE] + [(257, g) for g in WAVE[1:] + WIDE] + [(255, 256), (256, 1024)])
def test_norm(rows, groups, dtype, out, pad):
    for cols in around(groups * (8 if dtype == BF16 else 4)):
        check_norm(rows, cols, dtype, out, pad)


def check_gradient(rows, cols, dtype, pad, dsum):
    h, dy = matrix(rows, cols, dtype, 1, pad, 2.0)[0], matrix(rows, cols, dtype, 2, pad)[0]
    ds = matrix(rows, cols, dtype, 3, pad)[0] if dsum else None
    w = matrix(1, cols, F32, 4)[0][0] + 1
    inv = torch.rsqrt(h.float().square().mean(dim=1) + 1e-5)
    (dx, dx_whole), (dw, dw_whole) = matrix(rows, cols, dtype, 0, pad, None), floats(cols)
    ws, ws_whole = floats(cleave.rms_norm_workspace(rows, cols))
    cleave.rms_norm_backward(dy, h, w, inv, dx, dw, ws, dsum=ds)
    xhat, d = h.double() * inv.double()[:, None], dy.double()
    g = d * w.double()
    want = inv.double()[:, None] * (g - xhat * (g * xhat).mean(dim=1, keepdim=True))
    n_err = (cols / 64 + 16) * U32
    slack = inv.double()[:, None] * (g.abs() * 8 * U32 + xhat.abs() * (g * xhat).abs().mean(dim=1, keepdim=True) * n_err)
    if dsum:
        want, slack = want + ds.double(), slack + 2 * U32 * ds.double().abs()
    near(dx, want, dtype, slack + 4 * U32 * want.abs(), "dx")
    # a sum over the rows: up to rows / 8 + 64 additions one behind the other
    assert torch.all((dw.double() - (d * xhat).sum(dim=0)).abs() <= (d * xhat).abs().sum(dim=0) * (rows / 8 + 64) * U32)
    for whole, view in ((dx_whole, dx), (dw_whole, dw), (ws_whole, ws)):
        beside(whole, view)


# a wave to a row with one group to a lane and, with more than 2048 rows, two; 256, 512 and 1024 threads
@pytest.mark.parametrize("pad,dsum", [(0, True), (5, False)])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,groups", [(2049, 64), (2049, 128), (5001, 125), (2048, 128), (40, 64), (2049, 256), (900, 512), (900, 1024)])
def test_norms_gradient(rows, groups, dtype, pad, dsum):
    for cols in around(groups * (8 if dtype == BF16 else 4)):
        check_gradient(rows, cols, dtype, pad, dsum)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,cols", [(1, 1), (31, 63), (333, 1001), (5000, 40), (4096, 2048)])
def test_bias_gradient(rows, cols, dtype):
    dy = matrix(rows, cols, dtype, 1, 3)[0]
    (db, db_whole), (ws, ws_whole) = floats(cols), floats(cleave.bias_grad_workspace(rows, cols))
    cleave.bias_grad(dy, db, ws)
    assert torch.all((db.double() - dy.double().sum(dim=0)).abs() <= dy.double().abs().sum(dim=0) * (rows / 8 + 64) * U32)
    beside(db_whole, db)
    beside(ws_whole, ws)


@pytest.mark.parametrize("cols", [64, 100, 1000, 4096, 40000])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_8_bit_rows_that_hold_an_infinity_are_nan(cols, dtype):
    """From finite x: an infinite weight, or a product with the weight beyond fp32."""
    x = torch.ones(3, cols, dtype=dtype, device="cuda")
    x[1, 5] = 0
    x[2] = 0                                            # 0 times infinity
    q, scales = torch.empty(x.shape, dtype=E4M3, device="cuda"), torch.empty(3, device="cuda")
    w = torch.ones(cols, device="cuda")
    w[cols // 2] = float("inf")
    cleave.rms_norm(x, w, q, scales=scales)
    assert torch.all(scales.isnan()) and torch.all(q.float().isnan())
    x[2], x[2, cols // 3] = 1, 8                        # 8 / rms is above 1.3
    w[cols // 2], w[cols // 3] = 1, 3e38
    cleave.rms_norm(x, w, q, scales=scales)
    assert scales[2].isnan() and torch.all(q[2].float().isnan())
    for row in (0, 1):                                  # 3e38 itself is finite
        assert scales[row].isfinite() and q[row, cols // 3].float() == 448
