"""Layer norm and its gradient against fp64, and what they refuse."""
import pytest
import torch

import paper_2512_22142_amd as cleave

pytestmark = pytest.mark.gpu

F32, BF16, E4M3 = torch.float32, torch.bfloat16, torch.float8_e4m3fn
U32, U16 = 2.0 ** -24, 2.0 ** -8   # unit roundoffs: 24 and 8 bits of significand
EPS = 1e-5
SPARE = 70                         # sevens behind every output

# every number of groups that a thread holds, whole and ragged; rows for waves of their own, few and many
SIZES = [(1, 1), (3, 64), (2, 511), (5, 512), (6, 513), (4, 1001), (2, 2048), (3, 2056), (7, 4096), (2, 5120), (2, 8200),
         (3, 16384), (1, 16392), (2, 32768), (1, 40000), (1500, 100), (1500, 768), (1100, 1111), (1030, 2048), (300, 3000), (300, 5120),
         (260, 9000), (260, 16384), (3, 700), (1000, 1000), (2, 1600), (9, 6000), (256, 9000), (2, 20000), (2, 11111)]


def matrix(rows, cols, dtype, seed, pad=0, shift=0, std=1.0, mean=0.0):
    """A rows x cols view, `shift` elements into a buffer of sevens with a leading dimension of cols + pad, and the buffer."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    flat = torch.full((rows * (cols + pad) + shift + SPARE,), 7.0, device="cuda").to(dtype)
    view = flat[shift: shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    if std is not None:
        view.copy_((torch.randn(rows, cols, generator=g, device="cuda") * std + mean).to(dtype))
    return view, flat


def floats(n):
    flat = torch.full((n + SPARE,), 7.0, device="cuda")
    return flat[:n], flat


def beside(view, whole):
    """Nothing is written beside the view."""
    keep = view.clone()
    view.fill_(7.0)
    assert torch.all(whole.float() == 7.0)
    view.copy_(keep)


def near(got, want, dtype, slack, what):
    """Within the output type's rounding and `slack`, an absolute error per element."""
    bad = (got.double() - want).abs() - (want.abs() * (U16 if dtype == BF16 else U32) * 1.01 + slack)
    assert bad.max() <= 0, (what, float(bad.max()))


def check_norm(rows, cols, dtype, out, residual=True, bias=True, pad=0, shift=0, mean=0.5):
    x = matrix(rows, cols, dtype, 1, pad, shift, 2.0, mean)[0]
    r = matrix(rows, cols, dtype, 2, pad, shift)[0] if residual else None
    w = matrix(1, cols, F32, 3)[0][0] + 1
    b = matrix(1, cols, F32, 4)[0][0].contiguous() if bias else None
    y, y_whole = matrix(rows, cols, out, 0, pad, shift, None)
    s, s_whole = matrix(rows, cols, dtype, 0, pad, shift, None)
    (m, m_whole), (inv, inv_whole), (scales, scales_whole) = floats(rows), floats(rows), floats(rows)
    cleave.layer_norm(x, w, y, bias=b, residual=r, sum_out=s if residual else None, mean=m, inv_std=inv,
                      scales=scales if out == E4M3 else None, eps=EPS)
    h = x.double() + (r.double() if residual else 0)
    want_m = h.mean(dim=1)
    d = h - want_m[:, None]
    want_inv = 1 / (d.square().mean(dim=1) + EPS).sqrt()
    want = d * want_inv[:, None] * w.double() + (b.double() if bias else 0)
    # sums of n values in any tree: n roundings at most, in practice the depth
    n_err = (cols / 64 + 16) * U32
    # an element's: of h itself (and so of their mean), of h - mean, of the mean of these
    h_err = U32 * (h.abs() + h.abs().mean(dim=1, keepdim=True))
    d_err = h_err + 3 * U32 * d.abs() + n_err * d.abs().mean(dim=1, keepdim=True)
    near(m, want_m, F32, d_err.mean(dim=1), "mean")
    inv_err = want_inv * (n_err + (d_err * d.abs()).mean(dim=1) * want_inv ** 2)
    near(inv, want_inv, F32, inv_err, "1 / std")
    if residual:
        near(s, h, dtype, 2 * U32 * h.abs(), "sum")
        beside(s, s_whole)
    part = (d * w.double()).abs()
    slack = w.double().abs() * want_inv[:, None] * d_err + part * inv_err[:, None] + 3 * U32 * (part * want_inv[:, None] + want.abs())
    if out == E4M3:
        want_scale = want.abs().amax(dim=1) / 448
        scale_err = slack.amax(dim=1) / 448 + 2 * U32 * want_scale
        near(scales, want_scale, F32, scale_err, "scales")
        q = want / want_scale[:, None]
        # half a step: 2^-4 of the value, 2^-10 below the normal numbers
        moved = slack / want_scale[:, None] + q.abs() * (scale_err / want_scale)[:, None] + 2 * U32 * q.abs()
        bound = torch.maximum(q.abs() * 2.0 ** -4, torch.full_like(q, 2.0 ** -10)) * 1.001 + moved * 1.1
        assert ((y.double() - q).abs() - bound).max() <= 0
        assert y.float().abs().amax(dim=1).min() == 448.0
    else:
        near(y, want, dtype, slack, "y")
    for view, whole in ((y, y_whole), (m, m_whole), (inv, inv_whole)):
        beside(view, whole)
    if out == E4M3:
        beside(scales, scales_whole)
    return y, m, inv


@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("dtype,out", [(BF16, BF16), (BF16, E4M3), (F32, F32), (F32, E4M3)])
def test_norm(rows, cols, dtype, out):
    # (one column has no deviation: its 8-bit row is the bias's, its value without one zero)
    check_norm(rows, cols, dtype, out, residual=rows % 2 == 1, bias=cols % 3 > 0 or cols == 1)


# rows that eight or sixteen lanes share, and the next wider ones; numbers of them that end within a wave
NARROW = [(1, 2), (33, 8), (100, 31), (4099, 32), (35, 33), (1000, 63), (4097, 64), (2055, 65), (70, 100), (515, 127), (9001, 128), (129, 129),
          (47, 200), (3003, 255), (5001, 256), (14, 257)]


@pytest.mark.parametrize("rows,cols", NARROW)
@pytest.mark.parametrize("dtype,out", [(BF16, BF16), (BF16, E4M3), (F32, F32), (F32, E4M3)])
def test_narrow_rows(rows, cols, dtype, out):
    check_norm(rows, cols, dtype, out, residual=rows % 2 == 1, bias=cols % 2 == 0)
    check_norm(rows, cols, dtype, out, residual=rows % 2 == 0, pad=3, shift=1)


@pytest.mark.parametrize("pad,shift", [(8, 0), (3, 0), (8, 1), (0, 4), (5, 7)])
@pytest.mark.parametrize("dtype,out", [(BF16, BF16), (BF16, E4M3), (F32, F32)])
@pytest.mark.parametrize("cols", [768, 70001])
def test_strides_and_alignment(pad, shift, dtype, out, cols):
    check_norm(9, cols, dtype, out, True, True, pad, shift)


@pytest.mark.parametrize("cols", [100, 4096, 40000])
def test_a_mean_far_from_zero(cols):
    """The deviations of fp32 rows a thousand deviations from zero: the bound counts the roundings of h - mean, not the mean's."""
    check_norm(5, cols, F32, F32, False, mean=2000.0)
    check_norm(5, cols, F32, F32, True, mean=-2000.0)


def test_rows_of_equal_values_and_what_is_not_finite():
    for cols in (64, 100, 4096, 40000):
        x = matrix(6, cols, F32, 1)[0].clone()
        x[1] = 3.7
        x[2, cols // 2] = float("nan")
        x[3, 0] = float("inf")
        x[4] = 0
        w, b = torch.ones(cols, device="cuda"), torch.zeros(cols, device="cuda")
        y, q = torch.empty_like(x), torch.empty(x.shape, dtype=E4M3, device="cuda")
        scales, inv = torch.empty(6, device="cuda"), torch.empty(6, device="cuda")
        cleave.layer_norm(x, w, y, bias=b, inv_std=inv, eps=EPS)
        cleave.layer_norm(x, w, q, scales=scales, eps=EPS)
        # equal values: what is left of h - mean is its rounding, over sqrt(eps)
        assert y[1].abs().max() <= 4 * U32 * 3.7 / EPS ** 0.5 and abs(float(inv[1]) * EPS ** 0.5 - 1) < 1e-4
        for k in (2, 3):
            assert torch.all(y[k].isnan()) and torch.all(q[k].float().isnan()) and scales[k].isnan()
        assert torch.all(y[4] == 0) and torch.all(q[4].float() == 0) and scales[4] == 0
        for k in (0, 5):
            assert torch.all(y[k].isfinite()) and torch.all(q[k].float().isfinite()) and scales[k] > 0


def test_one_column_is_its_bias():
    x, w = matrix(5, 1, F32, 1)[0], torch.full((1,), 3.0, device="cuda")
    b, y = torch.full((1,), 0.25, device="cuda"), torch.empty(5, 1, device="cuda")
    cleave.layer_norm(x, w, y, bias=b)
    assert torch.all(y == 0.25)


def test_in_place():
    for cols in (1000, 40000):
        x, r = matrix(5, cols, BF16, 1)[0].contiguous(), matrix(5, cols, BF16, 2)[0].contiguous()
        w = torch.ones(cols, device="cuda")
        y, s = torch.empty_like(x), torch.empty_like(x)
        cleave.layer_norm(x, w, y, residual=r, sum_out=s)
        x2, r2 = x.clone(), r.clone()
        cleave.layer_norm(x2, w, x2, residual=r2, sum_out=r2)        # y over x, the sum over the residual
        assert torch.equal(y, x2) and torch.equal(s, r2)


def test_no_rows():
    w, x = torch.ones(64, device="cuda"), torch.empty(0, 64, device="cuda")
    cleave.layer_norm(x, w, torch.empty_like(x), bias=w)
    dw, db = torch.full((64,), 7.0, device="cuda"), torch.full((64,), 7.0, device="cuda")
    ws, none = torch.empty(cleave.layer_norm_workspace(0, 64), device="cuda"), torch.empty(0, device="cuda")
    cleave.layer_norm_backward(x, x, w, none, none, torch.empty_like(x), dw, ws, dbias=db)
    assert torch.all(dw == 0) and torch.all(db == 0)


def check_backward(rows, cols, dtype, dsum, bias=True, pad=0, shift=0):
    h = matrix(rows, cols, dtype, 1, pad, shift, 2.0, 0.5)[0]
    dy = matrix(rows, cols, dtype, 2, pad, shift)[0]
    ds = matrix(rows, cols, dtype, 3, pad, shift)[0] if dsum else None
    w = matrix(1, cols, F32, 4)[0][0] + 1
    m = h.double().mean(dim=1).float()
    inv = (1 / ((h.double() - m.double()[:, None]).square().mean(dim=1) + EPS).sqrt()).float()
    dx, dx_whole = matrix(rows, cols, dtype, 0, pad, shift, None)
    (dw, dw_whole), (db, db_whole) = floats(cols), floats(cols)
    ws = torch.full((cleave.layer_norm_workspace(rows, cols),), float("nan"), device="cuda")
    cleave.layer_norm_backward(dy, h, w, m, inv, dx, dw, ws, dbias=db if bias else None, dsum=ds)
    xhat = (h.double() - m.double()[:, None]) * inv.double()[:, None]
    g, up = dy.double() * w.double(), dy.double()
    want = inv.double()[:, None] * (g - g.mean(dim=1, keepdim=True) - xhat * (g * xhat).mean(dim=1, keepdim=True))
    if dsum:
        want = want + ds.double()
    n_err = (cols / 64 + 16) * U32
    # roundings of g, the two sums, the products and differences
    size = g.abs() + g.abs().mean(dim=1, keepdim=True) + xhat.abs() * (g * xhat).abs().mean(dim=1, keepdim=True)
    slack = inv.double()[:, None] * (8 * U32 * size + n_err * (size - g.abs())) + 4 * U32 * want.abs()
    near(dx, want, dtype, slack + (2 * U32 * ds.double().abs() if dsum else 0), "dx")
    # a sum over the rows: up to rows / 8 + 64 additions one behind the other; xhat's own roundings
    assert ((dw.double() - (up * xhat).sum(dim=0)).abs() <= (up * xhat).abs().sum(dim=0) * (rows / 8 + 64) * U32).all()
    if bias:
        assert ((db.double() - up.sum(dim=0)).abs() <= up.abs().sum(dim=0) * (rows / 8 + 64) * U32).all()
    for view, whole in ((dx, dx_whole), (dw, dw_whole), (db, db_whole)):
        beside(view, whole)
    return dx, dw, db


@pytest.mark.parametrize("rows,cols", SIZES + [(2500, 64), (2500, 500), (2500, 768), (2500, 1024), (2500, 1111), (2500, 1280),
                                               (2500, 1281), (2500, 1537), (2500, 2000), (2500, 2072), (2100, 4096), (2050, 5120),
                                               (2100, 6145), (1100, 8193), (300, 10241), (300, 12290), (270, 16001), (5000, 256), (9000, 40), (30, 70000)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_backward(rows, cols, dtype):
    check_backward(rows, cols, dtype, dsum=cols % 2 == 0, bias=rows % 3 > 0)


@pytest.mark.parametrize("pad,shift", [(8, 0), (3, 0), (8, 1), (5, 7)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_backward_strides_and_alignment(pad, shift, dtype):
    check_backward(9, 768, dtype, True, True, pad, shift)
    check_backward(3000, 100, dtype, True, True, pad, shift)


@pytest.mark.parametrize("rows,cols", NARROW + [(20000, 64), (40000, 24), (17000, 128), (9000, 200)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_backward_of_narrow_rows(rows, cols, dtype):
    check_backward(rows, cols, dtype, dsum=rows % 2 == 0, bias=cols % 2 == 0)
    check_backward(rows, cols, dtype, True, True, 3, 1)


def test_backward_repeats_its_bits_and_writes_over_its_inputs():
    a, b = check_backward(777, 1000, BF16, True), check_backward(777, 1000, BF16, True)
    assert all(torch.equal(p, q) for p, q in zip(a, b))
    for rows, cols in ((33, 256), (3000, 256), (5, 40000)):
        dy, h, ds = (matrix(rows, cols, F32, k)[0].contiguous() for k in (1, 2, 3))
        m, inv = h.mean(dim=1), 1 / h.std(dim=1)
        w, ws = torch.ones(cols, device="cuda"), torch.empty(cleave.layer_norm_workspace(rows, cols), device="cuda")
        dx, dw = torch.empty_like(dy), torch.empty(cols, device="cuda")
        cleave.layer_norm_backward(dy, h, w, m, inv, dx, dw, ws, dsum=ds)
        for over in range(3):
            t = [dy.clone(), h.clone(), ds.clone()]
            dw2 = torch.empty(cols, device="cuda")
            cleave.layer_norm_backward(t[0], t[1], w, m, inv, t[over], dw2, ws, dsum=t[2])
            assert torch.equal(dx, t[over]) and torch.equal(dw, dw2)


def test_gradient_against_differences_of_the_kernel():
    rows, cols, step = 4, 96, 1.0 / 64
    x, c, d = (matrix(rows, cols, F32, k)[0].contiguous() for k in (1, 2, 3))
    w = torch.ones(cols, device="cuda")
    y, m, inv = torch.empty_like(x), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    cleave.layer_norm(x, w, y, mean=m, inv_std=inv)
    dx, dw = torch.empty_like(x), torch.empty(cols, device="cuda")
    cleave.layer_norm_backward(c, x, w, m, inv, dx, dw, torch.empty(cleave.layer_norm_workspace(rows, cols), device="cuda"))

    def loss(t):
        cleave.layer_norm(t, w, y)
        return float((c.double() * y.double()).sum())

    along = (loss(x + step * d) - loss(x - step * d)) / (2 * step)
    # third order: step^2 / 6 of third derivatives along d (a few times |c| |d|^3 over the row's norm); rounding 1e-6 / step
    assert abs(along - float((dx.double() * d.double()).sum())) <= step ** 2 * 4 * float((c.norm() * d.norm())) / cols ** 0.5 + 1e-3


def test_more_rows_than_one_launch_takes():
    check_norm(2 ** 21 + 77, 3, BF16, BF16)
    check_norm(2 ** 21 + 77, 3, BF16, E4M3)


def test_offsets_beyond_32_bits():
    """Rows that lie 2^27 elements apart: the last begins beyond 2^32 bytes."""
    rows, cols, ld = 18, 100, 2 ** 27
    flat = torch.empty((rows - 1) * ld + cols, dtype=BF16, device="cuda")
    x = flat.as_strided((rows, cols), (ld, 1))
    near_x = matrix(rows, cols, BF16, 1)[0].contiguous()
    x.copy_(near_x)
    w, y, far = torch.ones(cols, device="cuda"), torch.empty_like(near_x), torch.empty_like(near_x)
    m, inv, dw = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"), torch.empty(cols, device="cuda")
    cleave.layer_norm(near_x, w, y, mean=m, inv_std=inv)
    cleave.layer_norm(x, w, far)
    assert torch.equal(y, far)
    ws = torch.empty(cleave.layer_norm_workspace(rows, cols), device="cuda")
    cleave.layer_norm_backward(y, near_x, w, m, inv, far, dw, ws)
    cleave.layer_norm_backward(y, x, w, m, inv, x, dw, ws)
    assert torch.equal(x, far)


def test_on_another_stream_and_in_a_graph():
    x, r = matrix(64, 4096, BF16, 1)[0], matrix(64, 4096, BF16, 2)[0]
    w, b = torch.ones(4096, device="cuda"), torch.zeros(4096, device="cuda")
    y, dw, db = torch.empty(64, 4096, dtype=BF16, device="cuda"), torch.empty(4096, device="cuda"), torch.empty(4096, device="cuda")
    m, inv = torch.empty(64, device="cuda"), torch.empty(64, device="cuda")
    ws = torch.empty(cleave.layer_norm_workspace(64, 4096), device="cuda")
    dx = torch.empty_like(y)

    def step():
        cleave.layer_norm(x, w, y, bias=b, residual=r, mean=m, inv_std=inv)
        cleave.layer_norm_backward(y, x, w, m, inv, dx, dw, ws, dbias=db)

    outs = (y, m, inv, dx, dw, db)
    step()
    want = [t.clone() for t in outs]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(p, q) for p, q in zip(want, outs))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        for t in outs:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(want, outs))


def test_refusals():
    x, w = torch.zeros(4, 64, device="cuda"), torch.ones(64, device="cuda")
    y, s = torch.empty_like(x), torch.empty(4, device="cuda")
    q = torch.empty(4, 64, dtype=E4M3, device="cuda")
    for args, kw in (((x, w[:-1], y), {}), ((x, w, y[:, :-1]), {}), ((x, w, q), {}), ((x, w, y), dict(scales=s)), ((x.t(), w, y), {}),
                     ((x.cpu(), w, y), {}), ((x, w, y), dict(residual=x.bfloat16())), ((x, w, y), dict(bias=w[1:])),
                     ((x, w, y), dict(mean=s[1:])), ((x, w, y), dict(bias=w.bfloat16()))):
        with pytest.raises(ValueError):
            cleave.layer_norm(*args, **kw)
    with pytest.raises(TypeError):
        cleave.layer_norm(x.half(), w, y)
    with pytest.raises(cleave.CleaveError):
        cleave.layer_norm(x, w, y, eps=-1.0)
    with pytest.raises(cleave.CleaveError):
        cleave.layer_norm(x, w, y, mean=s, inv_std=s)                              # two outputs in one place
    with pytest.raises(cleave.CleaveError):
        cleave.layer_norm(torch.zeros(1, 64, device="cuda").expand(4, 64), w, y)   # rows of one place
    ws = torch.empty(cleave.layer_norm_workspace(4, 64), device="cuda")
    with pytest.raises(ValueError):
        cleave.layer_norm_backward(x, x, w, s, s, y, w.clone(), ws[:3])
    with pytest.raises(ValueError):
        cleave.layer_norm_backward(x, x, w, s, s[1:], y, w.clone(), ws)
    with pytest.raises(cleave.CleaveError):
        cleave.layer_norm(x, w, y, sum_out=y)
    dw = torch.empty(64, device="cuda")
    with pytest.raises(cleave.CleaveError):
        cleave.layer_norm_backward(x, x, w, s, s, y, dw, ws, dbias=dw)
