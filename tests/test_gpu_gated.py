"""Gated product and its gradient against fp64: every kernel by name, types, layouts, sizes, strides; what they refuse."""
import math

import pytest
import torch

import paper_2512_22142_amd as cleave

pytestmark = pytest.mark.gpu

F32, BF16, E4M3 = torch.float32, torch.bfloat16, torch.float8_e4m3fn
U32, U16 = 2.0 ** -24, 2.0 ** -8   # unit roundoffs: 24 and 8 bits of significand
ACTS = ["none", "relu", "gelu_tanh", "silu"]


def matrix(rows, cols, dtype, seed, pad=0, shift=0, std=1.0):
    """A rows x cols view, `shift` elements into a buffer of sevens with a leading dimension of cols + pad, and the buffer."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    flat = torch.full((rows * (cols + pad) + shift + 64,), 7.0, device="cuda").to(dtype)
    view = flat[shift: shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    if std is not None:
        view.copy_((torch.randn(rows, cols, generator=g, device="cuda") * std).to(dtype))
    return view, flat


def beside(view, whole):
    """Nothing is written beside the view."""
    keep = view.clone()
    view.fill_(7.0)
    assert torch.all(whole.float() == 7.0)
    view.copy_(keep)


def act_of(z, name):
    if name == "relu":
        return z.clamp_min(0)
    if name == "silu":
        return z * torch.sigmoid(z)
    if name == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    return z


def slope_of(z, name):
    if name == "none":
        return torch.ones_like(z)
    if name == "relu":      # zero at zero
        return (z > 0).double()
    z = z.clone().requires_grad_()
    return torch.autograd.grad(act_of(z, name).sum(), z)[0]


def f64(t):
    return t.float().double() if t.dtype == E4M3 else t.double()


def product_error(a, b):
    """K products summed in fp32, in any order: an eleven-sigma bound of a random walk."""
    return 8 * U32 * torch.outer(a.norm(dim=1), b.norm(dim=0))


def check(M, N, K, dtype=BF16, out=None, transB=0, act="silu", bias=False, keep=False, pad=0, shift=0, merged=False, workspace=None,
          up_first=False):
    out = out or (BF16 if dtype == E4M3 else dtype)
    transB = 1 if dtype == E4M3 else transB
    std = 50.0 if dtype == E4M3 else 1.0
    ipad, ishift = (16 * pad, 0) if dtype == E4M3 else (pad, shift)
    A = matrix(M, K, dtype, 1, ipad, ishift, std)[0]
    if merged:      # halves of one matrix
        w = matrix(*((2 * N, K) if transB else (K, 2 * N)), dtype, 2, ipad, ishift, std / K ** 0.5)[0]
        Bg, Bu = (w[:N], w[N:]) if transB else (w[:, :N], w[:, N:])
    else:
        Bg, Bu = (matrix(*((N, K) if transB else (K, N)), dtype, k, ipad, ishift, std / K ** 0.5)[0] for k in (2, 3))
    if up_first:    # in front of gate in memory
        Bg, Bu = Bu, Bg
    C, C_whole = matrix(M, N, out, 0, pad, shift, None)
    bg, bu = (matrix(1, N, F32, k)[0][0] if bias else None for k in (4, 5))
    (zg, zg_whole), (zu, zu_whole) = (matrix(M, N, out, 0, pad + k, shift, None) if keep else (None, None) for k in (1, 2))
    scale = lambda n, seed: matrix(1, n, F32, seed)[0][0].abs() / 50 if dtype == E4M3 else None   # noqa: E731
    sa, sg, su = scale(M, 6), scale(N, 7), scale(N, 8)
    plan = cleave.plan_gated(M, N, K, dtype)
    if workspace is None:
        workspace = cleave.gated_workspace(plan)
    ws = torch.full((workspace,), float("nan"), device="cuda")
    cleave.linear_gated(plan, A, Bg, Bu, C, transB=transB, act=act, bias_gate=bg, bias_up=bu, gate=zg, up=zu, scale_a=sa,
                        scale_gate=sg, scale_up=su, partials=ws)
    a, wg, wu = f64(A), f64(Bg), f64(Bu)
    wg, wu = (wg.t().contiguous(), wu.t().contiguous()) if transB else (wg, wu)
    if dtype == E4M3:
        a, wg, wu = a * sa.double()[:, None], wg * sg.double(), wu * su.double()
    g, u = a @ wg, a @ wu
    # the scales' two products; the bias's addition
    g_err, u_err = product_error(a, wg) + 2 * U32 * g.abs(), product_error(a, wu) + 2 * U32 * u.abs()
    if bias:
        g, u = g + bg.double(), u + bu.double()
    g_err, u_err = g_err + 2 * U32 * g.abs(), u_err + 2 * U32 * u.abs()
    half = U16 if out == BF16 else U32
    if keep:
        for got, want, err, whole in ((zg, g, g_err, zg_whole), (zu, u, u_err, zu_whole)):
            assert torch.all((got.double() - want).abs() <= half * 1.01 * want.abs() + err), plan.last_kernel
            beside(got, whole)
    # slopes are below 1.2; the sigmoid's argument is known to 2^-23, and it to a few ulps: 32 roundings of the activation
    value = act_of(g, act)
    value_err = 1.2 * g_err + 32 * U32 * (1 + g.abs())
    want = value * u
    err = value_err * (u.abs() + u_err) + value.abs() * u_err + 2 * U32 * want.abs()
    bad = (C.double() - want).abs() - (half * 1.01 * want.abs() + err)
    assert bad.max() <= 0, (plan.last_kernel, float(bad.max()), divmod(int(bad.argmax()), N))
    beside(C, C_whole)
    return C, plan.last_kernel


@pytest.mark.parametrize("M,N,K,name", [
    (4096, 2048, 192, "gated_direct_bf16_256x128"), (4096, 4096, 128, "gated_direct_bf16_256x128"),
    (4000, 4040, 200, "gated_direct_bf16_256x128"), (2048, 1280, 200, "gated_direct_bf16_128x64"),
    (1280, 1024, 264, "gated_direct_bf16_128x64_deep"), (1271, 1000, 320, "gated_direct_bf16_128x64_deep"),
    (100, 304, 136, "gated_direct_bf16_64x32"), (300, 200, 512, "gated_direct_bf16_64x32"), (17, 8, 8, "gated_direct_bf16_64x32"),
    (64, 24, 1032, "gated_direct_bf16_64x32")])
@pytest.mark.parametrize("transB", [0, 1])
@pytest.mark.parametrize("out", [BF16, F32])
def test_every_shape_of_the_direct_kernel(M, N, K, name, transB, out):
    kernel = name + ("_nt" if transB else "_nn")
    for kw in (dict(act="silu"), dict(act="gelu_tanh", bias=True, keep=True), dict(act="relu", pad=1, keep=True)):
        if "pad" in kw:                     # (outputs of any stride; the operands' stay whole)
            kw = {**kw, "pad": 8}
        C, used = check(M, N, K, out=out, transB=transB, workspace=0, **kw)
        assert used == kernel
    assert check(M, N, K, out=out, transB=transB, merged=True, workspace=0)[1] == kernel
    assert check(M, N, K, out=out, transB=transB, merged=True, up_first=True, workspace=0)[1] == kernel


@pytest.mark.parametrize("M,N,K", [(100, 301, 136), (1300, 1027, 200), (4000, 2049, 192), (33, 1, 64)])
def test_ragged_columns_of_weights_stored_by_column(M, N, K):
    for out in (BF16, F32):
        assert "direct" in check(M, N, K, out=out, transB=1, keep=True, bias=True, workspace=0)[1]


@pytest.mark.parametrize("M,N,K,name", [(4096, 2048, 192, "gated_direct_e4m3_128x64_nt"), (2049, 2047, 208, "gated_direct_e4m3_128x64_nt"),
                                        (1280, 1024, 256, "gated_direct_e4m3_128x64_deep_nt"),
                                        (1271, 1001, 272, "gated_direct_e4m3_128x64_deep_nt"),
                                        (100, 300, 144, "gated_direct_e4m3_64x32_nt"), (17, 5, 16, "gated_direct_e4m3_64x32_nt")])
@pytest.mark.parametrize("out", [BF16, F32])
def test_8_bit_operands(M, N, K, name, out):
    for kw in (dict(), dict(act="gelu_tanh", bias=True, keep=True), dict(act="none", pad=1), dict(merged=True)):
        assert check(M, N, K, E4M3, out, **kw)[1] == name


@pytest.mark.parametrize("M,N,K", [(169, 256, 7680), (64, 128, 6192), (4086, 64, 10880), (33, 264, 6016)])
@pytest.mark.parametrize("out", [BF16, F32])
def test_8_bit_operands_with_a_split_inner_dimension(M, N, K, out):
    plan = cleave.plan_gated(M, N, K, E4M3)
    assert cleave.gated_workspace(plan) > 2 * M * N and cleave.gated_workspace(plan, whole=True) == cleave.gated_workspace(plan)
    for kw in (dict(), dict(act="gelu_tanh", bias=True, keep=True), dict(pad=1, shift=1), dict(merged=True, up_first=True)):
        check(M, N, K, E4M3, out, **kw)


@pytest.mark.parametrize("M,N,K,splits", [(46, 1280, 4800, 3), (17, 2560, 5120, 4), (130, 200, 2048, 4), (40, 2048, 2304, 2), (200, 11008, 4096, 2),
                                          (450, 4096, 8192, 4), (17, 2816, 1024, 1), (300, 4096, 2048, 1)])
@pytest.mark.parametrize("transB", [0, 1])
def test_splits_of_the_inner_dimension(M, N, K, splits, transB):
    plan = cleave.plan_gated(M, N, K, BF16)
    assert cleave.gated_workspace(plan, whole=True) == (splits * 2 * M * N if splits > 1 else 0)
    check(M, N, K, transB=transB, keep=True)
    check(M, N, K, transB=transB, act="gelu_tanh", bias=True, out=F32, merged=True)
    check(M, N, K, transB=transB, act="relu", pad=3, shift=1)


FEW = [(1, 11008, 256), (1, 64, 64), (2, 1, 16), (16, 1000, 512), (5, 4096, 4096), (3, 300, 4096), (16, 77, 8192), (7, 9000, 48)]


@pytest.mark.parametrize("M,N,K", FEW)
@pytest.mark.parametrize("dtype,transB", [(BF16, 0), (BF16, 1), (F32, 0), (F32, 1), (E4M3, 1)])
def test_few_rows(M, N, K, dtype, transB):
    direct = dtype == BF16 and K <= 1024 and N <= 4096 and (transB or N % 8 == 0)     # (whole operands, short K)
    for kw in (dict(), dict(act="gelu_tanh", bias=True, keep=True, out=F32)):
        name = check(M, N, K, dtype, transB=transB, **kw)[1]
        assert name == "gated_few_rows" if not direct else name.startswith("gated_direct_bf16_64x32"), name
    if dtype != E4M3:
        check(M, N, K, dtype, transB=transB, pad=3, shift=1, keep=True)
        check(M, N, K - 1, dtype, transB=transB, act="relu")


@pytest.mark.parametrize("M,N,K,names", [(1, 8200, 4104, ("few", "direct")), (13, 12200, 4096, ("few", "direct")), (16, 12296, 4096, ("few", "few")),
                                         (3, 4096, 1024, ("direct", "direct")), (15, 4104, 1024, ("few", "few")), (1, 8, 8, ("direct", "direct")),
                                         (16, 1000, 1000, ("direct", "direct")), (2, 1003, 96, ("few", "direct")), (4, 8200, 4088, ("few", "few"))])
def test_few_rows_on_the_direct_kernel(M, N, K, names):
    for transB in (0, 1):
        for kw in (dict(), dict(bias=True, keep=True, act="gelu_tanh", out=F32), dict(merged=True)):
            if kw.get("merged") and N % 8 and not transB:
                continue
            name = check(M, N, K, transB=transB, **kw)[1]
            assert ("gated_direct" in name) == (names[transB] == "direct"), name
        check(M, N, K, transB=transB, shift=1)
        check(M, N, K, transB=transB, pad=1)
    plan = cleave.plan_gated(M, N, K, BF16)
    if names == ("direct", "direct"):
        assert cleave.gated_workspace(plan, whole=True) == 0


@pytest.mark.parametrize("M,N,K", [(17, 1, 1), (37, 53, 71), (200, 50, 100), (129, 257, 65), (300, 77, 1000), (64, 512, 4096),
                                   (33, 128, 3001), (500, 1000, 1000), (1100, 2052, 333), (2000, 2500, 200), (400, 300, 1003),
                                   (800, 1001, 328), (2049, 4100, 72), (900, 1, 9)])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("transB", [0, 1])
def test_any_size_and_alignment(M, N, K, dtype, transB):
    check(M, N, K, dtype, transB=transB, bias=True, keep=True)
    check(M, N, K, dtype, transB=transB, act="gelu_tanh", pad=3, shift=1, out=F32)
    check(M, N, K, dtype, transB=transB, act="relu", merged=True)


def test_operands_that_are_laid_out_again():
    """bf16 with rows, addresses or sizes that are not whole sixteen bytes run on the direct kernel where there are rows enough."""
    for M, N, K, kw in ((400, 301, 203, dict(transB=0)), (400, 301, 203, dict(transB=1)), (800, 301, 200, dict(transB=0)),
                        (800, 304, 200, dict(transB=1, pad=3)), (800, 304, 200, dict(transB=0, shift=1)), (800, 304, 200, dict(transB=1, shift=4))):
        assert "gated_direct" in check(M, N, K, bias=True, keep=True, **kw)[1]
        assert "gated_direct" in check(M, N, K, merged=True, **kw)[1]
    for M, N, K, kw in ((400, 304, 203, dict(transB=0)), (400, 304, 203, dict(transB=1)), (400, 304, 200, dict(transB=0, pad=3)),
                        (2050, 301, 2050, dict(transB=0)), (2050, 301, 2056, dict(transB=1, shift=1))):
        assert "gated_grad_direct" in check_grad(M, N, K, **kw)


def test_the_workspace_is_all_that_is_used():
    """NaN behind the workspace stay, and what is in it does not count."""
    for M, N, K in ((800, 301, 203), (300, 301, 203), (9, 300, 8192)):
        plan = cleave.plan_gated(M, N, K, BF16)
        n = cleave.gated_workspace(plan)
        for shift in (0, 1, 3):          # floats of any alignment
            whole = torch.full((n + 64,), float("nan"), device="cuda")
            x, w = matrix(M, K, BF16, 1)[0], matrix(K, 2 * N, BF16, 2, 0, 0, 0.1)[0]
            y = torch.empty(M, N, dtype=BF16, device="cuda")
            cleave.linear_gated(plan, x, w[:, :N], w[:, N:], y, partials=whole[shift: shift + n])
            assert torch.all(y.isfinite()) and torch.all(whole[shift + n:].isnan()) and torch.all(whole[:shift].isnan())


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("M,N,K,dtype", [(1, 500, 128, BF16), (200, 200, 128, BF16), (200, 200, 130, F32), (200, 200, 128, E4M3)])
def test_activations(act, M, N, K, dtype):
    check(M, N, K, dtype, act=act, bias=True, keep=True)


def check_grad(M, N, K, dtype=BF16, out=None, transB=1, act="silu", pad=0, shift=0, side_by_side=False, in_place=False, workspace=None):
    out = out or dtype
    A = matrix(M, K, dtype, 1, pad, shift)[0]
    B = matrix(*((N, K) if transB else (K, N)), dtype, 2, pad, shift, 1 / K ** 0.5)[0]
    zg, zu = matrix(M, N, out, 3, pad, shift, 2.0)[0], matrix(M, N, out, 4, pad + 1, shift, 2.0)[0]
    if side_by_side:
        both, whole = matrix(M, 2 * N, out, 0, pad, shift, None)
        dg, du = both[:, :N], both[:, N:]
    else:
        (dg, dg_whole), (du, du_whole) = matrix(M, N, out, 0, pad, shift, None), matrix(M, N, out, 0, pad + 2, shift, None)
    g, u = zg.double(), zu.double()
    if in_place:
        dg, du = zg, zu
    plan = cleave.plan_linear(M, N, K, dtype)
    ws = torch.full((cleave.gated_grad_workspace(plan) if workspace is None else workspace,), float("nan"), device="cuda")
    cleave.linear_gated_grad(plan, A, B, zg, zu, dg, du, transB=transB, act=act, partials=ws)
    a, b = A.double(), B.double()
    b = b.t().contiguous() if transB else b
    p, p_err = a @ b, product_error(a, b)
    half = U16 if out == BF16 else U32
    value, slope = act_of(g, act), slope_of(g, act)
    # 32 roundings of the activation, 64 of the slope (the sigmoid's argument is known to 2^-23, and it to a few ulps)
    for got, factor, factor_err in ((dg, u * slope, 64 * U32 * u.abs()), (du, value, 32 * U32 * (1 + g.abs()))):
        want = p * factor
        err = p_err * (factor.abs() + factor_err) + p.abs() * factor_err + 3 * U32 * want.abs()
        bad = (got.double() - want).abs() - (half * 1.01 * want.abs() + err)
        assert bad.max() <= 0, (plan.last_kernel, float(bad.max()), divmod(int(bad.argmax()), N))
    if side_by_side:
        beside(both, whole)
    elif not in_place:
        beside(dg, dg_whole)
        beside(du, du_whole)
    return plan.last_kernel


@pytest.mark.parametrize("M,N,K,name", [
    (4096, 4096, 192, "gated_grad_direct_bf16_256x256"), (4000, 4040, 200, "gated_grad_direct_bf16_256x256"),
    (8192, 4096, 128, "gated_grad_direct_bf16_256x256"), (2048, 2560, 200, "gated_grad_direct_bf16_128x128"),
    (1280, 2048, 264, "gated_grad_direct_bf16_128x128_deep"), (100, 304, 136, "gated_grad_direct_bf16_64x64"),
    (17, 8, 8, "gated_grad_direct_bf16_64x64")])
@pytest.mark.parametrize("transB", [0, 1])
@pytest.mark.parametrize("out", [BF16, F32])
def test_gradient_in_every_shape_of_the_direct_kernel(M, N, K, name, transB, out):
    for kw in (dict(), dict(act="gelu_tanh", side_by_side=True), dict(act="relu", in_place=True), dict(pad=8)):
        assert check_grad(M, N, K, out=out, transB=transB, workspace=0, **kw) == name + ("_nt" if transB else "_nn")


@pytest.mark.parametrize("M,N,K", [(1, 1, 1), (1, 2752, 1024), (16, 1000, 77), (9, 300, 8192), (37, 53, 71), (129, 257, 65), (300, 77, 1000),
                                   (64, 512, 4096), (33, 128, 3001), (1100, 2052, 333), (400, 304, 1003), (2050, 1001, 2051),
                                   (2050, 513, 2056), (500, 8, 9)])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("transB", [0, 1])
def test_gradient_of_any_size_and_alignment(M, N, K, dtype, transB):
    for kw in (dict(), dict(act="gelu_tanh", pad=3, shift=1, out=F32), dict(act="relu", side_by_side=True), dict(in_place=True)):
        check_grad(M, N, K, dtype, transB=transB, **kw)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("M,N,K,dtype", [(3, 500, 128, BF16), (200, 200, 128, BF16), (200, 200, 130, F32)])
def test_gradient_of_every_activation(act, M, N, K, dtype):
    check_grad(M, N, K, dtype, act=act)


def test_gradient_against_differences_of_the_kernel():
    """The product's two arguments moved by hand: with K = 1 and a column of ones for A, they are the weights."""
    N, step = 96, 1.0 / 64
    g, u, c, dg, du = (matrix(1, N, F32, k)[0].contiguous() for k in (1, 2, 3, 4, 5))
    one = torch.ones(1, 1, device="cuda")
    for act in ACTS:
        plan = cleave.plan_gated(1, N, 1, F32)
        ws = torch.empty(max(1, cleave.gated_workspace(plan)), device="cuda")

        def loss(t):
            y = torch.empty(1, N, device="cuda")
            cleave.linear_gated(plan, one, g + t * dg, u + t * du, y, act=act, partials=ws)
            return float((c.double() * y.double()).sum())

        # p = c: the product of a row of ones' entry with it
        back = cleave.plan_linear(1, N, 1, F32)
        a, b = torch.empty_like(g), torch.empty_like(g)
        cleave.linear_gated_grad(back, one, c, g, u, a, b, act=act,
                                 partials=torch.empty(max(1, cleave.gated_grad_workspace(back)), device="cuda"))
        along = (loss(step) - loss(-step)) / (2 * step)
        got = float((a.double() * dg.double() + b.double() * du.double()).sum())
        # third order: step^2 / 6 of third derivatives, below 4 |c| |d|^3 (1 + |u|) for these; an element at relu's corner moves
        # within |step d| of it: step |d|^2 (|u| + |d|) at most
        cubes = float((c.abs() * (dg.abs() + du.abs()) ** 3 * (1 + u.abs())).sum())
        corner = float(((g.abs() <= step * dg.abs()) * c.abs() * dg.abs() * (u.abs() + du.abs())).sum()) if act == "relu" else 0.0
        assert abs(along - got) <= step ** 2 * 4 * cubes + corner + 1e-3, act


def test_repeats_its_bits_on_another_stream_and_in_a_graph():
    M, N, K = 300, 512, 256
    x, w, wd = matrix(M, K, BF16, 1)[0], matrix(K, 2 * N, BF16, 2, 0, 0, 0.1)[0], matrix(N, K, BF16, 3, 0, 0, 0.1)[0]
    y, zg, zu = (torch.empty(M, N, dtype=BF16, device="cuda") for _ in range(3))
    dz = torch.empty(M, 2 * N, dtype=BF16, device="cuda")
    one = torch.empty(1, N, dtype=BF16, device="cuda")
    plan, back, single = cleave.plan_gated(M, N, K, BF16), cleave.plan_linear(M, N, K, BF16), cleave.plan_gated(1, N, K, BF16)
    odd = cleave.plan_gated(M, N - 3, K, BF16)          # not in whole sixteen bytes
    y_odd = torch.empty(M, N - 3, dtype=BF16, device="cuda")
    ws = torch.empty(max(cleave.gated_workspace(odd), cleave.gated_workspace(single), cleave.gated_grad_workspace(back)), device="cuda")
    for p in (plan, back, single, odd):
        p.upload()

    def step():
        cleave.linear_gated(plan, x, w[:, :N], w[:, N:], y, gate=zg, up=zu, partials=ws)
        cleave.linear_gated_grad(back, x, wd, zg, zu, dz[:, :N], dz[:, N:], transB=1, partials=ws)
        cleave.linear_gated(single, x[:1], w[:, :N], w[:, N:], one, partials=ws)
        cleave.linear_gated(odd, x, w[:, :N - 3], w[:, N:-3], y_odd, partials=ws)

    outs = (y, zg, zu, dz, one, y_odd)
    step()
    want = [t.clone() for t in outs]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(want, outs))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        for t in outs:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, outs))


def test_values_that_are_not_finite_stay_in_their_rows():
    for M in (3, 40):
        x, w = matrix(M, 64, BF16, 1)[0].contiguous(), matrix(64, 64, BF16, 2)[0].contiguous()
        x[1, 5], x[2, 6] = float("nan"), float("inf")
        y = torch.empty(M, 32, dtype=BF16, device="cuda")
        plan = cleave.plan_gated(M, 32, 64, BF16)
        cleave.linear_gated(plan, x, w[:, :32], w[:, 32:], y, act="relu",
                            partials=torch.empty(max(1, cleave.gated_workspace(plan)), device="cuda"))
        assert torch.all(y[1].isnan()) and not torch.any(y[2].isfinite() & (y[2] != 0))
        rest = [k for k in range(M) if k not in (1, 2)]
        assert torch.all(y[rest].isfinite())


def test_refusals():
    M, N, K = 40, 64, 32
    x, w, y = matrix(M, K, BF16, 1)[0], matrix(K, N, BF16, 2)[0], torch.empty(M, N, dtype=BF16, device="cuda")
    plan = cleave.plan_gated(M, N, K, BF16)
    for args, kw in (((x, w, w[:, :-1], y), {}), ((x[:-1], w, w, y), {}), ((x, w, w, y[:-1]), {}), ((x, w, w, y), dict(gate=y[:, 1:])),
                     ((x, w, w, y), dict(gate=y.float())), ((x, w, w, y), dict(bias_gate=y[0])), ((x.cpu(), w, w, y), {}),
                     ((x, w, w, y), dict(act="tanh")), ((x, w, w, y), dict(scale_a=torch.ones(M, device="cuda"))),
                     ((x, matrix(K, N, BF16, 3, 8)[0], w, y), {})):
        with pytest.raises(ValueError):
            cleave.linear_gated(plan, *args, **kw)
    with pytest.raises(TypeError):
        cleave.linear_gated(plan, x, w.float(), w, y)
    with pytest.raises(TypeError):
        cleave.linear_gated(plan, x, w, w, y.half())
    with pytest.raises(TypeError):
        cleave.plan_gated(M, N, K, torch.float16)
    for kw in (dict(gate=y), dict(up=y), dict(gate=torch.empty_like(y))):
        if len(kw) == 1 and "gate" in kw and kw["gate"] is not y:
            kw["up"] = kw["gate"]
        with pytest.raises(cleave.CleaveError):
            cleave.linear_gated(plan, x, w, w, y, **kw)
    with pytest.raises(cleave.CleaveError):
        cleave.linear_gated(cleave.plan_linear(M, N, K, BF16), x, w, w, y)
    with pytest.raises(cleave.CleaveError):     # operands that are not whole sixteen bytes, and no workspace
        cleave.linear_gated(plan, matrix(M, K, BF16, 1, 1)[0], w, w, y)
    with pytest.raises(cleave.CleaveError):
        cleave.linear(plan, x, w, y)
    with pytest.raises(cleave.CleaveError):
        cleave.execute(plan, x, w, torch.empty(plan.partial_elems, device="cuda"))
    back = cleave.plan_linear(M, N, K, BF16)
    a, b = torch.empty_like(y), torch.empty_like(y)
    with pytest.raises(cleave.CleaveError):
        cleave.linear_gated_grad(back, x, w, y, y.clone(), a, a)
    with pytest.raises(cleave.CleaveError):
        cleave.linear_gated_grad(back, x, w, a, b, b, y)
    with pytest.raises(ValueError):
        cleave.linear_gated_grad(back, x, w, y, y[:-1], a, b)
    with pytest.raises(cleave.CleaveError):
        cleave.linear_gated_grad(plan, x, w, y, y.clone(), a, b)
    with pytest.raises(cleave.CleaveError):
        cleave.gated_workspace(back)
    with pytest.raises(cleave.CleaveError):
        cleave.gated_grad_workspace(plan)
