"""Linear product with its epilogue against fp64: layouts, types, sizes from one row on, strides, splits; its refusals."""
import numpy as np
import pytest
import torch

import paper_2512_22142_amd as cleave
from oracle import operators as oo

pytestmark = pytest.mark.gpu

F32, BF16, E4M3 = torch.float32, torch.bfloat16, torch.float8_e4m3fn
U32, U16 = 2.0 ** -24, 2.0 ** -8   # unit roundoffs: 24 and 8 bits of significand
ACTS = ["none", "relu", "gelu_tanh", "silu"]


def matrix(rows, cols, dtype, seed, pad=0, shift=0, std=1.0):
    """A rows x cols view on the GPU with a leading dimension of cols + pad, `shift` elements into its buffer, and the buffer."""
    g = torch.Generator().manual_seed(seed)
    flat = torch.full((rows * (cols + pad) + shift + 64,), 7.0, device="cuda").to(dtype)
    view = flat[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    if std is not None:
        view.copy_((torch.randn(rows, cols, generator=g) * std).to(dtype))
    return view, flat


def f64(t):
    return None if t is None else t.double().cpu().numpy()


def check(M, N, K, dtype=BF16, out=None, transA=0, transB=0, act="none", grad=False, bias=False, residual=False, preact=False,
          plan=None, pad=0, shift=0, in_place=False, seed=0):
    out = out or (BF16 if dtype == E4M3 else dtype)
    if dtype == E4M3:
        transB, std = 1, 50.0
    else:
        std = 1.0
    ipad = pad if dtype != E4M3 else 16 * (pad // 16)
    A, _ = matrix(*((K, M) if transA else (M, K)), dtype, seed + 1, ipad, 0 if dtype == E4M3 else shift, std)
    B, _ = matrix(*((N, K) if transB else (K, N)), dtype, seed + 2, ipad, 0 if dtype == E4M3 else shift, std / K ** 0.5)
    C, whole = matrix(M, N, out, seed + 3, pad, shift, None)
    b = matrix(1, N, F32, seed + 4)[0][0] if bias else None
    r = matrix(M, N, out, seed + 5, pad + 1, shift)[0] if residual else None
    z, z_whole = matrix(M, N, out, seed + 6, pad, shift, 2.0 if grad else None) if preact or grad else (None, None)
    sa = matrix(1, M, F32, seed + 7)[0][0].abs() / 50 if dtype == E4M3 else None
    sb = matrix(1, N, F32, seed + 8)[0][0].abs() / 50 if dtype == E4M3 else None
    if in_place:
        C.copy_(r)
        r = C
    opA, opB = f64(A.float()), f64(B.float())
    opA, opB = opA.T if transA else opA, opB.T if transB else opB
    want_r, want_z = f64(r), f64(z)
    plan = plan or cleave.plan_linear(M, N, K, dtype)
    partials = torch.full((max(1, plan.linear_workspace),), float("nan"), device="cuda")
    kw = dict(act_grad=act) if grad else dict(act=act)
    cleave.linear(plan, A, B, C, transA, transB, bias=b, residual=r, preact=z, scale_a=sa, scale_b=sb, partials=partials, **kw)
    torch.cuda.synchronize()
    # sums of K products in fp32: 8 * 2^-24 |a| |b| (an eleven-sigma bound of a random walk), exact products
    s, t = (f64(sa), f64(sb)) if dtype == E4M3 else (np.ones(M), np.ones(N))
    err = 8 * U32 * np.outer(np.linalg.norm(opA, axis=1) * s, np.linalg.norm(opB, axis=0) * t)
    if dtype == E4M3 and out == BF16 and M > 16:
        # the 8-bit instruction drops what lies below 2^-13 of the largest product of a group: up to that per product, of
        # either sign (uniform: standard deviation 2^-13 / sqrt(3)), six sigma
        most = np.outer(np.abs(opA).max(axis=1) * s, np.abs(opB).max(axis=0) * t)
        err = err + 6 / 3 ** 0.5 * K ** 0.5 * 2.0 ** -13 * most
    if grad:
        sums = (opA @ opB) * s[:, None] * t
        slope = oo.act_grad(want_z, act)
        want = sums * slope
        # the slope: sigmoid to a few ulps of an argument known to 2^-23, times z up to where it matters
        err = err * 1.2 + np.abs(sums) * 64 * U32
    else:
        want, zz = oo.linear(opA, opB, f64(b), act, None, s, t)
        err = err + 4 * U32 * np.abs(zz)
        if preact:
            u = U16 if out == BF16 else U32
            assert np.all(np.abs(f64(z) - zz) <= u * 1.01 * np.abs(zz) + err), "preact"
            beside(z_whole, z)
        err = err * 1.2 + 32 * U32 * (1 + np.abs(zz))
    if residual:
        want = want + want_r
    u = U16 if out == BF16 else U32
    bad = np.abs(f64(C) - want) - (u * 1.01 * np.abs(want) + err + 2 * U32 * np.abs(want))
    assert np.all(bad <= 0), (plan.last_kernel, float(bad.max()), np.unravel_index(np.argmax(bad), bad.shape))
    beside(whole, C)
    return C, z, plan.last_kernel


def beside(whole, view):
    """Nothing is written beside the view: the rest of its buffer still holds sevens."""
    keep = view.clone()
    view.fill_(7.0)
    assert torch.all(whole.float() == 7.0)
    view.copy_(keep)


EPILOGUES = [dict(), dict(bias=True, act="gelu_tanh", preact=True), dict(bias=True, act="silu", residual=True),
             dict(act="relu", residual=True, preact=True), dict(grad=True, act="gelu_tanh"), dict(grad=True, act="silu", residual=True),
             dict(grad=True, act="relu")]
FEW = [(1, 128, 256), (1, 1408, 64), (1, 8, 8), (3, 136, 72), (16, 256, 512), (17, 264, 520), (33, 128, 1000), (64, 512, 4096),
       (2, 4096, 4096), (40, 96, 2048), (1, 3076, 1024), (15, 11008, 160), (7, 3136, 40), (9, 100, 2056)]
MANY = [(65, 128, 64), (128, 256, 64), (130, 264, 96), (256, 256, 256), (300, 520, 200), (513, 256, 64), (1000, 768, 1024),
        (2048, 512, 128), (1100, 4096, 512)]
ODD = [(1, 1, 1), (5, 7, 3), (37, 53, 71), (1, 333, 1001), (200, 1, 50), (100, 100, 100), (129, 257, 65), (300, 77, 1000)]


@pytest.mark.parametrize("size", FEW + MANY + ODD)
@pytest.mark.parametrize("epilogue", range(len(EPILOGUES)))
@pytest.mark.parametrize("transB", [0, 1])
def test_bf16(size, epilogue, transB):
    check(*size, transB=transB, **EPILOGUES[epilogue])


@pytest.mark.parametrize("size", FEW + MANY + ODD)
@pytest.mark.parametrize("epilogue", [0, 1, 2, 5])
def test_bf16_into_fp32(size, epilogue):
    check(*size, out=F32, **EPILOGUES[epilogue])


@pytest.mark.parametrize("size", FEW + MANY + ODD)
@pytest.mark.parametrize("epilogue", [0, 1, 2, 4])
@pytest.mark.parametrize("transB", [0, 1])
def test_fp32(size, epilogue, transB):
    check(*size, dtype=F32, transB=transB, **EPILOGUES[epilogue])


E4M3_SIZES = [(1, 128, 256), (1, 11, 16), (3, 136, 80), (16, 257, 512), (33, 130, 1008), (64, 512, 4096), (65, 128, 64), (130, 261, 96),
              (256, 256, 256), (300, 523, 208), (513, 256, 64), (1000, 768, 1024), (100, 64, 4096), (2048, 512, 128),
              (100, 67, 8192), (16, 67, 8208), (9, 200, 11008), (300, 200, 8192), (1100, 203, 6016)]


@pytest.mark.parametrize("size", E4M3_SIZES)
@pytest.mark.parametrize("epilogue", range(len(EPILOGUES)))
def test_e4m3(size, epilogue):
    check(*size, dtype=E4M3, **EPILOGUES[epilogue])
    check(*size, dtype=E4M3, out=F32, pad=16, **EPILOGUES[epilogue])


@pytest.mark.parametrize("size", [(200, 128, 96), (37, 53, 71), (3, 64, 64), (1000, 520, 600)])
@pytest.mark.parametrize("epilogue", [0, 2, 5])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("transB", [0, 1])
def test_a_transposed(size, epilogue, dtype, transB):
    check(*size, dtype=dtype, transA=1, transB=transB, **EPILOGUES[epilogue])


@pytest.mark.parametrize("pad,shift", [(8, 0), (3, 0), (8, 1), (24, 8), (5, 3)])
@pytest.mark.parametrize("size", [(7, 256, 512), (300, 520, 200)])
@pytest.mark.parametrize("dtype,transB", [(BF16, 0), (BF16, 1), (F32, 0), (F32, 1)])
def test_strides_and_alignment(pad, shift, size, dtype, transB):
    check(*size, dtype=dtype, transB=transB, pad=pad, shift=shift, **EPILOGUES[2])
    check(*size, dtype=dtype, transB=transB, pad=pad, shift=shift, **EPILOGUES[5])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("size,tile,splits", [((300, 520, 600), 128, 3), ((65, 100, 1000), 64, 4), ((700, 300, 512), 256, 2),
                                              ((20, 256, 512), 128, 4), ((20, 100, 513), 32, 3)])
def test_plans_with_splits(dtype, size, tile, splits):
    plan = cleave.plan_uniform(*size, tile, tile, splits)
    check(*size, dtype=dtype, plan=plan, **EPILOGUES[1])
    check(*size, dtype=dtype, plan=plan, **EPILOGUES[5])


def test_plans_of_unequal_tiles_and_splits():
    plan = cleave.plan_explicit(300, 200, 512, [100, 200], [[120, 80], [64, 72, 64]], [1, 2, 4, 1, 3])
    for dtype in (BF16, F32):
        check(300, 200, 512, dtype=dtype, plan=plan, **EPILOGUES[2])


@pytest.mark.parametrize("size", [(3, 256, 512), (300, 520, 200), (37, 53, 71), (70, 64, 8192)])
def test_residual_in_place(size):
    check(*size, bias=True, act="silu", residual=True, in_place=True)


def test_which_kernel():
    assert check(1, 128, 256)[2] == "linear_few_rows"
    assert check(16, 4096, 256, transB=1)[2] == "linear_few_rows"
    assert check(16, 132, 256, dtype=F32)[2] == "linear_few_rows"
    assert check(16, 131, 256, dtype=E4M3)[2] == "linear_few_rows"
    assert "direct" in check(17, 128, 256, bias=True)[2]
    assert "direct" in check(512, 512, 512, bias=True)[2]
    assert "direct" in check(512, 512, 512, dtype=E4M3)[2]
    assert "direct" in check(512, 511, 512, transB=1, bias=True)[2]


def test_a_layers_backward_is_the_chain_of_products():
    """dz, dw and db of act(z) . w + b, against fp64 and against differences of the forward kernel."""
    T, fin, fout = 96, 64, 48
    z = matrix(T, fin, F32, 1)[0]
    w = matrix(fin, fout, F32, 2, std=0.2)[0]
    dy = matrix(T, fout, F32, 3)[0]
    a = torch.nn.functional.gelu(z, approximate="tanh")
    dz, dw, db = torch.empty_like(z), torch.empty_like(w), torch.empty(fout, device="cuda")
    to_z, to_w = cleave.plan_linear(T, fin, fout, F32), cleave.plan_linear(fin, fout, T, F32)
    ws = torch.empty(max(1, to_z.linear_workspace, to_w.linear_workspace, cleave.bias_grad_workspace(T, fout)), device="cuda")
    cleave.linear(to_z, dy, w, dz, transB=1, act_grad="gelu_tanh", preact=z, partials=ws)
    cleave.linear(to_w, a, dy, dw, transA=1, partials=ws)
    cleave.bias_grad(dy, db, ws)
    want = (f64(dy) @ f64(w).T) * oo.act_grad(f64(z), "gelu_tanh")
    assert np.allclose(f64(dz), want, rtol=1e-5, atol=1e-5)
    assert np.allclose(f64(dw), f64(a).T @ f64(dy), rtol=1e-5, atol=1e-4)
    # differences along a direction of the forward product's inputs: its kernel is linear in w and in act(z)
    d = matrix(T, fin, F32, 4)[0]
    y = torch.empty(T, fout, device="cuda")
    plan = cleave.plan_linear(T, fout, fin, F32)

    def loss(t):
        h = torch.nn.functional.gelu(t.double(), approximate="tanh").float()
        cleave.linear(plan, h, w, y, partials=ws)
        return float((y.double() * dy.double()).sum())

    step = 1e-2
    along, grad = (loss(z + step * d) - loss(z - step * d)) / (2 * step), float((dz.double() * d.double()).sum())
    # third order: step^2 / 6 times third derivatives (below 2) of T * fin terms of size |dz| |d|^3, signs at random
    assert abs(along - grad) <= step ** 2 * 10 * float(dz.norm()) + 1e-2


def test_bits_repeat_on_another_stream_and_in_a_graph():
    for M, N, K, dtype in ((3, 4096, 4096, BF16), (300, 520, 512, BF16), (100, 64, 4096, E4M3), (80, 256, 4096, F32)):
        A = matrix(M, K, dtype, 1)[0]
        B = matrix(N, K, dtype, 2)[0]
        C = torch.empty(M, N, dtype=BF16, device="cuda")
        bias = torch.randn(N, device="cuda")
        scales = dict(scale_a=torch.rand(M, device="cuda"), scale_b=torch.rand(N, device="cuda")) if dtype == E4M3 else {}
        plan = cleave.plan_linear(M, N, K, dtype)
        plan.upload()
        ws = torch.empty(max(1, plan.linear_workspace), device="cuda")

        def step():
            cleave.linear(plan, A, B, C, transB=1, bias=bias, act="silu", partials=ws, **scales)

        step()
        want = C.clone()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step()
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(want, C)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        for _ in range(3):
            C.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(want, C)


@pytest.mark.parametrize("size", [(3, 256, 512), (300, 520, 200), (37, 53, 71), (100, 64, 4096)])
def test_what_is_not_finite_stays_in_its_row(size):
    M, N, K = size
    A, B = matrix(M, K, BF16, 1)[0], matrix(K, N, BF16, 2)[0]
    A[1] = float("nan")
    A[2, K // 2] = float("inf")
    plan = cleave.plan_linear(M, N, K, BF16)
    ws = torch.empty(max(1, plan.linear_workspace), device="cuda")
    for act in ACTS:
        C = torch.empty(M, N, device="cuda")
        cleave.linear(plan, A, B, C, act=act, partials=ws)
        assert torch.all(C[1].isnan()), act
        assert not torch.any(C[2].isfinite() & (C[2] > 0)), act        # infinite, or what the activation makes of -inf
        C[1:3] = 0
        assert torch.all(C.isfinite()), act
    z = torch.full((M, N), float("inf"), device="cuda")
    z[0] = -float("inf")
    A[1:3] = 1
    for act in ("relu", "gelu_tanh", "silu"):     # slopes at infinity: 1 and 0
        C = torch.empty(M, N, device="cuda")
        plain = torch.empty(M, N, device="cuda")
        cleave.linear(plan, A, B, C, act_grad=act, preact=z, partials=ws)
        cleave.linear(plan, A, B, plain, partials=ws)
        assert torch.all(C[0] == 0) and torch.equal(C[1:], plain[1:]), act


def test_8_bit_values_that_are_not_a_number_stay_in_their_row():
    for M, N, K in ((4, 128, 256), (100, 64, 8192), (300, 523, 208), (600, 512, 512)):
        A, B = matrix(M, K, E4M3, 1, std=50.0)[0], matrix(N, K, E4M3, 2, std=5.0)[0]
        A.view(torch.uint8)[1, K // 3] = 0x7f
        B.view(torch.uint8)[5, K // 2] = 0xff
        plan = cleave.plan_linear(M, N, K, E4M3)
        ws = torch.empty(max(1, plan.linear_workspace), device="cuda")
        for out in (BF16, F32):
            C = torch.empty(M, N, dtype=out, device="cuda")
            cleave.linear(plan, A, B, C, transB=1, scale_a=torch.ones(M, device="cuda"), scale_b=torch.ones(N, device="cuda"),
                          partials=ws)
            assert torch.all(C[1].isnan()) and torch.all(C[:, 5].isnan())
            C[1], C[:, 5] = 0, 0
            assert torch.all(C.isfinite())


def test_a_leading_dimension_beyond_32_bits_of_bytes():
    """Rows 2^31 elements apart in all: offsets of the last rows pass 32 bits."""
    rows, cols = 70000, 64
    wide = torch.empty(rows, 33000, dtype=BF16, device="cuda")     # 4.6 GB
    A = wide[:, :cols]
    A.copy_(torch.randn(rows, cols, device="cuda").to(BF16))
    B = torch.randn(cols, 64, device="cuda").to(BF16)
    C = wide[:, 4096:4160]
    plan = cleave.plan_linear(rows, 64, cols, BF16)
    cleave.linear(plan, A, B, C, act="relu", residual=A)
    last = slice(rows - 300, rows)
    want = (A[last].double().cpu() @ B.double().cpu()).clamp_min(0) + A[last].double().cpu()
    got = C[last].double().cpu()
    assert torch.all((got - want).abs() <= U16 * 1.02 * want.abs() + 1e-4)


def test_refusals():
    A, B, C = (torch.zeros(4, 16, device="cuda"), torch.zeros(16, 8, device="cuda"), torch.empty(4, 8, device="cuda"))
    plan = cleave.plan_linear(4, 8, 16, F32)
    z = torch.zeros(4, 8, device="cuda")
    bad_values = [dict(bias=torch.zeros(7, device="cuda")), dict(bias=torch.zeros(8, device="cuda", dtype=BF16)),
                  dict(residual=z.bfloat16()), dict(residual=z[:, :-1]), dict(preact=z.cpu()), dict(act="tanh"),
                  dict(act="relu", act_grad="relu"), dict(scale_a=torch.zeros(4, device="cuda")), dict(transB=1), dict(transA=1)]
    for bad in bad_values:
        with pytest.raises(ValueError):
            cleave.linear(plan, A, B, C, **bad)
    with pytest.raises(TypeError):
        cleave.linear(plan, A, B.bfloat16(), C)
    with pytest.raises(TypeError):
        cleave.linear(plan, A, B, C.half())
    for bad in (dict(act_grad="relu"), dict(act_grad="relu", preact=z, bias=torch.zeros(8, device="cuda"))):
        with pytest.raises(cleave.CleaveError):
            cleave.linear(plan, A, B, C, **bad)
    q, qb = torch.zeros(4, 16, device="cuda").to(E4M3), torch.zeros(8, 16, device="cuda").to(E4M3)
    s = dict(scale_a=torch.ones(4, device="cuda"), scale_b=torch.ones(8, device="cuda"))
    plan8 = cleave.plan_linear(4, 8, 16, E4M3)
    with pytest.raises(ValueError):
        cleave.linear(plan8, q, qb, C, transB=1)                       # no scales
    with pytest.raises(cleave.CleaveError):
        cleave.linear(plan, q, qb, C, transB=1, **s)                   # another type's plan
    with pytest.raises((cleave.CleaveError, ValueError)):
        cleave.linear(plan8, A, B, C)
    with pytest.raises(cleave.CleaveError):                            # rows that do not start on sixteen bytes
        cleave.linear(plan8, torch.zeros(4, 24, device="cuda").to(E4M3)[:, :16], qb, C, transB=1, **s)
    with pytest.raises(cleave.CleaveError):
        cleave.plan_linear(4, 8, 24, E4M3)
    with pytest.raises(TypeError):
        cleave.plan_linear(4, 8, 16, torch.float16)
    split = cleave.plan_uniform(4, 8, 16, 4, 8, 2)
    with pytest.raises((ValueError, TypeError)):
        cleave.linear(split, A, B, C)                                  # no partials
    with pytest.raises(cleave.CleaveError):                            # a plan of 8-bit operands is no other call's
        cleave.execute(plan8, torch.zeros(4, 8, device="cuda", dtype=BF16), torch.zeros(8, 8, device="cuda", dtype=BF16),
                       torch.empty(plan8.partial_elems, device="cuda"))


@pytest.mark.parametrize("size", [(1, 1001, 333), (2, 1067, 674), (16, 130, 4099), (5, 3, 70), (4, 2, 1), (7, 65, 31)])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("transB", [0, 1])
@pytest.mark.parametrize("epilogue", [0, 1, 2])
def test_few_rows_of_any_length(size, dtype, transB, epilogue):
    assert check(*size, dtype=dtype, transB=transB, **EPILOGUES[epilogue])[2] == "linear_few_rows"
    check(*size, dtype=dtype, transB=transB, pad=3, shift=1, **EPILOGUES[epilogue])


@pytest.mark.parametrize("size,splits", [((3, 67, 1000), 3), ((16, 33, 515), 4), ((1, 5, 130), 2)])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("transB", [0, 1])
def test_few_rows_split_at_any_length(size, splits, dtype, transB):
    plan = cleave.plan_uniform(*size, 64, 64, splits)
    check(*size, dtype=dtype, transB=transB, plan=plan, **EPILOGUES[1])
