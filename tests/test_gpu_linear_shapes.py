"""Linear product: every kernel and shape that a plan's size leads to, by name, against fp64 over the whole output."""
import math

import pytest
import torch

import paper_2512_22142_amd as cleave

pytestmark = pytest.mark.gpu

F32, BF16, E4M3 = torch.float32, torch.bfloat16, torch.float8_e4m3fn
U32, U16 = 2.0 ** -24, 2.0 ** -8   # unit roundoffs: 24 and 8 bits of significand


def matrix(rows, cols, dtype, seed, pad=0, std=1.0):
    """A rows x cols view with a leading dimension of cols + pad in a buffer of sevens that is longer than it, and the buffer."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    flat = torch.full((rows * (cols + pad) + 64,), 7.0, device="cuda").to(dtype)
    view = flat[:rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    if std is not None:
        view.copy_((torch.randn(rows, cols, generator=g, device="cuda") * std).to(dtype))
    return view, flat


def act_of(z, name):
    if name == "silu":
        return z * torch.sigmoid(z)
    if name == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    return z


def slope_of(z, name):
    z = z.clone().requires_grad_()
    return torch.autograd.grad(act_of(z, name).sum(), z)[0]


def beside(whole, view):
    """Nothing is written beside the view."""
    keep = view.clone()
    view.fill_(7.0)
    assert torch.all(whole.float() == 7.0)
    view.copy_(keep)


def check(M, N, K, dtype, out, transB, act="none", grad=False, bias=False, residual=False, preact=False, pad=0, offset=0):
    std = 50.0 if dtype == E4M3 else 1.0
    ipad = 16 * pad if dtype == E4M3 else 0
    A, _ = matrix(M, K, dtype, 1, ipad, std)
    B, _ = matrix(*((N, K) if transB else (K, N)), dtype, 2, ipad, std / K ** 0.5)
    if offset:
        B = torch.cat([B.new_zeros(offset), B.flatten()])[offset:].view(B.shape)
    C, whole = matrix(M, N, out, 3, pad, None)
    b = matrix(1, N, F32, 4)[0][0] if bias else None
    r = matrix(M, N, out, 5, pad)[0] if residual else None
    z, z_whole = matrix(M, N, out, 6, pad, 2.0 if grad else None) if preact or grad else (None, None)
    sa, sb = ((matrix(1, n, F32, 7 + k)[0][0].abs() / 50 if dtype == E4M3 else None) for k, n in enumerate((M, N)))
    plan = cleave.plan_linear(M, N, K, dtype)
    ws = torch.full((max(1, plan.linear_workspace),), float("nan"), device="cuda")
    kw = dict(act_grad=act) if grad else dict(act=act)
    cleave.linear(plan, A, B, C, transB=transB, bias=b, residual=r, preact=z, scale_a=sa, scale_b=sb, partials=ws, **kw)
    a, w = A.float().double(), B.float().double()
    w = w.t().contiguous() if transB else w
    if dtype == E4M3:
        a, w = a * sa.double()[:, None], w * sb.double()
    sums = a @ w
    # K products summed in fp32: an eleven-sigma bound of a random walk; the scales' two products beside it
    err = 8 * U32 * torch.outer(a.norm(dim=1), w.norm(dim=0)) + 2 * U32 * sums.abs()
    u = U16 if out == BF16 else U32
    if grad:
        want = sums * slope_of(z.double(), act)
        err = err * 1.2 + sums.abs() * 64 * U32
    else:
        zz = sums + b.double() if bias else sums
        err = err + 2 * U32 * zz.abs()
        if preact:
            assert torch.all((z.double() - zz).abs() <= u * 1.01 * zz.abs() + err), plan.last_kernel
            beside(z_whole, z)
        want = act_of(zz, act)
        err = err * 1.2 + 32 * U32 * (1 + zz.abs())
    if residual:
        want = want + r.double()
    bad = (C.double() - want).abs() - (u * 1.01 * want.abs() + err + 2 * U32 * want.abs())
    assert bad.max() <= 0, (plan.last_kernel, float(bad.max()), int(bad.argmax()))
    beside(whole, C)
    return plan.last_kernel


EPILOGUES = [dict(bias=True, act="gelu_tanh", preact=True), dict(bias=True, act="silu", residual=True, pad=8),
             dict(grad=True, act="gelu_tanh", residual=True, pad=3), dict(grad=True, act="silu")]

# 512 and 768 tiles of 256 x 256, two and three to a workgroup; the same with clipped ones, chunks that end within a step
LARGE = [(8192, 4096, 192), (8192, 6144, 128), (8100, 4090, 200), (8192, 4096, 72)]
# more than 512 tiles of 128 x 128, several to a workgroup
SMALL = [(4352, 4352, 192), (4300, 4350, 200)]
DEEP = [(1920, 1920, 512), (1900, 1910, 200)]       # 225 of them, one to a CU
PARTS = [(300, 520, 256), (100, 261, 136)]          # 64 x 64


@pytest.mark.parametrize("epilogue", range(len(EPILOGUES)))
@pytest.mark.parametrize("out", [BF16, F32])
@pytest.mark.parametrize("shape,size", [(s, x) for s, xs in (("256x256", LARGE), ("128x128", SMALL), ("128x128_deep", DEEP),
                                                             ("64x64", PARTS)) for x in xs])
def test_bf16(shape, size, out, epilogue):
    assert check(*size, BF16, out, 1, **EPILOGUES[epilogue]) == "linear_direct_bf16_%s_nt" % shape
    if size[1] % 8 == 0:
        assert check(*size, BF16, out, 0, **EPILOGUES[epilogue]) == "linear_direct_bf16_%s_nn" % shape


@pytest.mark.parametrize("epilogue", range(len(EPILOGUES)))
@pytest.mark.parametrize("out", [BF16, F32])
@pytest.mark.parametrize("shape,size", [(s, x) for s, xs in (("128x128", SMALL), ("128x128_deep", DEEP), ("64x64", PARTS))
                                        for x in xs])
def test_e4m3(shape, size, out, epilogue):
    M, N, K = size
    for k in (2 * K, 2 * K + 16):      # whole steps of 128 values, and a last one that is none
        assert check(M, N, k, E4M3, out, 1, **EPILOGUES[epilogue]) == "linear_direct_e4m3_%s_nt" % shape


@pytest.mark.parametrize("epilogue", range(len(EPILOGUES)))
@pytest.mark.parametrize("size,dtype,transB,offset,name", [
    ((3000, 2500, 136), BF16, 0, 0, "bf16_128x128_nn"), ((1100, 1003, 100), BF16, 0, 0, "bf16_64x64_nn"),
    ((1100, 1004, 96), BF16, 1, 3, "bf16_64x64_nt"), ((200, 100, 52), BF16, 0, 0, "bf16_64x64_nn"),
    ((4096, 4096, 100), F32, 1, 0, "f32_128x128_nt"), ((2000, 3001, 64), F32, 0, 0, "f32_64x64_nn"),
    ((500, 600, 100), F32, 0, 1, "f32_64x64_nn"), ((300, 5, 96), BF16, 0, 0, "bf16_element"), ((300, 200, 3), F32, 1, 0, "f32_element")])
def test_general(size, dtype, transB, offset, name, epilogue):
    assert check(*size, dtype, dtype, transB, offset=offset, **EPILOGUES[epilogue]) == "linear_" + name


@pytest.mark.parametrize("size,dtype,transB,names", [
    ((300, 512, 512), BF16, 0, ("linear_direct_bf16_64x64_nn", "execute_direct_bf16_64x64_nn")),
    ((3000, 2500, 136), BF16, 0, ("linear_bf16_128x128_nn", "execute_bf16_128x128_nn")),
    ((9, 512, 512), F32, 1, ("linear_few_rows", "linear_few_rows"))])
def test_names_of_products_with_and_without_an_epilogue(size, dtype, transB, names):
    """A product with nothing behind its sums is a plain execute."""
    assert check(*size, dtype, dtype, transB, bias=True) == names[0]
    assert check(*size, dtype, dtype, transB) == names[1]


# chunks of K, joined by a second kernel, of every type; one size that is not split
@pytest.mark.parametrize("epilogue", range(len(EPILOGUES)))
@pytest.mark.parametrize("size,dtype,chunks", [((64, 512, 8192), BF16, 4), ((200, 1000, 4096), BF16, 2), ((64, 512, 8192), E4M3, 4),
                                               ((600, 1024, 8192), E4M3, 0), ((64, 2048, 4096), F32, 4), ((65, 1003, 3001), F32, 4)])
def test_split(size, dtype, chunks, epilogue):
    assert cleave.plan_linear(*size, dtype).linear_workspace == chunks * size[0] * size[1]
    check(*size, dtype, BF16 if dtype != F32 else F32, 1, **EPILOGUES[epilogue])
