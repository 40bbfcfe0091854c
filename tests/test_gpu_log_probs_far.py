"""The gradient of the logits in rows whose log of the sum of exponentials lies far from zero (masked by a finite value, offset, cold),
where fp32 holds little or nothing of the sum beside the largest logit: against fp64 of the logits, not of the rounded sum."""
import math

import pytest
import torch

import paper_2512_22142_amd as cleave

pytestmark = pytest.mark.gpu

F32, BF16, I64 = torch.float32, torch.bfloat16, torch.int64
U32, U16 = 2.0 ** -24, 2.0 ** -8   # unit roundoffs: 24 and 8 bits of significand
INF = math.inf


def matrix(rows, cols, dtype, seed, pad=0, shift=0, std=2.5):
    g = torch.Generator(device="cuda").manual_seed(seed)
    flat = torch.full((rows * (cols + pad) + shift + 70,), 7.0, device="cuda").to(dtype)
    view = flat[shift: shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    if std:
        view.copy_((torch.randn(rows, cols, generator=g, device="cuda") * std).to(dtype))
    return view, flat


def vector(rows, seed, std=2.5):
    return torch.randn(rows, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda") * std


def exact(logits, scale):
    """(p, log p, entropy, d) in fp64, d the distance from the row's largest; differences first, so that offsets leave no trace."""
    x = logits.double()
    d = (x - x.amax(dim=1, keepdim=True)) * scale
    logp = d - d.exp().sum(dim=1, keepdim=True).log()
    p = logp.exp()
    return p, logp, torch.special.entr(p).sum(dim=1), d


def check(change, rows, cols, dtype, scale=1.0, pad=0, shift=0, in_place=False, dent=True):
    logits = matrix(rows, cols, dtype, 1, pad, shift)[0]
    ids = torch.randint(0, cols, (rows,), generator=torch.Generator(device="cuda").manual_seed(2), device="cuda")
    change(logits)
    scale = float(torch.tensor(scale))
    p, logp, h, far = exact(logits, scale)
    d, dh = vector(rows, 3), vector(rows, 4)
    got_logp, lse, ent = (torch.empty(rows, device="cuda") for _ in range(3))
    cleave.log_probs(logits, ids, got_logp, lse=lse, entropy=ent, scale=scale,
                     workspace=torch.empty(cleave.log_probs_workspace(rows, cols), device="cuda"))
    assert lse.abs().min() >= 1000
    out, whole = (logits, None) if in_place else matrix(rows, cols, dtype, 0, pad, shift, None)
    kw = dict(entropy=ent, dentropy=dh) if dent else {}
    cleave.log_probs_backward(logits, lse, out, ids=ids, dlogp=d, scale=scale, **kw)
    # the sum of n exponentials of rounded differences; log p from it; p from an argument rounded twice and the exponential
    n_err = (cols / 256 + 32) * U32
    left = p > 0
    far = torch.where(left, far.abs(), torch.zeros_like(far))
    t = torch.where(left, logp, torch.zeros_like(logp))
    s_err = n_err + 5 * U32 * (p * far).sum(dim=1)
    t_err = s_err[:, None] + 4 * U32 * far + 2 * U32 * t.abs()
    p_err = t_err + U32 * (4 * t.abs() + 4)
    h_err = s_err + (p * far).sum(dim=1) * 2 * n_err + 8 * U32 * (p * far * far).sum(dim=1) + 2 * U32 * h
    dd, eh, hh = d.double()[:, None], dh.double()[:, None] if dent else 0.0, h[:, None]
    hot = torch.zeros_like(p).scatter_(1, ids[:, None], 1.0)
    want = scale * (dd * (hot - p) - eh * p * (t + hh))
    size = dd.abs() + abs(eh) * (t + hh).abs()
    err = p * (size * p_err + abs(eh) * (t_err + h_err[:, None] + 2 * U32 * (t.abs() + hh))) + 4 * U32 * (p * size + hot * dd.abs())
    half = U16 if dtype == BF16 else U32
    bad = (out.double() - want).abs() - scale * err - half * 1.01 * (want.abs() + scale * err) - 2.0 ** -126 * max(scale, 1.0)
    assert bad.max() <= 0, (float(bad.max()), float(out.double().sum(dim=1).abs().max()))
    if whole is not None:
        out.fill_(7)
        assert torch.all(whole.float() == 7)


def filled(value):
    return lambda logits: logits.fill_(value)


def partly(value):
    """Masked by `value` in the first row, the others' logits near it; some masked by minus infinity."""
    def change(logits):
        logits.add_(value)
        logits[0] = value
        logits[:, ::5] = -INF
        logits[:, 1] = value
    return change


def offset(value):
    return lambda logits: logits.add_(value)


# a wave's row, a workgroup's, several workgroups' parts, whole and ragged
SIZES = [(3, 1), (5, 40), (3, 1000), (1100, 300), (3, 2048), (2, 2049), (3, 5000), (3, 8192), (2, 9001), (2, 32000), (2, 131073)]


@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rows_masked_by_a_finite_value(rows, cols, dtype):
    for value in (-1e4, -1e7, -1e8, -1e9, -1e20):
        check(filled(value), rows, cols, dtype)
    if cols > 1:
        check(partly(-1e4), rows, cols, dtype)
        check(partly(-1e9), rows, cols, dtype, in_place=True)


@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_offsets_and_low_temperatures(rows, cols, dtype):
    for value in (2e3, -2e3, 1e5, -1e5, 1e7, -1e7):
        check(offset(value), rows, cols, dtype)
    check(offset(1e5), rows, cols, dtype, dent=False)
    check(offset(1.0), rows, cols, dtype, scale=1e6)
    check(offset(-1e5), rows, cols, dtype, scale=0.7, in_place=True)


@pytest.mark.parametrize("pad,shift", [(8, 0), (3, 0), (8, 1), (5, 7)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_strides_and_alignment(pad, shift, dtype):
    for cols in (1000, 5001, 20003):
        check(offset(1e4), 3, cols, dtype, pad=pad, shift=shift)
        check(offset(1e4), 3, cols, dtype, pad=pad, shift=shift, in_place=True)


@pytest.mark.parametrize("cols", [700, 5000, 20003])
def test_a_log_of_the_sum_that_fp32_cannot_hold(cols):
    """scale times the largest logit overflows, the differences do not."""
    def change(logits):
        logits.mul_(1e36)

    check(change, 4, cols, F32, scale=300.0)
    check(change, 4, cols, F32, scale=1e-36 * 2000)        # (and one that it holds)


@pytest.mark.parametrize("cols", [300, 20003])
def test_far_and_near_rows_side_by_side(cols):
    """Rows of one launch: near ones keep their bits whatever lies beside them."""
    x = matrix(9, cols, F32, 1)[0].contiguous()
    ids = torch.arange(9, device="cuda")
    d = vector(9, 3)
    mixed = x.clone()
    mixed[1::2] += 1e5
    out = []
    for t in (x, mixed):
        lse, dx = torch.empty(9, device="cuda"), torch.empty_like(x)
        cleave.log_probs(t, lse=lse)
        cleave.log_probs_backward(t, lse, dx, ids=ids, dlogp=d)
        out.append(dx)
    assert torch.equal(out[0][::2], out[1][::2])
    assert not torch.equal(out[0][1::2], out[1][1::2])
    # (a sum over a row is zero: n roundings of its elements and of their p)
    assert out[1].double().sum(dim=1).abs().max() <= float(d.abs().max()) * 2 * (cols / 256 + 64) * U32


def test_repeats_its_bits_in_a_graph():
    x = matrix(6, 20003, BF16, 1)[0].contiguous()
    x[::2] += 3e4
    x[1] = -1e9
    ids = torch.arange(6, device="cuda")
    lse, ent, dx, d = torch.empty(6, device="cuda"), torch.empty(6, device="cuda"), torch.empty_like(x), vector(6, 3)

    def step():
        cleave.log_probs(x, lse=lse, entropy=ent)
        cleave.log_probs_backward(x, lse, dx, ids=ids, dlogp=d, entropy=ent, dentropy=d)

    step()
    want = [t.clone() for t in (lse, ent, dx)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        for t in (lse, ent, dx):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, (lse, ent, dx)))
