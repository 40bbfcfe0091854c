"""Log probabilities of tokens, entropy, the most likely tokens and the gradient of the logits against fp64; what they refuse."""
import math

import pytest
import torch

import paper_2512_22142_amd as cleave

pytestmark = pytest.mark.gpu

F32, BF16, I64 = torch.float32, torch.bfloat16, torch.int64
U32, U16 = 2.0 ** -24, 2.0 ** -8   # unit roundoffs: 24 and 8 bits of significand
INF = math.inf
SPARE = 70

# one thread's groups, whole and ragged, strips of one group to many, rows for wide and narrow workgroups, rows in parts
SIZES = [(1, 1), (3, 2), (2, 7), (5, 33), (4, 511), (3, 1000), (2, 8192), (1, 32000), (7, 50257), (3, 131072), (1, 262143), (64, 131073),
         (65, 140000), (1100, 257), (1030, 32000), (1500, 3001)]


def matrix(rows, cols, dtype, seed, pad=0, shift=0, std=2.5):
    """A rows x cols view, `shift` elements into a buffer of sevens with a leading dimension of cols + pad, and the buffer."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    flat = torch.full((rows * (cols + pad) + shift + SPARE,), 7.0, device="cuda").to(dtype)
    view = flat[shift: shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    if std is not None:
        view.copy_((torch.randn(rows, cols, generator=g, device="cuda") * std).to(dtype))
    return view, flat


def flat_of(n, dtype=F32):
    flat = torch.full((n + SPARE,), 7, dtype=dtype, device="cuda")
    return flat[:n], flat


def tokens(rows, cols, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(0, cols, (rows,), generator=g, device="cuda")


def exact(logits, scale):
    """(p, log p, lse, entropy) of the rows in fp64; rows without a token left have p 0."""
    l = logits.double() * scale
    lse = torch.logsumexp(l, dim=1)
    none = lse == -INF
    logp = torch.where(none[:, None], torch.full_like(l, -INF), l - torch.where(none, torch.zeros_like(lse), lse)[:, None])
    p = logp.exp()
    return p, logp, lse, torch.special.entr(p).sum(dim=1)


def order(logits, k):
    return torch.sort(logits.float(), dim=1, descending=True, stable=True)[1][:, :k]


def check(rows, cols, dtype, top, scale=1.0, pad=0, shift=0, change=None, seed=1, entropy=True):
    logits = matrix(rows, cols, dtype, seed, pad, shift)[0]
    ids = tokens(rows, cols, seed + 1)
    if change:
        change(logits, ids)
    (logp, logp_w), (lse, lse_w), (ent, ent_w) = flat_of(rows), flat_of(rows), flat_of(rows)
    kw, top_whole = {}, None
    if top:
        (top_ids, top_ids_w), (top_logp, top_logp_w) = flat_of(rows * top, I64), flat_of(rows * top)
        top_ids, top_logp = top_ids.view(rows, top), top_logp.view(rows, top)
        kw = dict(top_ids=top_ids, top_logp=top_logp)
    ws = torch.full((cleave.log_probs_workspace(rows, cols, top),), float("nan"), device="cuda")
    cleave.log_probs(logits, ids, logp, lse=lse, entropy=ent if entropy else None, scale=scale, workspace=ws, **kw)
    p, want, want_lse, want_ent = exact(logits, scale)
    a = logits.double() * scale
    most = a.amax(dim=1)
    far = torch.where(p > 0, (a - most[:, None]).abs(), torch.zeros_like(a))     # |d|
    n_err = (cols / 256 + 32) * U32                      # a sum of n terms, the exponential's own roundings
    s_err = n_err + 5 * U32 * (p * far).sum(dim=1)       # roundings of d, relative to d
    fine = want_lse != -INF                              # something is left
    given = (ids >= 0) & fine

    def near(got, want, err, what):
        bad = (got.double() - want).abs() - err - 2 * U32 * want.abs()
        assert bad.numel() == 0 or bad.max() <= 0, (what, float(bad.max()))

    near(lse[fine], want_lse[fine], (s_err + 3 * U32 * most.abs())[fine], "lse")
    if entropy:
        ent_err = s_err + (p * far).sum(dim=1) * 2 * n_err + 8 * U32 * (p * far * far).sum(dim=1)
        near(ent[fine], want_ent[fine], ent_err[fine], "entropy")
    at = ids.clamp_min(0)[:, None]
    own = want.gather(1, at)[:, 0]
    own_far = torch.where(own > -INF, (a.gather(1, at)[:, 0] - most).abs(), torch.zeros_like(own))
    seen = given & (own > -INF)
    near(logp[seen], own[seen], (s_err + 4 * U32 * own_far)[seen], "logp")
    assert torch.all(logp[ids < 0] == 0) and torch.all(logp[given & (own == -INF)] == -INF)
    assert torch.all(lse[~fine] == -INF) and torch.all(logp[~fine & (ids >= 0)] == -INF)
    if entropy:
        assert torch.all(ent[~fine] == 0) and torch.all(ent[fine] >= 0)
        assert torch.all(ent_w[rows:] == 7)
    if top:
        first = order(logits, top)
        assert torch.equal(top_ids, first), "top ids"
        t = want.gather(1, first)
        left = t > -INF
        t_far = torch.where(left, (a.gather(1, first) - most[:, None]).abs(), torch.zeros_like(t))
        near(top_logp[left], t[left], (s_err[:, None] + 4 * U32 * t_far)[left], "top log probabilities")
        assert torch.all(top_logp[~left] == -INF)
        assert torch.all(top_ids_w[rows * top:] == 7) and torch.all(top_logp_w[rows * top:] == 7)
    assert torch.all(logp_w[rows:] == 7) and torch.all(lse_w[rows:] == 7)
    return logp, lse, ent


@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("top", [0, 1, 20, 32])
def test_log_probs(rows, cols, dtype, top):
    check(rows, cols, dtype, min(top, cols), scale=1.0 if top != 1 else 0.7, entropy=top != 20)


@pytest.mark.parametrize("rows,cols", [(3000, 1), (1100, 7), (2001, 64), (1500, 255), (1026, 256), (1030, 257), (1500, 512), (1100, 513),
                                       (1025, 777), (1111, 1024), (1100, 1025)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_many_short_rows(rows, cols, dtype):
    check(rows, cols, dtype, 0)
    check(rows, cols, dtype, min(8, cols), shift=1)
    check(rows, cols, dtype, min(32, cols), pad=3)
    check(rows, cols, dtype, 1, entropy=False)


@pytest.mark.parametrize("pad,shift", [(8, 0), (3, 0), (8, 1), (0, 4), (5, 7)])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,cols", [(9, 1000), (3, 131100), (1200, 300)])
def test_strides_and_alignment(pad, shift, dtype, rows, cols):
    check(rows, cols, dtype, 7, pad=pad, shift=shift)


@pytest.mark.parametrize("rows,cols", [(40, 50257), (1100, 4099), (3, 9001), (2, 100001)])
@pytest.mark.parametrize("shift", [0, 1])
def test_rows_that_begin_within_a_word(rows, cols, shift):
    check(rows, cols, BF16, 5, shift=shift)
    check(rows, cols, BF16, 0, shift=shift)


def masks(kind):
    def change(logits, ids):
        rows, cols = logits.shape
        g = torch.Generator(device="cuda").manual_seed(9)
        if kind == "most":
            logits.masked_fill_(torch.rand(rows, cols, generator=g, device="cuda") < 0.97, -INF)
        elif kind == "one left":
            keep = logits.gather(1, ids[:, None]).clone()
            logits.fill_(-INF)
            logits.scatter_(1, ids[:, None], keep)
        elif kind == "nothing left":
            logits[::2] = -INF
        elif kind == "lowest value":
            logits.masked_fill_(torch.rand(rows, cols, generator=g, device="cuda") < 0.5, torch.finfo(logits.dtype).min)
        elif kind == "a long run":         # a thread's whole strip, and its neighbours'
            logits[:, : cols // 2] = -INF
        elif kind == "no token":
            ids[::2] = -1
            ids[1::3] = -100
    return change


@pytest.mark.parametrize("kind", ["most", "one left", "nothing left", "lowest value", "a long run", "no token"])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,cols", [(5, 40), (4, 5000), (3, 140000), (1100, 700)])
def test_masks(kind, dtype, rows, cols):
    check(rows, cols, dtype, 20, change=masks(kind))


def test_a_row_of_the_lowest_value_is_even():
    for dtype in (F32, BF16):
        logits = torch.full((2, 1000), torch.finfo(dtype).min, dtype=dtype, device="cuda")
        logp, ent = torch.empty(2, device="cuda"), torch.empty(2, device="cuda")
        cleave.log_probs(logits, torch.zeros(2, dtype=I64, device="cuda"), logp, entropy=ent)
        for t, want in ((logp, -math.log(1000)), (ent, math.log(1000))):
            assert (t - want).abs().max() <= 64 * U32 * 7


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,cols", [(3, 100), (2, 9000), (2, 70000), (2, 262144), (1100, 2000)])
def test_ties_go_to_the_lower_id(dtype, rows, cols):
    def equal(logits, ids):
        logits.fill_(1.5)

    def steps(logits, ids):
        logits.copy_((torch.arange(cols, device="cuda") % 5).to(dtype).expand(rows, cols))

    def zeros(logits, ids):               # of both signs
        logits.fill_(-1.0)
        logits[:, 3::7] = 0.0
        logits[:, 1::7] = -0.0

    def one_strip(logits, ids):           # the largest ones in the strips of a few threads
        logits.fill_(-5.0)
        v = torch.arange(cols, device="cuda")
        near = (v // 8) % 64 == 5
        logits[:, near] = (v[near] % 97).to(dtype) / 64

    def rising(logits, ids):
        logits.copy_((torch.arange(cols, device="cuda").float() / cols * 8).to(dtype).expand(rows, cols))

    def falling(logits, ids):
        logits.copy_((-torch.arange(cols, device="cuda").float() / cols * 8).to(dtype).expand(rows, cols))

    for change in (equal, steps, zeros, one_strip, rising, falling):
        check(rows, cols, dtype, 32, change=change)
        check(rows, cols, dtype, 3, change=change)


def test_large_logits_and_temperatures():
    def large(logits, ids):
        logits.mul_(1000)

    for scale in (1.0, 1e-3, 40.0):
        check(5, 3000, F32, 5, scale=scale)
        check(5, 3000, F32, 5, scale=scale, change=large)


@pytest.mark.parametrize("cols", [50, 3000, 140000])
@pytest.mark.parametrize("top", [0, 4])
def test_rows_that_are_not_finite_and_tokens_beyond_the_row(cols, top):
    logits = matrix(5, cols, F32, 1)[0].clone()
    logits[1, cols // 2], logits[2, 3] = float("nan"), INF
    logits[3, 5] = float("nan")
    logits[3, 7] = -INF
    ids = torch.tensor([0, 1, 2, 3, cols], device="cuda")
    logp, lse, ent = (torch.empty(5, device="cuda") for _ in range(3))
    kw = dict(top_ids=torch.empty(5, top, dtype=I64, device="cuda"), top_logp=torch.empty(5, top, device="cuda")) if top else {}
    cleave.log_probs(logits, ids, logp, lse=lse, entropy=ent, workspace=torch.empty(cleave.log_probs_workspace(5, cols, top),
                                                                                    device="cuda"), **kw)
    for k in (1, 2, 3):
        assert logp[k].isnan() and lse[k].isnan() and ent[k].isnan()
        if top:
            assert torch.all(kw["top_logp"][k].isnan())
    assert logp[0].isfinite() and lse[4].isfinite() and logp[4].isnan()
    if top:      # a NaN's place is minus infinity's
        assert torch.equal(kw["top_ids"], order(torch.where(logits.isnan(), torch.full_like(logits, -INF), logits), top))


def test_parts_left_out():
    logits, ids = matrix(3, 999, BF16, 1)[0], tokens(3, 999, 2)
    logp, lse, ent = check(3, 999, BF16, 5)
    ids = tokens(3, 999, 2)
    a, b, c = (torch.empty(3, device="cuda") for _ in range(3))
    cleave.log_probs(logits, ids, a)
    cleave.log_probs(logits, lse=b)
    cleave.log_probs(logits, entropy=c)
    t, tl = torch.empty(3, 5, dtype=I64, device="cuda"), torch.empty(3, 5, device="cuda")
    cleave.log_probs(logits, top_ids=t, top_logp=tl)
    assert torch.equal(t, order(logits, 5)) and torch.equal(a, logp) and torch.equal(b, lse) and torch.equal(c, ent)


def check_backward(rows, cols, dtype, scale=1.0, pad=0, shift=0, change=None, dlogp=True, dent=True, in_place=False):
    logits = matrix(rows, cols, dtype, 1, pad, shift)[0]
    ids = tokens(rows, cols, 2)
    if change:
        change(logits, ids)
    p, logp, lse64, h64 = exact(logits, scale)
    lse, h = lse64.float(), h64.float()
    d, dh = matrix(1, rows, F32, 3)[0][0].contiguous(), matrix(1, rows, F32, 4)[0][0].contiguous()
    out, whole = matrix(rows, cols, dtype, 0, pad, shift, None)
    if in_place:
        out = logits
    kw = dict(ids=ids, dlogp=d) if dlogp else {}
    if dent:
        kw.update(entropy=h, dentropy=dh)
    a = logits.double() * scale
    cleave.log_probs_backward(logits, lse, out, scale=scale, **kw)
    fine = (lse64 != -INF)[:, None]
    # with the given lse
    t = torch.where(fine, a - lse.double()[:, None].clamp_min(-1e300), torch.full_like(a, -INF))
    p = t.exp()
    seen = p > 0
    t0 = torch.where(seen, t, torch.zeros_like(t))
    dd = torch.where(ids >= 0, d.double(), torch.zeros_like(h64))[:, None] if dlogp else torch.zeros_like(h64)[:, None]
    hh, eh = (h.double()[:, None], dh.double()[:, None]) if dent else (0.0, torch.zeros_like(h64)[:, None])
    factor = dd + eh * (t0 + hh)
    want = -p * factor
    if dlogp:
        hot = torch.zeros_like(a).scatter_(1, ids.clamp_min(0)[:, None], 1.0)
        want = want + torch.where(fine, hot * dd, torch.zeros_like(a))
    want = want * scale
    size = dd.abs() + eh.abs() * (t0.abs() + (hh if dent else 0.0))
    # p: an argument of |t| rounded twice, and the exponential; the factor's and the product's roundings
    err = scale * (p * size * U32 * (4 * t0.abs() + 12) + (hot * dd.abs() * 2 * U32 if dlogp else 0.0)) + 2 * U32 * want.abs()
    half = U16 if dtype == BF16 else U32
    bad = (out.double() - want).abs() - (half * 1.01 * want.abs() + err + 2.0 ** -140)     # (what fp32 holds no more)
    assert bad.max() <= 0, float(bad.max())
    if not in_place:
        keep = out.clone()
        out.fill_(7)
        assert torch.all(whole.float() == 7)
        out.copy_(keep)
    return out


@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_backward(rows, cols, dtype):
    check_backward(rows, cols, dtype)
    if cols < 100000:
        check_backward(rows, cols, dtype, dent=False, scale=0.7)
        check_backward(rows, cols, dtype, dlogp=False)
        check_backward(rows, cols, dtype, in_place=True)


@pytest.mark.parametrize("pad,shift", [(8, 0), (3, 0), (8, 1), (5, 7)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_backward_strides_and_alignment(pad, shift, dtype):
    check_backward(9, 1000, dtype, pad=pad, shift=shift)
    check_backward(9, 1000, dtype, pad=pad, shift=shift, in_place=True)


@pytest.mark.parametrize("kind", ["most", "one left", "nothing left", "a long run", "no token"])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_backward_of_masks(kind, dtype):
    for rows, cols in ((5, 40), (4, 5000), (1100, 700)):
        logits = matrix(rows, cols, dtype, 1)[0]
        masks(kind)(logits, tokens(rows, cols, 2))
        out = check_backward(rows, cols, dtype, change=masks(kind))
        gone = (logits == -INF).clone()
        hot = torch.zeros_like(gone)
        ids = tokens(rows, cols, 2)
        masks(kind)(logits.clone(), ids)
        hot.scatter_(1, ids.clamp_min(0)[:, None], True)
        assert torch.all(out[gone & ~hot] == 0)


def test_backward_of_rows_without_a_token_left_and_of_tokens_beyond_the_row():
    for dtype in (F32, BF16):
        x = matrix(4, 1000, dtype, 1)[0].clone()
        x[0], x[1] = -INF, torch.finfo(dtype).min
        ids = torch.tensor([3, 4, 1000, -5], device="cuda")
        logp, lse, ent = (torch.empty(4, device="cuda") for _ in range(3))
        cleave.log_probs(x, ids, logp, lse=lse, entropy=ent)
        d = torch.ones(4, device="cuda")
        dx = torch.empty_like(x)
        cleave.log_probs_backward(x, lse, dx, ids=ids, dlogp=d, entropy=ent, dentropy=d)
        assert torch.all(dx[:2] == 0) and torch.all(dx[2].isnan()) and torch.all(dx[3].isfinite()) and torch.any(dx[3] != 0)
        cleave.log_probs_backward(x, lse, dx, ids=ids, dlogp=d)
        assert torch.all(dx[3] == 0)


@pytest.mark.parametrize("mask", [-INF, -3e38])
def test_masked_tokens_have_no_gradient_however_large_the_given_one(mask):
    x = matrix(3, 1000, BF16, 1)[0].clone()
    x[:, 100:900] = mask
    ids = torch.tensor([3, 950, -1], device="cuda")
    logp, lse, ent = (torch.empty(3, device="cuda") for _ in range(3))
    cleave.log_probs(x, ids, logp, lse=lse, entropy=ent)
    d = torch.full((3,), 1e20, device="cuda")
    dx = torch.empty_like(x)
    cleave.log_probs_backward(x, lse, dx, ids=ids, dlogp=d, entropy=ent, dentropy=d)
    assert torch.all(dx[:, 100:900] == 0) and torch.all(dx.isfinite())


def test_backward_against_differences_of_the_kernel():
    rows, cols, step = 3, 50, 1.0 / 64
    x, u = matrix(rows, cols, F32, 1)[0].contiguous(), matrix(rows, cols, F32, 2, std=1.0)[0].contiguous()
    ids = tokens(rows, cols, 3)
    a, b = matrix(1, rows, F32, 4)[0][0].contiguous(), matrix(1, rows, F32, 5)[0][0].contiguous()
    for scale in (1.0, 0.6):
        logp, lse, ent = (torch.empty(rows, device="cuda") for _ in range(3))

        def loss(t):
            cleave.log_probs(t, ids, logp, lse=lse, entropy=ent, scale=scale)
            return float((a.double() * logp.double() + b.double() * ent.double()).sum())

        up, down = loss(x + step * u), loss(x - step * u)
        loss(x)
        dx = torch.empty_like(x)
        cleave.log_probs_backward(x, lse, dx, ids=ids, dlogp=a, entropy=ent, dentropy=b, scale=scale)
        along = (up - down) / (2 * step)
        # third order: step^2 / 6 of third derivatives along u, below 30 (|a| + |b|) max|u|^3; rounding 1e-5 / step
        most = float(((a.abs() + b.abs()) * u.abs().amax(dim=1) ** 3).sum())
        assert abs(along - float((dx.double() * u.double()).sum())) <= step ** 2 * 5 * most + 1e-3


def test_no_rows_and_more_rows_than_one_launch_takes():
    none, ids = torch.empty(0, 40, device="cuda"), torch.empty(0, dtype=I64, device="cuda")
    cleave.log_probs(none, ids, none[:, 0].contiguous(), workspace=torch.empty(0, device="cuda"))
    cleave.log_probs_backward(none, none[:, 0].contiguous(), torch.empty_like(none), ids=ids, dlogp=none[:, 0].contiguous())
    check(2 ** 21 + 77, 3, BF16, 2)
    check_backward(2 ** 21 + 77, 3, BF16)


def test_offsets_beyond_32_bits():
    """Rows that lie 2^27 elements apart: the last begins beyond 2^32 bytes."""
    rows, cols, ld = 18, 1000, 2 ** 27
    flat = torch.empty((rows - 1) * ld + cols, dtype=BF16, device="cuda")
    far = flat.as_strided((rows, cols), (ld, 1))
    x, ids = matrix(rows, cols, BF16, 1)[0].contiguous(), tokens(rows, cols, 2)
    far.copy_(x)
    out = []
    for t in (x, far):
        logp, lse, top, tl = (torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"),
                              torch.empty(rows, 5, dtype=I64, device="cuda"), torch.empty(rows, 5, device="cuda"))
        cleave.log_probs(t, ids, logp, lse=lse, top_ids=top, top_logp=tl)
        cleave.log_probs_backward(t, lse, t, ids=ids, dlogp=logp)
        out.append((logp, lse, top, tl, t))
    assert all(torch.equal(a, b) for a, b in zip(*out))


def test_repeats_its_bits_on_another_stream_and_in_a_graph():
    x, ids = matrix(40, 32000, BF16, 1)[0], tokens(40, 32000, 2)
    long, one = matrix(2, 150000, BF16, 3)[0], tokens(2, 150000, 4)
    logp, lse, ent, d = (torch.empty(40, device="cuda") for _ in range(4))
    d.fill_(-1 / 40)
    dl = torch.empty(40, 32000, dtype=BF16, device="cuda")
    top, tl = torch.empty(2, 20, dtype=I64, device="cuda"), torch.empty(2, 20, device="cuda")
    logp2 = torch.empty(2, device="cuda")
    ws = torch.empty(cleave.log_probs_workspace(2, 150000, 20), device="cuda")
    assert ws.numel() > 0

    def step():
        cleave.log_probs(x, ids, logp, lse=lse, entropy=ent)
        cleave.log_probs_backward(x, lse, dl, ids=ids, dlogp=d, entropy=ent, dentropy=d)
        cleave.log_probs(long, one, logp2, top_ids=top, top_logp=tl, workspace=ws)

    outs = (logp, lse, ent, dl, top, tl, logp2)
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


def test_refusals():
    x, ids, r = torch.zeros(4, 64, device="cuda"), torch.zeros(4, dtype=I64, device="cuda"), torch.empty(4, device="cuda")
    t, tl = torch.empty(4, 5, dtype=I64, device="cuda"), torch.empty(4, 5, device="cuda")
    for kw in (dict(ids=ids), dict(logp=r), dict(ids=ids.int(), logp=r), dict(ids=ids[:3], logp=r), dict(ids=ids, logp=r[:3]),
               dict(ids=ids.cpu(), logp=r), dict(top_ids=t), dict(top_ids=t, top_logp=tl[:, :4].contiguous()),
               dict(top_ids=t[:3], top_logp=tl), dict(lse=r.double())):
        with pytest.raises(ValueError):
            cleave.log_probs(x, **kw)
    with pytest.raises(TypeError):
        cleave.log_probs(x.half(), ids, r)
    for kw in (dict(scale=0.0), dict(scale=-1.0), dict(scale=INF), dict(scale=float("nan")), dict(lse=r)):
        with pytest.raises(cleave.CleaveError):
            cleave.log_probs(x, ids, r, **kw)
    with pytest.raises(cleave.CleaveError):
        cleave.log_probs(x, top_ids=torch.empty(4, 33, dtype=I64, device="cuda"), top_logp=torch.empty(4, 33, device="cuda"))
    with pytest.raises(cleave.CleaveError):
        cleave.log_probs(x[:, :3], top_ids=t, top_logp=tl)
    with pytest.raises((ValueError, TypeError)):
        cleave.log_probs(torch.zeros(1, 200000, device="cuda"), ids[:1], r[:1])        # no workspace
    for args, kw in (((x, r, x.bfloat16()), dict(ids=ids, dlogp=r)), ((x, r[:3], x), dict(ids=ids, dlogp=r)), ((x, r, x), {}),
                     ((x, r, x), dict(ids=ids)), ((x, r, x), dict(entropy=r))):
        with pytest.raises(ValueError):
            cleave.log_probs_backward(*args, **kw)
    with pytest.raises(cleave.CleaveError):
        cleave.log_probs_backward(x, r, x, ids=ids, dlogp=r, scale=0.0)
