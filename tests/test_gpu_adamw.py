"""AdamW over many tensors: bit for bit what elementary fp32 operations give, near fp64, and its refusals."""
import numpy as np
import pytest
import torch

import paper_2512_22142_amd as cleave
from oracle import operators as oo

pytestmark = pytest.mark.gpu

F32, BF16, E4M3 = torch.float32, torch.bfloat16, torch.float8_e4m3fn
HYPER = dict(lr=1e-3, beta1=0.9, beta2=0.95, eps=1e-8, weight_decay=0.1)


def root(x):
    """Correctly rounded (torch's own on the CPU is an ulp off now and then)."""
    return torch.from_numpy(np.sqrt(x.numpy()))


def to_blocks(x, up):
    """e4m3 values and scales of a CPU tensor, in elementary fp32 operations."""
    n, blocks = x.numel(), -(-x.numel() // 256)
    b = torch.zeros(blocks * 256)
    b[:n] = x
    b = b.view(blocks, 256)
    most = torch.where(b.isfinite(), b.abs(), torch.zeros_like(b)).amax(dim=1)
    scale = torch.where(most >= 2.0 ** -100, most * torch.tensor(1 / 448), torch.zeros_like(most))
    q = torch.where(scale[:, None] > 0, b * (1 / scale)[:, None], torch.zeros_like(b))
    if up:
        q = torch.where((b > 0) & (scale[:, None] > 0), q.clamp_min(2.0 ** -9), q)
    q = torch.where(b.isfinite(), q, torch.full_like(q, float("nan")))
    return q.view(-1)[:n].to(E4M3), scale


def from_blocks(q, scale):
    return q.float() * scale.repeat_interleave(256)[: q.numel()]


class Tensors:
    """The same tensors on the CPU and, as views `shift` elements into one buffer each, on the GPU."""

    def __init__(self, sizes, grad, states, seed=0, shift=0, copy=True):
        g = torch.Generator().manual_seed(seed)
        rand = lambda n, std: torch.randn(n, generator=g) * std   # noqa: E731
        self.states = states
        self.w = [rand(n, 0.02) for n in sizes]
        self.g = [rand(n, 1e-3).to(grad) for n in sizes]
        m, v = [rand(n, 3e-4) for n in sizes], [rand(n, 1e-3).square() * 0.5 for n in sizes]
        if states == 8:
            m, v = [to_blocks(x, False) for x in m], [to_blocks(root(x), True) for x in v]
            self.m, self.ms, self.v, self.vs = ([x[i] for x in p] for p in (m, v) for i in (0, 1))
        else:
            self.m, self.v, self.ms, self.vs = m, v, None, None
        self.copy = [torch.zeros(n, dtype=BF16) for n in sizes] if copy else None

        def gpu(list_):
            if list_ is None:
                return None
            out = []
            for t in list_:
                flat = torch.empty(t.numel() + shift, dtype=t.dtype, device="cuda")
                flat[shift:].copy_(t)
                out.append(flat[shift:])
            return out

        self.gpu = {k: gpu(getattr(self, k)) for k in ("w", "g", "m", "v", "ms", "vs", "copy")}

    def step_gpu(self, step, clip=None):
        d = self.gpu
        cleave.adamw(d["w"], d["g"], d["m"], d["v"], m_scales=d["ms"], v_scales=d["vs"], copies=d["copy"], step=step,
                     grad_scale=None if clip is None else torch.full((1,), clip, device="cuda"), **HYPER)

    def step_cpu(self, step, clip=1.0):
        b1, b2 = HYPER["beta1"], HYPER["beta2"]
        ib1, ib2 = 1 / (1 - b1 ** step), 1 / (1 - b2 ** step)
        for k in range(len(self.w)):
            if self.states == 8:
                m, r = from_blocks(self.m[k], self.ms[k]), from_blocks(self.v[k], self.vs[k])
                v = r * r
            else:
                m, v = self.m[k], self.v[k]
            g, w = self.g[k].float() * clip, self.w[k]
            m = b1 * m + (1 - b1) * g
            v = b2 * v + (1 - b2) * (g * g)
            self.w[k] = w - HYPER["lr"] * ((m * ib1) / (root(v * ib2) + HYPER["eps"]) + HYPER["weight_decay"] * w)
            if self.copy:
                self.copy[k] = self.w[k].to(BF16)
            if self.states == 8:
                m, self.ms[k] = to_blocks(m, False)
                v, self.vs[k] = to_blocks(root(v), True)
            self.m[k], self.v[k] = m, v

    def same(self):
        for name, list_ in self.gpu.items():
            for k, t in enumerate(list_ or []):
                a, b = t.cpu().float(), getattr(self, name)[k].float()
                assert torch.equal(a.view(torch.int32), b.view(torch.int32)) or torch.equal(a, b), (name, k)


SIZES = [1, 255, 256, 257, 0, 4095, 4096, 4097, 10000, 3, 65536]


@pytest.mark.parametrize("grad", [F32, BF16])
@pytest.mark.parametrize("states", [32, 8])
@pytest.mark.parametrize("shift", [0, 1, 2, 5])
def test_bits_of_elementary_operations(grad, states, shift):
    t = Tensors(SIZES, grad, states, shift=shift, copy=shift != 2)
    for step in (1, 2, 3):
        t.step_gpu(step, clip=0.75)
        t.step_cpu(step, clip=0.75)
        t.same()


@pytest.mark.parametrize("count", [0, 1, 55, 56, 57, 130])
def test_many_tensors(count):
    sizes = [(37 * k) % 700 + 1 for k in range(count)]
    t = Tensors(sizes, BF16, 8, seed=count)
    t.step_gpu(7)
    t.step_cpu(7)
    t.same()


@pytest.mark.parametrize("states", [32, 8])
def test_near_64_bits(states):
    t = Tensors([5000], F32, states, seed=3)
    d = lambda x: x.double().numpy()   # noqa: E731
    m, v = (from_blocks(t.m[0], t.ms[0]), from_blocks(t.v[0], t.vs[0]).double().square()) if states == 8 else (t.m[0], t.v[0])
    w, m, v = oo.adamw(d(t.w[0]), d(t.g[0]), d(m), d(v), step=9, grad_scale=0.5, **HYPER)
    t.step_gpu(9, clip=0.5)
    got = {k: x[0].double().cpu().numpy() for k, x in t.gpu.items() if x is not None}
    u = 2.0 ** -24
    # a dozen roundings of the update, two of the weight
    moved = np.abs(w - d(t.w[0]))
    assert np.all(np.abs(got["w"] - w) <= 2 * u * np.abs(w) + 20 * u * (moved + HYPER["lr"]))
    if states == 8:
        for name, x in (("m", m), ("v", np.sqrt(v))):
            scale = oo.block_scales(x)
            assert np.allclose(got[name + "s"], scale, rtol=16 * u, atol=0)
            x = x / np.repeat(scale, 256)[:5000]
            near = np.abs(x)
            # half a step of e4m3; what is above zero in the second state is at least its smallest value
            bound = np.maximum(near * 2.0 ** -4, 2.0 ** -9 if name == "v" else 2.0 ** -10) + near * 32 * u
            assert np.all(np.abs(got[name] - x) <= bound), name
    else:
        assert np.all(np.abs(got["m"] - m) <= 4 * u * (np.abs(m) + 1e-3)) and np.allclose(got["v"], v, rtol=8 * u, atol=1e-12)


def test_8_bit_states_from_nothing_and_blocks_that_fade():
    n = 700
    w, g = torch.ones(n, device="cuda"), torch.zeros(n, device="cuda")
    q = [torch.zeros(n, dtype=E4M3, device="cuda") for _ in range(2)]
    s = [torch.zeros(3, device="cuda") for _ in range(2)]
    hyper = dict(HYPER, weight_decay=0.0)
    cleave.adamw([w], [g], [q[0]], [q[1]], step=1, m_scales=[s[0]], v_scales=[s[1]], **hyper)
    assert torch.all(w == 1) and all(torch.all(x == 0) for x in s) and all(torch.all(x.float() == 0) for x in q)
    g[300:] = torch.linspace(1e-6, 1.0, 400, device="cuda")
    cleave.adamw([w], [g], [q[0]], [q[1]], step=1, m_scales=[s[0]], v_scales=[s[1]], **hyper)
    # the first step moves every weight with a gradient by lr against its sign
    assert torch.all(w[:300] == 1) and torch.allclose(w[300:], torch.full((400,), 1 - 1e-3, device="cuda"), rtol=0, atol=2e-5)
    assert s[0][0] == 0 and torch.all(s[0][1:] > 0)
    assert torch.all(q[1].float()[300:] > 0)      # never rounded to nothing
    g.fill_(1e-33)                                # both states of the first block end below 2^-100
    cleave.adamw([w], [g], [q[0]], [q[1]], step=2, m_scales=[s[0]], v_scales=[s[1]], **hyper)
    assert s[0][0] == 0 and s[1][0] == 0 and torch.all(w.isfinite())


@pytest.mark.parametrize("states", [32, 8])
def test_gradients_that_are_not_finite_stay_where_they_are(states):
    t = Tensors([600], F32, states, seed=4)
    t.gpu["g"][0][10] = float("nan")
    t.gpu["g"][0][20] = float("inf")
    t.gpu["g"][0][300] = -float("inf")
    t.step_gpu(5)
    t.g[0][[10, 20, 300]] = 0.0
    t.step_cpu(5)
    there = torch.ones(600, dtype=torch.bool)
    there[[10, 20, 300]] = False
    assert torch.equal(t.gpu["w"][0].cpu()[there], t.w[0][there])
    assert torch.equal(t.gpu["m"][0].cpu().float()[there], t.m[0].float()[there])
    assert not t.gpu["m"][0].cpu().float()[~there].isfinite().any() and t.gpu["w"][0].cpu()[10].isnan()


def test_beside_other_weights_nothing_is_written():
    for states in (32, 8):
        t = Tensors([300], BF16, states, shift=0)
        arrays = {name: list_ for name, list_ in t.gpu.items() if list_}
        for name, list_ in arrays.items():
            whole = torch.full((list_[0].numel() + 512,), 3.0, device="cuda").to(list_[0].dtype)
            whole[256:256 + list_[0].numel()] = list_[0]
            t.gpu[name] = [whole[256:256 + list_[0].numel()]]
            setattr(t, "whole_" + name, whole)
        t.step_gpu(2)
        for name, list_ in arrays.items():
            whole = getattr(t, "whole_" + name).float()
            assert torch.all(whole[:256] == 3) and torch.all(whole[256 + list_[0].numel():] == 3), name


def test_in_a_graph():
    t = Tensors([5000, 77], BF16, 8, seed=6)
    clip = torch.ones(1, device="cuda")
    d = t.gpu

    def step():
        cleave.adamw(d["w"], d["g"], d["m"], d["v"], m_scales=d["ms"], v_scales=d["vs"], copies=d["copy"], step=3,
                     grad_scale=clip, **HYPER)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        t.step_cpu(3)
        t.same()


def test_refusals():
    w, g = [torch.zeros(64, device="cuda")], [torch.zeros(64, device="cuda")]
    m, v = [torch.zeros(64, device="cuda")], [torch.zeros(64, device="cuda")]
    q, s = [torch.zeros(64, dtype=E4M3, device="cuda")], [torch.zeros(1, device="cuda")]
    ok = dict(HYPER, step=1)
    for bad in (dict(w=[w[0].bfloat16()]), dict(m=q), dict(grads=[g[0][:-1]]), dict(grads=g + g), dict(m=[m[0].cpu()]),
                dict(w=[torch.zeros(128, device="cuda")[::2]]), dict(m=q, v=q, m_scales=s),
                dict(m=q, v=q, m_scales=s, v_scales=[torch.zeros(2, device="cuda")]), dict(copies=[g[0]]),
                dict(grad_scale=torch.ones(2, device="cuda"))):
        with pytest.raises(ValueError):
            cleave.adamw(**{**dict(w=w, grads=g, m=m, v=v), **ok, **bad})
    with pytest.raises(TypeError):
        cleave.adamw(w, [g[0].half()], m, v, **ok)
    with pytest.raises(TypeError):
        cleave.adamw(w[0], None, m, v, **ok)
    for bad in (dict(step=0), dict(beta1=1.0), dict(beta2=-0.1), dict(eps=-1.0), dict(lr=float("nan"))):
        with pytest.raises(cleave.CleaveError):
            cleave.adamw(w, g, m, v, **dict(ok, **bad))
    assert torch.all(w[0] == 0)
