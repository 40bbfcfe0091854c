"""Operators around the GEMMs of a training or serving step, as cases that are timed and compared.

Three operators and their gradients: the root-mean-square norm of a residual
stream, the matrix product with bias, activation and residual, and the AdamW
step over many tensors.  `run` is one pass through one of them: through the
package where `own` is true, else in plain torch operations in 32 bits.

Sizes come from this repository's configurations (layers of width 768, 4096 and
5120, an inner width of 11008) or are generic.  `work` counts every input once
and every output once.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "bf16": 2, "e4m3": 1}
E4M3 = torch.float8_e4m3fn
E4M3_MAX = 448.0
LEAST = 2.0 ** -100        # a row or block whose largest value is below is stored as zeros
STATE_BLOCK = 256          # elements that share a scale of an 8-bit optimizer state
EPS = 1e-5
ADAM = dict(lr=1e-4, beta1=0.9, beta2=0.95, eps=1e-8, weight_decay=0.1, step=100)
CLIP = 0.75


def listed():
    return [
        # One token of a serving batch: the norm in front of an 8-bit product. Latency.
        dict(name="norm_token_8bit", kind="norm", rows=1, cols=4096, dtype="bf16", residual=True, out="e4m3"),
        # A micro-batch through the benchmark layer's norm: residual added, the sum and 1 / rms kept for the backward pass.
        dict(name="norm_layer", kind="norm", rows=4096, cols=4096, dtype="bf16", residual=True, out="bf16"),
        # The widest layer's prompt pass, in front of an 8-bit product.
        dict(name="norm_prompt_8bit", kind="norm", rows=16384, cols=5120, dtype="bf16", residual=True, out="e4m3"),
        # Its gradient in training, joined with the residual stream's.
        dict(name="norm_backward", kind="norm_backward", rows=8192, cols=4096, dtype="bf16", residual=True),
        # Packed sequences, a width that is no multiple of a vector, fp32.
        dict(name="norm_backward_ragged", kind="norm_backward", rows=3001, cols=1001, dtype="f32", residual=False),
        # One token through an MLP's up projection: the weight is read once. Latency.
        dict(name="linear_token", kind="linear", T=1, fin=4096, fout=11008, dtype="bf16", out="bf16", act="silu",
             bias=True, residual=False, preact=False),
        # The same projection in training: the value in front of the activation is kept for the backward pass.
        dict(name="linear_layer", kind="linear", T=4096, fin=4096, fout=11008, dtype="bf16", out="bf16", act="gelu_tanh",
             bias=True, residual=False, preact=True),
        # A projection of packed sequences back into the residual stream, no size a multiple of a tile.
        dict(name="linear_ragged", kind="linear", T=3001, fin=1000, fout=2500, dtype="bf16", out="bf16", act="none",
             bias=True, residual=True, preact=False),
        # Backward through the down projection and the activation in front of it.
        dict(name="linear_backward", kind="linear_backward", T=4096, fin=11008, fout=4096, dtype="bf16", act="gelu_tanh"),
        # A prompt through an 8-bit projection, as the norm above leaves its rows.
        dict(name="linear_8bit", kind="linear_8bit", T=4096, fin=4096, fout=11008, out="bf16", act="none", bias=False,
             residual=False),
        # Every weight, bias and norm of a narrow layer, states in 32 bits.
        dict(name="adamw_narrow", kind="adamw", tensors="layer", h=768, F=2048, grad="bf16", states=32, copy=True),
        # The benchmark layer (202 million weights), states in 8 bits.
        dict(name="adamw_layer_8bit", kind="adamw", tensors="layer", h=4096, F=11008, grad="bf16", states=8, copy=True),
    ]


# ---- drawn cases -------------------------------------------------------------

def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi, step):
    return max(step, _log(rng, lo, hi) // step * step)


def _limit(case, names, cost, most):
    """Shrinks the largest of the named sizes until `cost` fits."""
    while cost(case) > most:
        big = max(names, key=lambda n: case[n])
        step = 64 if case[big] % 64 == 0 else 16 if case[big] % 16 == 0 else 1
        case[big] = max(step, int(case[big] * 0.8) // step * step)
    return case


def draw(rng):
    kind = rng.choice(["norm", "norm", "norm_backward", "linear", "linear", "linear_token", "linear_backward", "linear_8bit",
                       "adamw", "adamw"])
    step = rng.choice([1, 8, 64, 64])
    if kind == "norm":
        dtype = rng.choice(["bf16", "bf16", "f32"])
        c = dict(kind="norm", rows=_log(rng, 1, 32768), cols=_size(rng, 64, 16384, step), dtype=dtype,
                 residual=rng.random() < 0.7, out=rng.choice([dtype, "e4m3"]))
        return _limit(c, ("rows", "cols"), lambda x: x["rows"] * x["cols"] * BYTES[x["dtype"]], 1.6e8)
    if kind == "norm_backward":
        c = dict(kind="norm_backward", rows=_log(rng, 1, 32768), cols=_size(rng, 64, 16384, step),
                 dtype=rng.choice(["bf16", "bf16", "f32"]), residual=rng.random() < 0.7)
        return _limit(c, ("rows", "cols"), lambda x: x["rows"] * x["cols"] * BYTES[x["dtype"]], 1.2e8)
    if kind in ("linear", "linear_token"):
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        few = kind == "linear_token"
        c = dict(kind="linear", T=_log(rng, 1, 64) if few else _log(rng, 64, 16384), fin=_size(rng, 128, 11008, step),
                 fout=_size(rng, 128, 11008, step), dtype=dtype, out=rng.choice([dtype, dtype, "f32"]),
                 act=rng.choice(["none", "relu", "gelu_tanh", "silu"]), bias=rng.random() < 0.6,
                 residual=rng.random() < 0.5, preact=not few and rng.random() < 0.4)
        return _limit(c, ("T", "fin", "fout"), lambda x: work(x)["flops"], 3.6e11 if dtype == "bf16" else 5e10)
    if kind == "linear_backward":
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        c = dict(kind="linear_backward", T=_log(rng, 1, 16384), fin=_size(rng, 128, 11008, step),
                 fout=_size(rng, 128, 11008, step), dtype=dtype, act=rng.choice(["none", "relu", "gelu_tanh", "silu"]))
        return _limit(c, ("T", "fin", "fout"), lambda x: work(x)["flops"], 7e11 if dtype == "bf16" else 1e11)
    if kind == "linear_8bit":
        c = dict(kind="linear_8bit", T=_log(rng, 1, 16384), fin=_size(rng, 256, 11008, 16), fout=_size(rng, 128, 11008, step),
                 out=rng.choice(["bf16", "f32"]), act=rng.choice(["none", "silu", "gelu_tanh"]), bias=rng.random() < 0.5,
                 residual=rng.random() < 0.5)
        return _limit(c, ("T", "fin", "fout"), lambda x: work(x)["flops"], 3.6e11)
    if rng.random() < 0.5:
        h = _size(rng, 128, 4096, rng.choice([8, 64]))
        return dict(kind="adamw", tensors="layer", h=h, F=int(h * rng.choice([2.6875, 3.5, 4]) * 0.65),
                    grad=rng.choice(["bf16", "f32"]), states=rng.choice([8, 32]) if h < 2500 else 8, copy=rng.random() < 0.8)
    # a flat buffer of tensors of any size, one behind the other
    return dict(kind="adamw", tensors="flat", count=_log(rng, 1, 200), most=_log(rng, 16, 400000), sizes=rng.randrange(1 << 20),
                grad=rng.choice(["bf16", "f32"]), states=rng.choice([8, 32]), copy=rng.random() < 0.8)


def _adam_sizes(c):
    if c["tensors"] == "layer":
        h, F = c["h"], c["F"]
        return [h * h] * 4 + [h * F] * 3 + [h] * 2
    g = torch.Generator()
    g.manual_seed(c["sizes"])
    return [int(x) for x in torch.randint(1, c["most"] + 1, (c["count"],), generator=g)]


# ---- inputs -----------------------------------------------------------------

class _Maker:
    def __init__(self, seed):
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(seed)

    def __call__(self, shape, dtype="f32", std=1.0, mean=0.0):
        t = torch.randn(shape, generator=self.g, device="cuda", dtype=torch.float32)
        return t.mul_(std).add_(mean).to(DTYPES[dtype])


def _empty(shape, dtype):
    return torch.empty(shape, dtype=dtype, device="cuda")


def _rows_in_8_bits(x):
    """Row-scaled e4m3 values of x, as a serving program has its weights."""
    scale = x.abs().amax(dim=1) / E4M3_MAX
    return (x / scale[:, None]).to(E4M3), scale


def prepare(case, seed):
    c, make = case, _Maker(seed)
    s = dict(case)
    if c["kind"] == "norm":
        shape = (c["rows"], c["cols"])
        # an outlier channel or two, as residual streams have them
        s["x"] = make(shape, c["dtype"], std=1.5)
        s["x"][:, :: max(1, c["cols"] // 3)] *= 8
        s["r"] = make(shape, c["dtype"]) if c["residual"] else None
        s["w"] = make(c["cols"], "f32", std=0.1, mean=1.0)
        s["y"] = _empty(shape, E4M3 if c["out"] == "e4m3" else DTYPES[c["out"]])
        s["scales"] = _empty(c["rows"], torch.float32) if c["out"] == "e4m3" else None
        s["sum"] = _empty(shape, DTYPES[c["dtype"]]) if c["residual"] else None
        s["inv_rms"] = _empty(c["rows"], torch.float32)
    elif c["kind"] == "norm_backward":
        shape = (c["rows"], c["cols"])
        s["h"] = make(shape, c["dtype"], std=1.5)
        s["dy"] = make(shape, c["dtype"], std=0.01)
        s["dsum"] = make(shape, c["dtype"], std=0.01) if c["residual"] else None
        s["w"] = make(c["cols"], "f32", std=0.1, mean=1.0)
        s["inv_rms"] = 1 / (s["h"].float().square().mean(dim=1) + EPS).sqrt()
        s["dx"] = _empty(shape, DTYPES[c["dtype"]])
        s["dw"] = _empty(c["cols"], torch.float32)
        if own:
            import paper_2512_22142_amd as cleave
            s["ws"] = _empty(cleave.rms_norm_workspace(*shape), torch.float32)
    elif c["kind"] == "linear":
        T, fin, fout = c["T"], c["fin"], c["fout"]
        s["x"] = make((T, fin), c["dtype"])
        s["w"] = make((fin, fout), c["dtype"], std=0.02)
        s["b"] = make(fout, "f32", std=0.1) if c["bias"] else None
        s["r"] = make((T, fout), c["out"]) if c["residual"] else None
        s["y"] = _empty((T, fout), DTYPES[c["out"]])
        s["z"] = _empty((T, fout), DTYPES[c["out"]]) if c["preact"] else None
        if own:
            _plans(s, (T, fout, fin, DTYPES[c["dtype"]]))
    elif c["kind"] == "linear_backward":
        # y = act(z) . w + b: from dy, the gradients of z, w and b
        T, fin, fout = c["T"], c["fin"], c["fout"]
        s["dy"] = make((T, fout), c["dtype"], std=0.01)
        s["z"] = make((T, fin), c["dtype"])
        s["a"] = _act(s["z"].float(), c["act"]).to(DTYPES[c["dtype"]])
        s["w"] = make((fin, fout), c["dtype"], std=0.02)
        s["dz"] = _empty((T, fin), DTYPES[c["dtype"]])
        s["dw"] = _empty((fin, fout), torch.float32)
        s["db"] = _empty(fout, torch.float32)
        if own:
            import paper_2512_22142_amd as cleave
            _plans(s, (T, fin, fout, DTYPES[c["dtype"]]), (fin, fout, T, DTYPES[c["dtype"]]))
            s["ws"] = _empty(cleave.bias_grad_workspace(T, fout), torch.float32)
    elif c["kind"] == "linear_8bit":
        T, fin, fout = c["T"], c["fin"], c["fout"]
        s["x"], s["sx"] = _rows_in_8_bits(make((T, fin)))
        s["w"], s["sw"] = _rows_in_8_bits(make((fout, fin), std=0.02))      # laid out x in
        s["b"] = make(fout, "f32", std=0.1) if c["bias"] else None
        s["r"] = make((T, fout), c["out"]) if c["residual"] else None
        s["y"] = _empty((T, fout), DTYPES[c["out"]])
        if own:
            _plans(s, (T, fout, fin, E4M3))
    else:
        _prepare_adamw(s, make)
    return s


def _plans(s, *shapes):
    """One plan per product and the workspace that they share, as a program keeps them."""
    import paper_2512_22142_amd as cleave
    s["plans"] = [cleave.plan_linear(*shape) for shape in shapes]
    for plan in s["plans"]:
        plan.upload()
    s["partials"] = _empty(max(plan.linear_workspace for plan in s["plans"]), torch.float32)


def _prepare_adamw(s, make):
    sizes = _adam_sizes(s)
    n = sum(sizes)
    g, w = make(n, s["grad"], std=1e-3), make(n, std=0.02)
    m = make(n, std=3e-4)
    v = make(n).mul_(0.8).exp_().mul_(1e-6)       # squares of gradients around 1e-3, over two decades
    parts = lambda t: list(t.split(sizes))        # noqa: E731  (views, at any alignment)
    if s["tensors"] == "layer":                   # allocations of their own
        parts = lambda t: [x.clone() for x in t.split(sizes)]   # noqa: E731
    s["flat"] = {"w": w, "copy": w.to(torch.bfloat16) if s["copy"] else None}
    if s["states"] == 8:
        ms, vs, m_scale, v_scale = zip(*(_states_8(a, b) for a, b in zip(m.split(sizes), v.split(sizes))))
        blocks = [len(x) for x in m_scale]
        s["flat"].update(m=torch.cat(ms), v=torch.cat(vs), m_scale=torch.cat(m_scale), v_scale=torch.cat(v_scale))
    else:
        s["flat"].update(m=m, v=v)
    s["g"] = parts(g)
    s["clip"] = torch.full((1,), CLIP, device="cuda")
    for name, t in s["flat"].items():
        if t is None:
            s[name + "s"] = None
        elif name.endswith("_scale"):
            s[name + "s"] = [x.clone() for x in t.split(blocks)] if s["tensors"] == "layer" else list(t.split(blocks))
        else:
            s[name + "s"] = parts(t)
    if s["tensors"] == "layer":
        del s["flat"]


def _states_8(m, v):
    m8, m_scale = _to_blocks(m, False)
    v8, v_scale = _to_blocks(v.sqrt(), True)
    return m8, v8, m_scale, v_scale


# ---- the plain forms ------------------------------------------------------------

def _act(z, act):
    if act == "relu":
        return z.clamp_min(0)
    if act == "silu":
        return z / (1 + (-z).exp())
    if act == "gelu_tanh":
        return z / (1 + (-2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z)).exp())
    return z


def _act_grad(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "silu":
        p = 1 / (1 + (-z).exp())
        return p * (1 + z * (1 - p))
    if act == "gelu_tanh":
        k = 2 * math.sqrt(2 / math.pi)
        p = 1 / (1 + (-k * (z + 0.044715 * z * z * z)).exp())
        return p + z * p * (1 - p) * k * (1 + 3 * 0.044715 * z * z)
    return torch.ones_like(z)


def _norm(s):
    h = s["x"].float()
    if s["r"] is not None:
        h = h + s["r"].float()
    inv = 1 / (h.square().mean(dim=1) + EPS).sqrt()
    y = h * inv[:, None] * s["w"]
    out = {"inv_rms": inv}
    if s["r"] is not None:
        out["sum"] = h.to(s["x"].dtype)
    if s["out"] != "e4m3":
        out["y"] = y.to(DTYPES[s["out"]])
        return out
    most = y.abs().amax(dim=1)
    scale = torch.where(most >= LEAST, most / E4M3_MAX, torch.zeros_like(most))
    out["y"] = torch.where(scale[:, None] > 0, y * (1 / scale)[:, None], torch.zeros_like(y)).to(E4M3)
    out["scales"] = scale
    return out


def _norm_backward(s):
    xhat = s["h"].float() * s["inv_rms"][:, None]
    dy = s["dy"].float()
    g = dy * s["w"]
    dx = (g - xhat * (g * xhat).mean(dim=1, keepdim=True)) * s["inv_rms"][:, None]
    if s["dsum"] is not None:
        dx = dx + s["dsum"].float()
    return {"dx": dx.to(s["dx"].dtype), "dw": (dy * xhat).sum(dim=0)}


def _epilogue(s, z):
    if s["b"] is not None:
        z = z + s["b"]
    y = _act(z, s["act"])
    if s["r"] is not None:
        y = y + s["r"].float()
    return z, y


def _linear(s):
    z, y = _epilogue(s, s["x"].float() @ s["w"].float())
    out = {"y": y.to(s["y"].dtype)}
    if s["preact"]:
        out["z"] = z.to(s["y"].dtype)
    return out


def _linear_8bit(s):
    z = (s["x"].float() @ s["w"].float().t().contiguous()) * s["sx"][:, None] * s["sw"]
    return {"y": _epilogue(s, z)[1].to(s["y"].dtype)}


def _linear_backward(s):
    dy = s["dy"].float()
    dz = (dy @ s["w"].float().t().contiguous()) * _act_grad(s["z"].float(), s["act"])
    return {"dz": dz.to(s["dz"].dtype), "dw": s["a"].float().t().contiguous() @ dy, "db": dy.sum(dim=0)}


def _to_blocks(x, up):
    """e4m3 values of x and a scale per block. `up`: nothing above zero becomes zero."""
    n = x.numel()
    blocks = -(-n // STATE_BLOCK)
    b = torch.zeros(blocks * STATE_BLOCK, dtype=torch.float32, device=x.device)
    b[:n] = x.reshape(-1)
    b = b.view(blocks, STATE_BLOCK)
    most = b.abs().amax(dim=1)
    scale = torch.where(most >= LEAST, most / E4M3_MAX, torch.zeros_like(most))
    q = torch.where(scale[:, None] > 0, b * (1 / scale)[:, None], torch.zeros_like(b))
    if up:
        q = torch.where((b > 0) & (scale[:, None] > 0), q.clamp_min(2.0 ** -9), q)
    return q.view(-1)[:n].to(E4M3), scale


def _from_blocks(q, scale):
    return q.float() * scale.repeat_interleave(STATE_BLOCK)[: q.numel()]


def _adamw(s):
    a = ADAM
    ib1, ib2 = 1 / (1 - a["beta1"] ** a["step"]), 1 / (1 - a["beta2"] ** a["step"])
    for k in range(len(s["ws"])):
        w, g = s["ws"][k], s["g"][k].float() * s["clip"]
        if s["states"] == 8:
            m, r = _from_blocks(s["ms"][k], s["m_scales"][k]), _from_blocks(s["vs"][k], s["v_scales"][k])
            v = r * r
        else:
            m, v = s["ms"][k], s["vs"][k]
        m = a["beta1"] * m + (1 - a["beta1"]) * g
        v = a["beta2"] * v + (1 - a["beta2"]) * (g * g)
        w.copy_(w - a["lr"] * ((m * ib1) / ((v * ib2).sqrt() + a["eps"]) + a["weight_decay"] * w))
        if s["copys"] is not None:
            s["copys"][k].copy_(w)
        if s["states"] == 8:
            m, m_scale = _to_blocks(m, False)
            v, v_scale = _to_blocks(v.sqrt(), True)
            s["m_scales"][k].copy_(m_scale)
            s["v_scales"][k].copy_(v_scale)
        s["ms"][k].copy_(m)
        s["vs"][k].copy_(v)
    return _adamw_out(s)


def _adamw_out(s):
    names = ["w", "m", "v"] + (["copy"] if s["copy"] else []) + (["m_scale", "v_scale"] if s["states"] == 8 else [])
    return {n: s["flat"][n] if s["tensors"] == "flat" else s[n + "s"] for n in names}


# ---- one pass ---------------------------------------------------------------------

def run(state):
    s, kind = state, state["kind"]
    if not own:
        return {"norm": _norm, "norm_backward": _norm_backward, "linear": _linear, "linear_backward": _linear_backward,
                "linear_8bit": _linear_8bit, "adamw": _adamw}[kind](s)
    import paper_2512_22142_amd as cleave
    if kind == "norm":
        cleave.rms_norm(s["x"], s["w"], s["y"], residual=s["r"], sum_out=s["sum"], inv_rms=s["inv_rms"], scales=s["scales"],
                        eps=EPS)
        names = ["y", "inv_rms"] + (["sum"] if s["residual"] else []) + (["scales"] if s["out"] == "e4m3" else [])
        return {n: s[n] for n in names}
    if kind == "norm_backward":
        cleave.rms_norm_backward(s["dy"], s["h"], s["w"], s["inv_rms"], s["dx"], s["dw"], s["ws"], dsum=s["dsum"])
        return {"dx": s["dx"], "dw": s["dw"]}
    if kind == "linear":
        cleave.linear(s["plans"][0], s["x"], s["w"], s["y"], bias=s["b"], act=s["act"], residual=s["r"], preact=s["z"],
                      partials=s["partials"])
        return {"y": s["y"], "z": s["z"]} if s["preact"] else {"y": s["y"]}
    if kind == "linear_backward":
        to_z, to_w = s["plans"]
        cleave.linear(to_z, s["dy"], s["w"], s["dz"], transB=1, act_grad=s["act"], preact=s["z"], partials=s["partials"])
        cleave.linear(to_w, s["a"], s["dy"], s["dw"], transA=1, partials=s["partials"])
        cleave.bias_grad(s["dy"], s["db"], s["ws"])
        return {"dz": s["dz"], "dw": s["dw"], "db": s["db"]}
    if kind == "linear_8bit":
        cleave.linear(s["plans"][0], s["x"], s["w"], s["y"], transB=1, scale_a=s["sx"], scale_b=s["sw"], bias=s["b"],
                      act=s["act"], residual=s["r"], partials=s["partials"])
        return {"y": s["y"]}
    cleave.adamw(s["ws"], s["g"], s["ms"], s["vs"], m_scales=s.get("m_scales"), v_scales=s.get("v_scales"), copies=s["copys"],
                 grad_scale=s["clip"], **ADAM)
    return _adamw_out(s)


# ---- what a pass cannot do without ------------------------------------------------

def work(case):
    c = case
    if c["kind"] == "norm":
        n, e = c["rows"] * c["cols"], BYTES[c["dtype"]]
        bytes_ = n * e * (3 if c["residual"] else 1) + n * BYTES[c["out"]] + 4 * c["cols"] + 4 * c["rows"]
        return {"bytes": bytes_ + (4 * c["rows"] if c["out"] == "e4m3" else 0), "flops": 5 * n}
    if c["kind"] == "norm_backward":
        n, e = c["rows"] * c["cols"], BYTES[c["dtype"]]
        return {"bytes": n * e * (4 if c["residual"] else 3) + 8 * c["cols"] + 4 * c["rows"], "flops": 10 * n}
    if c["kind"] == "adamw":
        n = sum(_adam_sizes(c))
        state = 2 * (1 + 4 / STATE_BLOCK) if c["states"] == 8 else 8
        return {"bytes": n * (BYTES[c["grad"]] + 8 + 2 * state + (2 if c["copy"] else 0)), "flops": 15 * n}
    T, fin, fout = c["T"], c["fin"], c["fout"]
    flops = 2 * T * fin * fout
    if c["kind"] == "linear_backward":
        e = BYTES[c["dtype"]]
        return {"bytes": e * (T * fout + 3 * T * fin + fin * fout) + 4 * (fin * fout + fout), "flops": 2 * flops}
    e, o = BYTES[c.get("dtype", "e4m3")], BYTES[c["out"]]
    bytes_ = e * (T * fin + fin * fout) + o * T * fout * (1 + bool(c["residual"]) + bool(c.get("preact"))) + 4 * fout * bool(c["bias"])
    return {"bytes": bytes_ + (4 * (T + fout) if c["kind"] == "linear_8bit" else 0), "flops": flops}


# ---- the definition, in 64 bits ------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    d = lambda k: s[k].double() if s[k] is not None else None   # noqa: E731
    kind = case["kind"]
    if kind == "norm":
        h = d("x") if s["r"] is None else d("x") + d("r")
        inv = torch.rsqrt(torch.mean(h * h, dim=-1) + EPS)
        y = torch.einsum("ij,i,j->ij", h, inv, d("w"))
        out = {"inv_rms": inv, "y": y}
        if s["r"] is not None:
            out["sum"] = h
        if case["out"] == "e4m3":
            out["scales"] = torch.amax(torch.abs(y), dim=-1) / 448
            out["y"] = y / out["scales"].unsqueeze(-1)
        return out
    if kind == "norm_backward":
        # y_j = h_j w_j / rms: dh = (J of the norm)^T dy + dsum, with the given 1 / rms
        h, dy, inv, w = d("h"), d("dy"), d("inv_rms"), d("w")
        dots = torch.sum(dy * w * h, dim=-1) / h.shape[1]
        dx = dy * w * inv.unsqueeze(-1) - h * (dots * inv ** 3).unsqueeze(-1)
        if s["dsum"] is not None:
            dx += d("dsum")
        return {"dx": dx, "dw": torch.mv((dy * h).t(), inv)}
    if kind == "adamw":
        return _exact_adamw(s)
    act, grad = _EXACT_ACT[case["act"]]
    if kind == "linear_backward":
        dy = d("dy")
        return {"dz": torch.mm(dy, d("w").t()) * grad(d("z")), "dw": torch.mm(d("a").t(), dy), "db": dy.sum(0)}
    if kind == "linear_8bit":
        z = torch.mm(d("x") * d("sx").unsqueeze(1), (d("w") * d("sw").unsqueeze(1)).t())
    else:
        z = torch.mm(d("x"), d("w"))
    if s["b"] is not None:
        z = z + d("b")
    y = act(z)
    if s["r"] is not None:
        y = y + d("r")
    return {"y": y, "z": z} if case.get("preact") else {"y": y}


_GELU = math.sqrt(2 / math.pi)


def _gelu_grad(z):
    t = torch.tanh(_GELU * (z + 0.044715 * z ** 3))
    return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * _GELU * (1 + 0.134145 * z * z)


_EXACT_ACT = {
    "none": (lambda z: z, lambda z: 1.0),
    "relu": (torch.relu, lambda z: (z > 0).double()),
    "silu": (lambda z: z * torch.sigmoid(z), lambda z: torch.sigmoid(z) + z * torch.sigmoid(z) * torch.sigmoid(-z)),
    "gelu_tanh": (lambda z: 0.5 * z * (1 + torch.tanh(_GELU * (z + 0.044715 * z ** 3))), _gelu_grad),
}


def _exact_adamw(s):
    out = {n: [] for n in ["w", "m", "v"] + ["copy"] * s["copy"] + ["m_scale", "v_scale"] * (s["states"] == 8)}
    for k, w in enumerate(s["ws"]):
        w, g = w.double(), s["g"][k].double() * CLIP
        m, v = s["ms"][k].double(), s["vs"][k].double()
        if s["states"] == 8:
            of = torch.arange(w.numel(), device=w.device) // STATE_BLOCK
            m, v = m * s["m_scales"][k].double()[of], (v * s["v_scales"][k].double()[of]) ** 2
        m = torch.lerp(g, m, ADAM["beta1"])
        v = torch.lerp(g * g, v, ADAM["beta2"])
        root = torch.sqrt(v / (1 - ADAM["beta2"] ** ADAM["step"])) + ADAM["eps"]
        w = w * (1 - ADAM["lr"] * ADAM["weight_decay"]) - ADAM["lr"] / (1 - ADAM["beta1"] ** ADAM["step"]) * m / root
        if s["states"] == 8:
            v = torch.sqrt(v)
            for name, x in (("m", m), ("v", v)):
                top = torch.zeros(int(of[-1]) + 1, dtype=torch.float64, device=w.device)
                top.scatter_reduce_(0, of, torch.abs(x), "amax")
                out[name + "_scale"].append(top / 448)
                out[name].append(x * (448 / top)[of])
        else:
            out["m"].append(m)
            out["v"].append(v)
        out["w"].append(w)
        if s["copy"]:
            out["copy"].append(w)
    return {n: torch.cat(x) for n, x in out.items()} if s["tensors"] == "flat" else out
