"""More operators of a training or serving step, as cases that are timed and compared.

Three operators and their gradients: the layer norm of a residual stream, the two
projections of a gated feed-forward block with the activation and the product between
them, and the log probabilities of given tokens with entropy and the most likely
alternatives.  `run` is one pass through one of them: through the package where `own`
is true, else in plain torch operations in 32 bits.

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
LEAST = 2.0 ** -100        # a row whose largest value is below is stored as zeros
EPS = 1e-5


def listed():
    return [
        # One token of a serving batch: the norm in front of an 8-bit product. Latency.
        dict(name="norm_token_8bit", kind="norm", rows=1, cols=4096, dtype="bf16", residual=True, bias=True, out="e4m3"),
        # A micro-batch through the narrow layer's norm: residual added, the sum and the statistics kept for the backward pass.
        dict(name="norm_layer", kind="norm", rows=8192, cols=768, dtype="bf16", residual=True, bias=True, out="bf16"),
        # The widest layer's gradient in training, joined with the residual stream's.
        dict(name="norm_backward", kind="norm_backward", rows=16384, cols=5120, dtype="bf16", residual=True, bias=True),
        # Packed sequences, a width that is no multiple of a vector, fp32, no bias.
        dict(name="norm_backward_ragged", kind="norm_backward", rows=2999, cols=1111, dtype="f32", residual=False, bias=False),
        # One token through gate and up: both weights are read once. Latency.
        dict(name="gated_token", kind="gated", T=1, fin=4096, F=11008, dtype="bf16", out="bf16", act="silu", layout="kn",
             bias=False, keep=False),
        # The same in training: both arguments are kept for the backward pass.
        dict(name="gated_layer", kind="gated", T=4096, fin=4096, F=11008, dtype="bf16", out="bf16", act="silu", layout="kn",
             bias=False, keep=True),
        # Packed sequences, no size a multiple of a tile, with biases.
        dict(name="gated_ragged", kind="gated", T=1999, fin=1000, F=2500, dtype="bf16", out="bf16", act="gelu_tanh", layout="kn",
             bias=True, keep=False),
        # A prompt through 8-bit weights, as a norm leaves its rows.
        dict(name="gated_8bit", kind="gated_8bit", T=4096, fin=4096, F=11008, out="bf16", act="silu", bias=False),
        # Backward through the block: the down projection, the gate, and the gradients of input and weights.
        dict(name="gated_backward", kind="gated_backward", T=4096, fin=4096, F=11008, dtype="bf16", act="silu"),
        # A token is sampled: its log probability and the twenty most likely ones. Latency.
        dict(name="log_probs_token", kind="log_probs", rows=1, cols=32000, dtype="bf16", top=20, masked=0.0, scale=1.0),
        # A prompt is scored at a temperature, a grammar leaving a tenth of a vocabulary that is no multiple of a vector.
        dict(name="log_probs_prompt", kind="log_probs", rows=3001, cols=50257, dtype="f32", top=5, masked=0.9, scale=1.25),
        # A training step's loss with an entropy bonus: log probabilities and the gradient of the logits.
        dict(name="log_probs_step", kind="log_probs_step", rows=8192, cols=32000, dtype="bf16", masked=0.0, scale=1.0),
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
    kind = rng.choice(["norm", "norm", "norm_backward", "gated", "gated", "gated_token", "gated_8bit", "gated_backward",
                       "log_probs", "log_probs", "log_probs_token", "log_probs_step"])
    step = rng.choice([1, 8, 64, 64])
    acts = ["silu", "silu", "gelu_tanh", "relu", "none"]
    if kind in ("norm", "norm_backward"):
        dtype = rng.choice(["bf16", "bf16", "f32"])
        c = dict(kind=kind, rows=_log(rng, 1, 32768), cols=_size(rng, 64, 16384, step), dtype=dtype,
                 residual=rng.random() < 0.7, bias=rng.random() < 0.7)
        if kind == "norm":
            c["out"] = rng.choice([dtype, dtype, "e4m3"])
        return _limit(c, ("rows", "cols"), lambda x: x["rows"] * x["cols"] * BYTES[x["dtype"]], 1.6e8)
    if kind in ("gated", "gated_token"):
        dtype, few = rng.choice(["bf16", "bf16", "bf16", "f32"]), kind == "gated_token"
        c = dict(kind="gated", T=_log(rng, 1, 64) if few else _log(rng, 64, 16384), fin=_size(rng, 128, 11008, step),
                 F=_size(rng, 64, 11008, step), dtype=dtype, out=rng.choice([dtype, dtype, "f32"]), act=rng.choice(acts),
                 layout=rng.choice(["kn", "nk", "merged"]), bias=rng.random() < 0.4, keep=rng.random() < 0.4)
        return _limit(c, ("T", "fin", "F"), lambda x: work(x)["flops"], 7e11 if dtype == "bf16" else 1e11)
    if kind == "gated_8bit":
        c = dict(kind=kind, T=_log(rng, 1, 16384), fin=_size(rng, 256, 11008, 16), F=_size(rng, 64, 11008, step),
                 out=rng.choice(["bf16", "f32"]), act=rng.choice(acts), bias=rng.random() < 0.5)
        return _limit(c, ("T", "fin", "F"), lambda x: work(x)["flops"], 7e11)
    if kind == "gated_backward":
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        c = dict(kind=kind, T=_log(rng, 1, 16384), fin=_size(rng, 128, 8192, step), F=_size(rng, 64, 11008, step), dtype=dtype,
                 act=rng.choice(acts))
        return _limit(c, ("T", "fin", "F"), lambda x: work(x)["flops"], 1.8e12 if dtype == "bf16" else 2e11)
    dtype = rng.choice(["bf16", "f32"])
    few = kind == "log_probs_token"
    c = dict(kind="log_probs" if few else kind, rows=_log(rng, 1, 16) if few else _log(rng, 16, 16384),
             cols=_size(rng, 1024, 262144, step), dtype=dtype, masked=rng.choice([0.0, 0.0, 0.5, 0.9]),
             scale=rng.choice([1.0, 0.5, 1.25]))
    if c["kind"] == "log_probs":
        c["top"] = rng.choice([0, 1, 5, 20, 32])
    return _limit(c, ("rows", "cols"), lambda x: x["rows"] * x["cols"] * BYTES[x["dtype"]], 4.5e8)


# ---- inputs -----------------------------------------------------------------

class _Maker:
    def __init__(self, seed):
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(seed)

    def __call__(self, shape, dtype="f32", std=1.0, mean=0.0):
        t = torch.randn(shape, generator=self.g, device="cuda", dtype=torch.float32)
        return t.mul_(std).add_(mean).to(DTYPES[dtype])

    def ints(self, most, shape):
        return torch.randint(0, most, shape, generator=self.g, device="cuda")

    def uniform(self, shape):
        return torch.rand(shape, generator=self.g, device="cuda")


def _empty(shape, dtype):
    return torch.empty(shape, dtype=dtype, device="cuda")


def _rows_in_8_bits(x):
    """Row-scaled e4m3 values of x, as a serving program has its weights."""
    scale = x.abs().amax(dim=1) / E4M3_MAX
    return (x / scale[:, None]).to(E4M3), scale


def prepare(case, seed):
    c, make = case, _Maker(seed)
    s = dict(case)
    if c["kind"].startswith("norm"):
        return _prepare_norm(s, make)
    if c["kind"].startswith("log_probs"):
        return _prepare_log_probs(s, make)
    T, fin, F = c["T"], c["fin"], c["F"]
    if c["kind"] == "gated":
        s["x"] = make((T, fin), c["dtype"])
        if c["layout"] == "merged":              # one matrix, gate's columns before up's
            w = make((fin, 2 * F), c["dtype"], std=0.02)
            s["wg"], s["wu"] = w[:, :F], w[:, F:]
        else:
            shape = (fin, F) if c["layout"] == "kn" else (F, fin)
            s["wg"], s["wu"] = make(shape, c["dtype"], std=0.02), make(shape, c["dtype"], std=0.02)
        s["bg"], s["bu"] = (make(F, "f32", std=0.1) if c["bias"] else None for _ in range(2))
        s["y"] = _empty((T, F), DTYPES[c["out"]])
        s["zg"], s["zu"] = (_empty((T, F), DTYPES[c["out"]]) if c["keep"] else None for _ in range(2))
        if own:
            _plan_gated(s, DTYPES[c["dtype"]])
    elif c["kind"] == "gated_8bit":
        s["x"], s["sx"] = _rows_in_8_bits(make((T, fin)))
        s["wg"], s["sg"] = _rows_in_8_bits(make((F, fin), std=0.02))      # laid out x in
        s["wu"], s["su"] = _rows_in_8_bits(make((F, fin), std=0.02))
        s["bg"], s["bu"] = (make(F, "f32", std=0.1) if c["bias"] else None for _ in range(2))
        s["y"] = _empty((T, F), DTYPES[c["out"]])
        if own:
            _plan_gated(s, E4M3)
    else:
        # o = (act(x wg) (x wu)) wd: from do, the gradients of both arguments, of x and of gate's and up's weights
        s["do"] = make((T, fin), c["dtype"], std=0.01)
        s["x"] = make((T, fin), c["dtype"])
        s["w"] = make((fin, 2 * F), c["dtype"], std=0.02)
        s["wd"] = make((F, fin), c["dtype"], std=0.02)
        s["zg"], s["zu"] = make((T, F), c["dtype"]), make((T, F), c["dtype"])
        s["dz"] = _empty((T, 2 * F), DTYPES[c["dtype"]])
        s["dx"] = _empty((T, fin), DTYPES[c["dtype"]])
        s["dw"] = _empty((fin, 2 * F), DTYPES[c["dtype"]])     # as an optimizer takes them
        if own:
            import paper_2512_22142_amd as cleave
            d = DTYPES[c["dtype"]]
            s["plans"] = [cleave.plan_linear(T, F, fin, d), cleave.plan_linear(T, fin, 2 * F, d), cleave.plan_linear(fin, 2 * F, T, d)]
            for plan in s["plans"]:
                plan.upload()
            s["partials"] = _empty(max([cleave.gated_grad_workspace(s["plans"][0], whole=fin % 8 == 0)] +
                                       [plan.linear_workspace for plan in s["plans"][1:]]), torch.float32)
    return s


def _plan_gated(s, dtype):
    """The plan and its workspace, as a program keeps them."""
    import paper_2512_22142_amd as cleave
    s["plan"] = cleave.plan_gated(s["T"], s["F"], s["fin"], dtype)
    s["plan"].upload()
    whole = s["fin"] % 8 == 0 and (s["F"] % 8 == 0 or s.get("layout") == "nk")     # rows in whole sixteen bytes
    s["partials"] = _empty(cleave.gated_workspace(s["plan"], whole=whole), torch.float32)


def _prepare_norm(s, make):
    shape, d = (s["rows"], s["cols"]), DTYPES[s["dtype"]]
    s["w"] = make(s["cols"], "f32", std=0.1, mean=1.0)
    s["b"] = make(s["cols"], "f32", std=0.1) if s["bias"] else None
    if s["kind"] == "norm":
        # a mean, and an outlier channel or two, as residual streams have them
        s["x"] = make(shape, s["dtype"], std=1.5, mean=0.5)
        s["x"][:, :: max(1, s["cols"] // 3)] *= 8
        s["r"] = make(shape, s["dtype"]) if s["residual"] else None
        s["y"] = _empty(shape, E4M3 if s["out"] == "e4m3" else DTYPES[s["out"]])
        s["scales"] = _empty(s["rows"], torch.float32) if s["out"] == "e4m3" else None
        s["sum"] = _empty(shape, d) if s["residual"] else None
        s["mean"], s["inv"] = _empty(s["rows"], torch.float32), _empty(s["rows"], torch.float32)
        return s
    s["h"] = make(shape, s["dtype"], std=1.5, mean=0.5)
    s["dy"] = make(shape, s["dtype"], std=0.01)
    s["dsum"] = make(shape, s["dtype"], std=0.01) if s["residual"] else None
    h = s["h"].float()
    s["mean"] = h.mean(dim=1)
    s["inv"] = 1 / ((h - s["mean"][:, None]).square().mean(dim=1) + EPS).sqrt()
    s["dx"] = _empty(shape, d)
    s["dw"] = _empty(s["cols"], torch.float32)
    s["db"] = _empty(s["cols"], torch.float32) if s["bias"] else None
    if own:
        import paper_2512_22142_amd as cleave
        s["ws"] = _empty(cleave.layer_norm_workspace(*shape), torch.float32)
    return s


def _prepare_log_probs(s, make):
    rows, cols = s["rows"], s["cols"]
    s["l"] = make((rows, cols), s["dtype"], std=2.5)
    s["ids"] = make.ints(cols, (rows,))
    if s["masked"]:
        # what a grammar forbids; the given tokens are allowed
        gone = make.uniform((rows, cols)) < s["masked"]
        gone.scatter_(1, s["ids"][:, None], False)
        s["l"].masked_fill_(gone, -math.inf)
        del gone
    if rows > 8:
        s["ids"][::7] = -1                       # positions without a target, as padding has them
    s["logp"], s["lse"], s["ent"] = (_empty(rows, torch.float32) for _ in range(3))
    if s["kind"] == "log_probs_step":
        s["dlogp"] = make(rows, std=0.1, mean=-1.0).div_(rows)
        s["dent"] = make(rows, std=0.01).div_(rows)
        s["dl"] = _empty((rows, cols), DTYPES[s["dtype"]])
    elif s["top"]:
        s["top_ids"] = _empty((rows, s["top"]), torch.int64)
        s["top_logp"] = _empty((rows, s["top"]), torch.float32)
    if own:
        import paper_2512_22142_amd as cleave
        s["ws"] = _empty(cleave.log_probs_workspace(rows, cols, s.get("top", 0)), torch.float32)
    return s


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
    mean = h.mean(dim=1)
    d = h - mean[:, None]
    inv = 1 / (d.square().mean(dim=1) + EPS).sqrt()
    y = d * inv[:, None] * s["w"]
    if s["b"] is not None:
        y = y + s["b"]
    out = {"mean": mean, "inv_std": inv}
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
    xhat = (s["h"].float() - s["mean"][:, None]) * s["inv"][:, None]
    dy = s["dy"].float()
    g = dy * s["w"]
    dx = (g - g.mean(dim=1, keepdim=True) - xhat * (g * xhat).mean(dim=1, keepdim=True)) * s["inv"][:, None]
    if s["dsum"] is not None:
        dx = dx + s["dsum"].float()
    out = {"dx": dx.to(s["dx"].dtype), "dw": (dy * xhat).sum(dim=0)}
    if s["bias"]:
        out["db"] = dy.sum(dim=0)
    return out


def _gated(s):
    x = s["x"].float()
    if s["kind"] == "gated_8bit":
        zg = (x @ s["wg"].float().t().contiguous()) * s["sx"][:, None] * s["sg"]
        zu = (x @ s["wu"].float().t().contiguous()) * s["sx"][:, None] * s["su"]
    elif s["layout"] == "nk":
        zg, zu = x @ s["wg"].float().t().contiguous(), x @ s["wu"].float().t().contiguous()
    else:
        zg, zu = x @ s["wg"].float(), x @ s["wu"].float()
    if s["bg"] is not None:
        zg, zu = zg + s["bg"], zu + s["bu"]
    d = s["y"].dtype
    out = {"y": (_act(zg, s["act"]) * zu).to(d)}
    if s.get("keep"):
        out["gate"], out["up"] = zg.to(d), zu.to(d)
    return out


def _gated_backward(s):
    p = s["do"].float() @ s["wd"].float().t().contiguous()
    zg, zu = s["zg"].float(), s["zu"].float()
    d = s["dz"].dtype
    dz = torch.cat([p * zu * _act_grad(zg, s["act"]), p * _act(zg, s["act"])], dim=1).to(d)
    dx = (dz.float() @ s["w"].float().t().contiguous()).to(d)
    return {"dz": dz, "dx": dx, "dw": (s["x"].float().t().contiguous() @ dz.float()).to(d)}


def _statistics(s):
    l = s["l"].float() * s["scale"]
    most = l.amax(dim=1)
    e = (l - most[:, None]).exp()
    total = e.sum(dim=1)
    lse = most + total.log()
    p = e / total[:, None]
    logp = l - lse[:, None]
    ent = -torch.where(p > 0, p * logp, torch.zeros_like(p)).sum(dim=1)
    given = s["ids"] >= 0
    at = s["ids"].clamp_min(0)
    return p, logp, lse, ent, given, at


def _log_probs(s):
    _, logp, lse, ent, given, at = _statistics(s)
    out = {"logp": torch.where(given, logp.gather(1, at[:, None])[:, 0], torch.zeros_like(lse)), "lse": lse, "entropy": ent}
    if s["top"]:
        order = torch.sort(s["l"], dim=1, descending=True, stable=True)[1][:, : s["top"]]
        out["top_ids"], out["top_logp"] = order.contiguous(), logp.gather(1, order)
    return out


def _log_probs_step(s):
    p, logp, lse, ent, given, at = _statistics(s)
    out = {"logp": torch.where(given, logp.gather(1, at[:, None])[:, 0], torch.zeros_like(lse)), "lse": lse, "entropy": ent}
    d = torch.where(given, s["dlogp"], torch.zeros_like(lse))
    dl = -d[:, None] * p - s["dent"][:, None] * torch.where(p > 0, p * (logp + ent[:, None]), torch.zeros_like(p))
    dl.scatter_add_(1, at[:, None], d[:, None])
    out["dlogits"] = (dl * s["scale"]).to(s["l"].dtype)
    return out


# ---- one pass ---------------------------------------------------------------------

def run(state):
    s, kind = state, state["kind"]
    if not own:
        return {"norm": _norm, "norm_backward": _norm_backward, "gated": _gated, "gated_8bit": _gated,
                "gated_backward": _gated_backward, "log_probs": _log_probs, "log_probs_step": _log_probs_step}[kind](s)
    import paper_2512_22142_amd as cleave
    if kind == "norm":
        cleave.layer_norm(s["x"], s["w"], s["y"], bias=s["b"], residual=s["r"], sum_out=s["sum"], mean=s["mean"],
                          inv_std=s["inv"], scales=s["scales"], eps=EPS)
        out = {"mean": s["mean"], "inv_std": s["inv"], "y": s["y"]}
        if s["residual"]:
            out["sum"] = s["sum"]
        if s["out"] == "e4m3":
            out["scales"] = s["scales"]
        return out
    if kind == "norm_backward":
        cleave.layer_norm_backward(s["dy"], s["h"], s["w"], s["mean"], s["inv"], s["dx"], s["dw"], s["ws"], dbias=s["db"],
                                   dsum=s["dsum"])
        return {"dx": s["dx"], "dw": s["dw"], "db": s["db"]} if s["bias"] else {"dx": s["dx"], "dw": s["dw"]}
    if kind == "gated":
        cleave.linear_gated(s["plan"], s["x"], s["wg"], s["wu"], s["y"], transB=int(s["layout"] == "nk"), act=s["act"],
                            bias_gate=s["bg"], bias_up=s["bu"], gate=s["zg"], up=s["zu"], partials=s["partials"])
        return {"y": s["y"], "gate": s["zg"], "up": s["zu"]} if s["keep"] else {"y": s["y"]}
    if kind == "gated_8bit":
        cleave.linear_gated(s["plan"], s["x"], s["wg"], s["wu"], s["y"], transB=1, act=s["act"], bias_gate=s["bg"],
                            bias_up=s["bu"], scale_a=s["sx"], scale_gate=s["sg"], scale_up=s["su"], partials=s["partials"])
        return {"y": s["y"]}
    if kind == "gated_backward":
        F, (to_z, to_x, to_w) = s["F"], s["plans"]
        cleave.linear_gated_grad(to_z, s["do"], s["wd"], s["zg"], s["zu"], s["dz"][:, :F], s["dz"][:, F:], transB=1, act=s["act"],
                                 partials=s["partials"])
        cleave.linear(to_x, s["dz"], s["w"], s["dx"], transB=1, partials=s["partials"])
        cleave.linear(to_w, s["x"], s["dz"], s["dw"], transA=1, partials=s["partials"])
        return {"dz": s["dz"], "dx": s["dx"], "dw": s["dw"]}
    top = dict(top_ids=s["top_ids"], top_logp=s["top_logp"]) if s.get("top") else {}
    cleave.log_probs(s["l"], s["ids"], s["logp"], lse=s["lse"], entropy=s["ent"], scale=s["scale"], workspace=s["ws"], **top)
    out = {"logp": s["logp"], "lse": s["lse"], "entropy": s["ent"], **top}
    if kind == "log_probs_step":
        cleave.log_probs_backward(s["l"], s["lse"], s["dl"], ids=s["ids"], dlogp=s["dlogp"], entropy=s["ent"],
                                  dentropy=s["dent"], scale=s["scale"])
        out["dlogits"] = s["dl"]
    return out


# ---- what a pass cannot do without ------------------------------------------------

def work(case):
    c = case
    if c["kind"] in ("norm", "norm_backward"):
        n, e = c["rows"] * c["cols"], BYTES[c["dtype"]]
        if c["kind"] == "norm_backward":
            return {"bytes": n * e * (4 if c["residual"] else 3) + (8 + 4 * c["bias"]) * c["cols"] + 8 * c["rows"], "flops": 13 * n}
        bytes_ = n * e * (3 if c["residual"] else 1) + n * BYTES[c["out"]] + 4 * c["cols"] * (1 + c["bias"]) + 8 * c["rows"]
        return {"bytes": bytes_ + (4 * c["rows"] if c["out"] == "e4m3" else 0), "flops": 8 * n}
    if c["kind"].startswith("log_probs"):
        n, e = c["rows"] * c["cols"], BYTES[c["dtype"]]
        if c["kind"] == "log_probs_step":
            return {"bytes": 2 * n * e + 28 * c["rows"], "flops": 16 * n}
        return {"bytes": n * e + (20 + 12 * c["top"]) * c["rows"], "flops": 8 * n}
    T, fin, F = c["T"], c["fin"], c["F"]
    flops = 4 * T * fin * F
    if c["kind"] == "gated_backward":
        e = BYTES[c["dtype"]]
        return {"bytes": e * (3 * T * fin + 5 * fin * F + 4 * T * F), "flops": 10 * T * fin * F}
    e, o = BYTES[c.get("dtype", "e4m3")], BYTES[c["out"]]
    bytes_ = e * (T * fin + 2 * fin * F) + o * T * F * (3 if c.get("keep") else 1) + 8 * F * bool(c["bias"])
    return {"bytes": bytes_ + (4 * (T + 2 * F) if c["kind"] == "gated_8bit" else 0), "flops": flops}


# ---- the definition, in 64 bits ------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    d = lambda k: s[k].double() if s[k] is not None else None   # noqa: E731
    kind = case["kind"]
    if kind == "norm":
        h = d("x") if s["r"] is None else d("x") + d("r")
        var, mean = torch.var_mean(h, dim=-1, correction=0)
        inv = torch.rsqrt(var + EPS)
        y = torch.addcmul(torch.zeros_like(h) if s["b"] is None else d("b").expand_as(h), (h - mean.unsqueeze(-1)) * d("w"),
                          inv.unsqueeze(-1))
        out = {"mean": mean, "inv_std": inv, "y": y}
        if s["r"] is not None:
            out["sum"] = h
        if case["out"] == "e4m3":
            out["scales"] = torch.amax(torch.abs(y), dim=-1) / 448
            out["y"] = y / out["scales"].unsqueeze(-1)
        return out
    if kind == "norm_backward":
        # y_j = xhat_j w_j + b_j, xhat = (h - mean) / std with the given statistics: dh = (J of xhat)^T (dy w) + dsum
        xhat, dy, inv, n = torch.sub(d("h"), d("mean").unsqueeze(1)).mul_(d("inv").unsqueeze(1)), d("dy"), d("inv"), case["cols"]
        g = dy * d("w")
        dx = (g - torch.sum(g, dim=1, keepdim=True) / n).sub_(xhat * (torch.sum(g * xhat, dim=1, keepdim=True) / n))
        dx = dx.mul_(inv.unsqueeze(1))
        if s["dsum"] is not None:
            dx += d("dsum")
        out = {"dx": dx, "dw": torch.sum(dy * xhat, dim=0)}
        if case["bias"]:
            out["db"] = torch.sum(dy, dim=0)
        return out
    if kind.startswith("log_probs"):
        return _exact_log_probs(s)
    act, slope = _EXACT_ACT[case["act"]]
    if kind == "gated_backward":
        F = case["F"]
        p = torch.mm(d("do"), d("wd").t())
        zg = d("zg")
        dz = torch.empty(case["T"], 2 * F, dtype=torch.float64, device="cuda")
        dz[:, :F] = slope(zg) * d("zu") * p
        dz[:, F:] = act(zg) * p
        stored = dz.to(s["dz"].dtype).double()    # the products take what the first step leaves
        return {"dz": dz, "dx": torch.mm(stored, d("w").t()), "dw": torch.mm(d("x").t(), stored)}
    if kind == "gated_8bit":
        x = d("x") * d("sx").unsqueeze(1)
        zg, zu = torch.mm(x, (d("wg") * d("sg").unsqueeze(1)).t()), torch.mm(x, (d("wu") * d("su").unsqueeze(1)).t())
    elif case["layout"] == "nk":
        zg, zu = torch.mm(d("x"), d("wg").t()), torch.mm(d("x"), d("wu").t())
    else:
        zg, zu = torch.mm(d("x"), d("wg")), torch.mm(d("x"), d("wu"))
    if s["bg"] is not None:
        zg, zu = torch.add(zg, d("bg")), torch.add(zu, d("bu"))
    out = {"y": act(zg) * zu}
    if case.get("keep"):
        out["gate"], out["up"] = zg, zu
    return out


def _exact_log_probs(s):
    rows, cols = s["l"].shape
    ids, scale = s["ids"], s["scale"]
    parts = {"logp": [], "lse": [], "entropy": []}
    step = "dl" in s
    top = s.get("top", 0)
    if step:
        parts["dlogits"] = []
    if top:
        parts["top_ids"], parts["top_logp"] = [], []
    some = max(1, (1 << 26) // cols)              # rows at a time
    for r in range(0, rows, some):
        l = s["l"][r: r + some].double() * scale
        t = ids[r: r + some]
        lse = torch.logsumexp(l, dim=1)
        logp = l - lse.unsqueeze(1)
        ent = torch.special.entr(torch.exp(logp)).sum(1)
        hot = torch.zeros_like(l)
        has = torch.nonzero(t >= 0)[:, 0]
        hot[has, t[has]] = 1.0
        given = torch.zeros_like(lse)
        given[has] = logp[has, t[has]]
        parts["logp"].append(given)
        parts["lse"].append(lse)
        parts["entropy"].append(ent)
        if top:
            # the largest logit, the lowest index among equals: `top` times
            left = s["l"][r: r + some].double().clone()
            picks = []
            for _ in range(top):
                most = left.amax(dim=1, keepdim=True)
                at = (left == most).to(torch.int8).argmax(dim=1)
                picks.append(at)
                left.scatter_(1, at[:, None], -math.inf)
            picks = torch.stack(picks, dim=1)
            parts["top_ids"].append(picks)
            parts["top_logp"].append(torch.gather(logp, 1, picks))
        if step:
            p = torch.exp(logp)
            dlogp, dent = s["dlogp"][r: r + some].double(), s["dent"][r: r + some].double()
            dlogp = dlogp * (t >= 0)
            dl = torch.sub(hot, p).mul_(dlogp.unsqueeze(1))
            dl += (torch.special.entr(p) - p * ent.unsqueeze(1)) * dent.unsqueeze(1)
            parts["dlogits"].append((dl * scale).float() if s["dl"].dtype == torch.bfloat16 else dl * scale)
    return {k: torch.cat(v) for k, v in parts.items()}


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
