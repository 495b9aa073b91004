"""Measured work of the operators around a gated block that is trained in the clear: the norms before and after it with its gate and
residual sum, the update of its matrices by orthogonalised momentum, and its answers from 4-bit weights.

A program that trains a head in the clear wraps each block in norms (r = a x + b gate * norm(f), n = norm(r)), takes their backward
pass, and moves the matrices along the orthogonalised momentum of their gradients (Newton-Schulz products).  Once trained, the
same block answers cleartext requests of a few rows from weights in 4 bits with a scale for every group.  `run` makes these calls
where `own` is true; where it is false it computes them by elementary torch operations in 32 bits, rounded once at the end.

Rows of a residual stream have a few channels far larger than the others; gradients of matrices are a few strong directions above
noise, as sums over a batch are, and differ in size from matrix to matrix; weights are N(0, 1/fan_in), their codes spread over the 16 values.
"""
import math
import random

import torch

own = False

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EPS, RESIDUAL, BLOCK_SCALE = 1e-5, 0.9, 0.8
LR, MOMENTUM, DECAY, NORM_EPS, STEPS = 0.02, 0.95, 0.01, 1e-7, 5
COEFFICIENTS = (3.4445, -4.7750, 2.0315)


def listed():
    return [
        # between two blocks while one request is answered: latency
        {"name": "norm_1x4096", "op": "norm", "rows": 1, "d": 4096, "type": "bf16", "weights": "bf16", "pre": "rms", "post": "rms", "gate": "none", "train": False},
        # a batch of answers at the fully connected width of Table 1, full precision
        {"name": "norm_4096x4096", "op": "norm", "rows": 4096, "d": 4096, "type": "f32", "weights": "f32", "pre": "layer", "post": "none", "gate": "channel", "train": False},
        # a training step of odd sizes, a gate for every element
        {"name": "norm_train_333x1021", "op": "norm", "rows": 333, "d": 1021, "type": "f16", "weights": "f32", "pre": "layer", "post": "layer", "gate": "element",
         "train": True},
        # ... of the largest block, a learned scale for every channel
        {"name": "norm_train_16384x2048", "op": "norm", "rows": 16384, "d": 2048, "type": "bf16", "weights": "f32", "pre": "rms", "post": "rms", "gate": "channel",
         "train": True},
        # the direction of one small matrix: launches
        {"name": "ortho_64x100", "op": "ortho", "sizes": "64x100", "type": "f32"},
        # ... of a large square one
        {"name": "ortho_4096x4096", "op": "ortho", "sizes": "4096x4096", "type": "bf16"},
        # a step over a small head's matrices (3136 -> 256 -> 2)
        {"name": "muon_3136", "op": "muon", "sizes": "256x3136 256x3136 2x256", "type": "f32", "grads": "f32", "copy": False},
        # ... over the matrices of four blocks (1024 -> 4096 -> 1024), 16-bit copies for the next forward pass
        {"name": "muon_12x1024", "op": "muon", "sizes": " ".join(["4096x1024 4096x1024 1024x4096"] * 4), "type": "f32", "grads": "bf16", "copy": True},
        # one request through a block with 4-bit weights: latency, the weights are read once
        {"name": "ff4_1x1024", "op": "ff4", "rows": 1, "d_in": 1024, "d_hidden": 4096, "d_out": 1024, "type": "bf16", "act": "silu", "group": 128},
        # a handful of requests at sizes that are multiples of nothing, small groups
        {"name": "ff4_7x999", "op": "ff4", "rows": 7, "d_in": 999, "d_hidden": 2731, "d_out": 501, "type": "f16", "act": "poly3", "group": 32},
        # one row and one wide matrix: the bytes of the codes
        {"name": "product4_1x8192", "op": "product4", "rows": 1, "d_in": 8192, "d_out": 16384, "type": "bf16", "group": 128},
        # the most rows that such products are meant for, in full precision
        {"name": "product4_64x4096", "op": "product4", "rows": 64, "d_in": 4096, "d_out": 4096, "type": "f32", "group": 64},
    ]


def _size(rng, least, most):
    """spread over the logarithm; half of the sizes multiples of 64, a quarter of 8, a quarter of anything"""
    n = int(round(math.exp(rng.uniform(math.log(least), math.log(most)))))
    step = rng.choice((64, 64, 8, 1))
    return max(least, min(most, n if n < step else n // step * step))


def _operations(rows, cols):
    """of the products of one matrix: X X^T and its square are symmetric, one half of each is enough"""
    m, n = min(rows, cols), max(rows, cols)
    return STEPS * (1.0 * m * m * n + 1.0 * m * m * m + 2.0 * m * m * n)


def draw(rng):
    op = rng.choice(("norm", "norm", "ortho", "muon", "ff4", "product4"))
    kind = rng.choice(("bf16", "bf16", "f16", "f32"))
    if op == "norm":
        while True:
            # single rows and a handful are drawn as often as batches
            rows, d = _size(rng, 1, rng.choice((16, 32768))), _size(rng, 8, 16384)
            if rows * d <= 16384 * 2048 / 2:
                break
        pre, post = rng.choice((("rms", "rms"), ("rms", "none"), ("none", "rms"), ("layer", "layer"), ("layer", "none"), ("rms", "layer")))
        return {"op": op, "rows": rows, "d": d, "type": kind, "weights": rng.choice((kind, "f32")), "pre": pre, "post": post,
                "gate": rng.choice(("none", "channel", "element")), "train": rng.random() < 0.6}
    if op in ("ortho", "muon"):
        while True:
            r, c = _size(rng, 1, 4096), _size(rng, 1, 4096)
            count = 1 if op == "ortho" else _size(rng, 1, 24)
            shapes = [(r, c) if rng.random() < 0.6 else (c, r) if rng.random() < 0.5 else (_size(rng, 1, 2048), c) for _ in range(count)]
            if sum(_operations(*s) for s in shapes) <= _operations(4096, 4096) / 2:
                break
        case = {"op": op, "sizes": " ".join("%dx%d" % s for s in shapes), "type": kind}
        return case if op == "ortho" else dict(case, grads=rng.choice((kind, "bf16")), copy=kind == "f32" and rng.random() < 0.5)
    rows, d_in, d_out = _size(rng, 1, rng.choice((8, 64))), _size(rng, 32, 8192), _size(rng, 2, 8192)
    case = {"op": op, "rows": rows, "d_in": d_in, "d_out": d_out, "type": kind, "group": rng.choice((32, 64, 128, 256))}
    return case if op == "product4" else dict(case, d_hidden=_size(rng, 32, 8192), act=rng.choice(("linear", "square", "poly2", "poly3", "relu", "silu", "gelu")))


# the cubics c0 + c1 g + c2 g^2 + c3 g^3 of the encrypted schedules
CUBICS = {
    "linear": (0.0, 1.0, 0.0, 0.0),
    "square": (0.0, 0.0, 1.0, 0.0),
    "poly2": (0.0, 0.500000000000008, 0.000469841857369822, 0.0),
    "poly3": (0.5, 0.25, 0.0, -0.02),
}


def _shapes(case):
    return [tuple(int(v) for v in s.split("x")) for s in case["sizes"].split()]


def _normal(g, shape, scale=1.0):
    return torch.randn(shape, generator=g, device=DEV).mul_(scale)


# --------------------------------------------------------------------------- inputs
def _norm_inputs(case, seed):
    g = torch.Generator(DEV).manual_seed(seed)
    M, d, t, tw = case["rows"], case["d"], TYPES[case["type"]], TYPES[case["weights"]]
    s = {"x": (_normal(g, (M, d)) * torch.exp(_normal(g, (d,), 0.7)) + 0.1).to(t), "f": _normal(g, (M, d), 0.5).to(t)}
    for k in ("pre", "post"):
        if case[k] != "none":
            s[k + "_weight"] = (1.0 + _normal(g, (d,), 0.2)).to(tw)
        if case[k] == "layer":
            s[k + "_bias"] = _normal(g, (d,), 0.1).to(tw)
    if case["gate"] != "none":
        s["gate"] = _normal(g, (d,), 0.5).to(tw) if case["gate"] == "channel" else torch.sigmoid(_normal(g, (M, d))).to(t)
    if case["train"]:
        s["dr"] = _normal(g, (M, d)).to(t)
        if case["pre"] != "none":
            s["dn"] = _normal(g, (M, d)).to(t)
    return s


def _matrix(g, rows, cols, scale):
    """four strong directions above noise (sums over a batch); elements of the order of `scale`"""
    a = _normal(g, (rows, cols), 0.3)
    for k in range(4):
        a += _normal(g, (rows, 1), 0.8 * 0.7**k) * _normal(g, (1, cols))
    return a.mul_(scale)


def _ortho_inputs(case, seed):
    g = torch.Generator(DEV).manual_seed(seed)
    return {"u": [_matrix(g, r, c, 1e-3).to(TYPES[case["type"]]) for r, c in _shapes(case)]}


def _muon_inputs(case, seed):
    """parameters, gradients and the momentum that earlier steps left"""
    g = torch.Generator(DEV).manual_seed(seed)
    s = {"p": [], "g": [], "m": []}
    for i, (r, c) in enumerate(_shapes(case)):
        scale = 10.0 ** (-3 + i % 3)
        s["p"].append(_normal(g, (r, c), c**-0.5).to(TYPES[case["type"]]))
        s["g"].append(_matrix(g, r, c, scale).to(TYPES[case["grads"]]))
        s["m"].append(_matrix(g, r, c, 0.3 * scale))
    if case["copy"]:
        s["copy"] = [p.to(torch.bfloat16) for p in s["p"]]
    return s


def _weights4(g, d_out, d_in, group, dtype):
    """codes (two's complement, the even element of a pair in the lower half of its byte, rows padded to whole 16 bytes) and scales"""
    c = torch.round(_normal(g, (d_out, d_in), 2.5)).clamp_(-8, 7).to(torch.int64) & 15
    whole = torch.zeros(d_out, -(-d_in // 32) * 32, dtype=torch.int64, device=DEV)
    whole[:, :d_in] = c
    scales = (torch.rand((d_out, -(-d_in // group)), generator=g, device=DEV) * 0.6 + 0.7) * (0.4 * d_in**-0.5)
    return (whole[:, 0::2] | whole[:, 1::2] << 4).to(torch.uint8), scales.to(dtype)


def _low_inputs(case, seed):
    g = torch.Generator(DEV).manual_seed(seed)
    t, K, O, G = TYPES[case["type"]], case["d_in"], case["d_out"], case["group"]
    s = {"x": _normal(g, (case["rows"], K)).to(t)}
    if case["op"] == "product4":
        s["w"] = _weights4(g, O, K, G, t)
    else:
        H = case["d_hidden"]
        s["gate"], s["up"], s["down"] = _weights4(g, H, K, G, t), _weights4(g, H, K, G, t), _weights4(g, O, H, G, t)
    return s


INPUTS = {"norm": _norm_inputs, "ortho": _ortho_inputs, "muon": _muon_inputs, "ff4": _low_inputs, "product4": _low_inputs}


def prepare(case, seed):
    s = INPUTS[case["op"]](case, seed)
    s["case"] = case
    if not own:
        return s
    from paper_1911_11377_amd import ckksmi, lowbit, training

    ctx = s["ctx"] = ckksmi.Context(12, 3, 40, 1, 41, 1, device=0)

    def space(n):
        return torch.empty(max(16, n), dtype=torch.uint8, device=DEV)

    if case["op"] == "norm":
        none = {"none": None}
        p = s["plan"] = training.ResidualNorm(ctx, case["d"], TYPES[case["type"]], pre=none.get(case["pre"], case["pre"]), post=none.get(case["post"], case["post"]),
                                              gate=none.get(case["gate"], case["gate"]), weight_dtype=TYPES[case["weights"]], eps=EPS, residual_scale=RESIDUAL,
                                              block_scale=BLOCK_SCALE)
        s["out"] = {"r": torch.empty_like(s["x"])}
        if case["pre"] != "none":
            s["out"]["n"] = torch.empty_like(s["x"])
        if case["train"]:
            s["saved"], s["ws"] = space(p.saved_bytes(case["rows"])), space(p.workspace_bytes(case["rows"]))
            s["d"] = {"d" + k: torch.empty_like(s[k]) for k in ("x", "f", "gate", "pre_weight", "pre_bias", "post_weight", "post_bias") if k in s}
    elif case["op"] == "ortho":
        s["out"] = [torch.empty_like(u) for u in s["u"]]
        s["plan"] = training.Orthogonalise(ctx, s["u"], s["out"])
        s["ws"] = space(s["plan"].workspace_bytes())
    elif case["op"] == "muon":
        s["plan"] = training.Muon(ctx, s["p"], s["g"], s["m"], copies=s.get("copy"))
        s["ws"] = space(s["plan"].workspace_bytes())
    elif case["op"] == "product4":
        s["plan"] = lowbit.Product4(ctx, case["d_in"], case["d_out"], s["x"].dtype, case["group"])
        s["y"] = torch.empty(case["rows"], case["d_out"], dtype=s["x"].dtype, device=DEV)
    else:
        act = CUBICS.get(case["act"], case["act"])
        s["plan"] = lowbit.GatedFF4(ctx, case["d_in"], case["d_hidden"], case["d_out"], s["x"].dtype, act, case["group"])
        s["y"] = torch.empty(case["rows"], case["d_out"], dtype=s["x"].dtype, device=DEV)
        s["ws"] = space(s["plan"].workspace_bytes(case["rows"]))
    return s


# --------------------------------------------------------------------------- one pass
def run(s):
    op = s["case"]["op"]
    if not own:
        return {"norm": _norm_plain, "ortho": _ortho_plain, "muon": _muon_plain, "ff4": _ff4_plain, "product4": _product4_plain}[op](s)
    if op == "norm":
        w = {k: s[k] for k in ("gate", "pre_weight", "pre_bias", "post_weight", "post_bias") if k in s}
        s["plan"].forward(s["x"], s["f"], s["out"]["r"], s["out"].get("n"), saved=s.get("saved"), **w)
        if not s["case"]["train"]:
            return s["out"]
        s["plan"].backward(s["x"], s["f"], s["saved"], s["dr"], s.get("dn"), s["ws"], **s["d"], **w)
        return {**s["out"], **s["d"]}
    if op == "ortho":
        s["plan"].run(s["ws"], eps=NORM_EPS, steps=STEPS, coefficients=COEFFICIENTS)
        return s["out"]
    if op == "muon":
        s["plan"].step(LR, MOMENTUM, s["ws"], weight_decay=DECAY, nesterov=True, eps=NORM_EPS, steps=STEPS, coefficients=COEFFICIENTS)
        return {k: s[k] for k in ("p", "m", "copy") if k in s}
    if op == "product4":
        s["plan"].forward(s["x"], *s["w"], s["y"])
    else:
        s["plan"].forward(s["x"], s["gate"], s["up"], s["down"], s["y"], s["ws"])
    return {"y": s["y"]}


# --------------------------------------------------------------------------- plain forms
def _normed(v, kind):
    """v in units of its row's size (around its row's mean), and the inverse of that size"""
    if kind == "layer":
        v = v - v.sum(1, keepdim=True) / v.shape[1]
    inverse = 1.0 / torch.sqrt((v * v).sum(1, keepdim=True) / v.shape[1] + EPS)
    return v * inverse, inverse


def _norm_back(dy, hat, inverse, kind):
    """the gradient by v from the gradient by hat"""
    d = dy - hat * ((dy * hat).sum(1, keepdim=True) / hat.shape[1])
    if kind == "layer":
        d = d - dy.sum(1, keepdim=True) / hat.shape[1]
    return d * inverse


def _norm_plain(s):
    case = s["case"]
    v = {k: t.float() for k, t in s.items() if torch.is_tensor(t)}
    u = v["f"]
    if case["post"] != "none":
        u_hat, u_inverse = _normed(u, case["post"])
        u = u_hat * v["post_weight"] + v.get("post_bias", 0.0)
    gated = u * v["gate"] if "gate" in v else u
    r = v["x"] * RESIDUAL + gated * BLOCK_SCALE
    out = {"r": r}
    if case["pre"] != "none":
        r_hat, r_inverse = _normed(r, case["pre"])
        out["n"] = r_hat * v["pre_weight"] + v.get("pre_bias", 0.0)
    t = s["x"].dtype
    out = {k: o.to(t) for k, o in out.items()}
    if not case["train"]:
        return out
    dr, d = v["dr"], {}
    if case["pre"] != "none":
        d["pre_weight"] = (v["dn"] * r_hat).sum(0)
        d["pre_bias"] = v["dn"].sum(0)
        dr = dr + _norm_back(v["dn"] * v["pre_weight"], r_hat, r_inverse, case["pre"])
    d["x"] = dr * RESIDUAL
    du = dr * BLOCK_SCALE
    if "gate" in v:
        d["gate"] = du * u if case["gate"] == "element" else (du * u).sum(0)
        du = du * v["gate"]
    d["f"] = du
    if case["post"] != "none":
        d["post_weight"] = (du * u_hat).sum(0)
        d["post_bias"] = du.sum(0)
        d["f"] = _norm_back(du * v["post_weight"], u_hat, u_inverse, case["post"])
    return {**out, **{"d" + k: d[k].to(s[k].dtype) for k in ("x", "f", "gate", "pre_weight", "pre_bias", "post_weight", "post_bias") if k in s}}


def _direction(u):
    a, b, c = COEFFICIENTS
    tall = u.shape[0] > u.shape[1]
    x = u.t() if tall else u
    x = x * (1.0 / (torch.sqrt((x * x).sum()) + NORM_EPS))
    for _ in range(STEPS):
        y = x @ x.t()
        x = x * a + (y * b + (y @ y) * c) @ x
    return x.t() if tall else x


def _ortho_plain(s):
    return [_direction(u.float()).to(u.dtype) for u in s["u"]]


def _update_scale(rows, cols):
    return math.sqrt(max(1.0, rows / cols))


def _muon_plain(s):
    for i, p in enumerate(s["p"]):
        g = s["g"][i].float()
        m = s["m"][i] * MOMENTUM + g * (1.0 - MOMENTUM)
        q = p.float() * (1.0 - LR * DECAY) - _direction(m * MOMENTUM + g * (1.0 - MOMENTUM)) * (LR * _update_scale(*p.shape))
        s["m"][i].copy_(m)
        p.copy_(q)
        if "copy" in s:
            s["copy"][i].copy_(q)
    return {k: s[k] for k in ("p", "m", "copy") if k in s}


def _values(w, d_in, group):
    """[d_out][d_in] in 32 bits"""
    codes, scales = w
    c = torch.stack((codes & 15, codes >> 4), 2).reshape(codes.shape[0], -1)[:, :d_in].to(torch.int32)
    c = torch.where(c > 7, c - 16, c).float()
    return c * scales.float().repeat_interleave(group, 1)[:, :d_in]


def _act(g, name):
    if name in CUBICS:
        c0, c1, c2, c3 = CUBICS[name]
        return ((c3 * g + c2) * g + c1) * g + c0
    if name == "relu":
        return g * (g > 0).to(g.dtype)
    if name == "silu":
        return g / (1.0 + torch.exp(-g))
    return g * 0.5 * (1.0 + torch.erf(g * 0.5**0.5))


def _product4_plain(s):
    case = s["case"]
    return {"y": (s["x"].float() @ _values(s["w"], case["d_in"], case["group"]).t()).to(s["x"].dtype)}


def _ff4_plain(s):
    case, x = s["case"], s["x"].float()
    wg, wu = (_values(s[k], case["d_in"], case["group"]) for k in ("gate", "up"))
    wd = _values(s["down"], case["d_hidden"], case["group"])
    return {"y": ((_act(x @ wg.t(), case["act"]) * (x @ wu.t())) @ wd.t()).to(s["x"].dtype)}


# --------------------------------------------------------------------------- 64 bits
def exact(case, seed):
    s = INPUTS[case["op"]](case, seed)
    return {"norm": _norm_exact, "ortho": _ortho_exact, "muon": _muon_exact, "ff4": _low_exact, "product4": _low_exact}[case["op"]](case, s)


def _statistics(v, kind):
    """the row's mean (0 for rms) and the root of its mean square around that"""
    mean = v.mean(1, keepdim=True) if kind == "layer" else torch.zeros_like(v[:, :1])
    return mean, torch.sqrt(((v - mean) ** 2).mean(1, keepdim=True) + EPS)


def _norm_exact(case, s):
    at = {k: t.double() for k, t in s.items()}
    d, one, zero = case["d"], torch.ones((), dtype=torch.float64, device=DEV), torch.zeros((), dtype=torch.float64, device=DEV)
    w1, b1, w2, b2 = (at.get(k, e) for k, e in (("post_weight", one), ("post_bias", zero), ("pre_weight", one), ("pre_bias", zero)))
    gate, f = at.get("gate", one), at["f"]
    if case["post"] == "none":
        mean1, size1, norm1 = None, None, f
    else:
        mean1, size1 = _statistics(f, case["post"])
        norm1 = w1 * (f - mean1) / size1 + b1
    r = RESIDUAL * at["x"] + BLOCK_SCALE * gate * norm1
    out = {"r": r}
    if case["pre"] != "none":
        mean2, size2 = _statistics(r, case["pre"])
        out["n"] = w2 * (r - mean2) / size2 + b2
    if not case["train"]:
        return out

    def through(grad, v, mean, size, kind):
        """sum over j of grad_j times the derivative of (v_j - mean) / size by v_i"""
        centred = v - mean
        by_size = -(grad * centred).sum(1, keepdim=True) / size**2  # d/d size
        by_v = grad / size + by_size * centred / (d * size)
        return by_v - grad.sum(1, keepdim=True) / (d * size) if kind == "layer" else by_v

    dr = at["dr"]
    if case["pre"] != "none":
        out["dpre_weight"], out["dpre_bias"] = (at["dn"] * (r - mean2) / size2).sum(0), at["dn"].sum(0)
        dr = dr + through(at["dn"] * w2, r, mean2, size2, case["pre"])
    out["dx"] = RESIDUAL * dr
    dgate = BLOCK_SCALE * dr * norm1
    out["dgate"] = dgate if case["gate"] == "element" else dgate.sum(0)
    dnorm = BLOCK_SCALE * dr * gate
    if case["post"] == "none":
        out["df"] = dnorm
    else:
        out["dpost_weight"], out["dpost_bias"] = (dnorm * (f - mean1) / size1).sum(0), dnorm.sum(0)
        out["df"] = through(dnorm * w1, f, mean1, size1, case["post"])
    return {k: out[k] for k in ["r"] + (["n"] if "n" in out else []) + ["d" + k for k in ("x", "f", "gate", "pre_weight", "pre_bias", "post_weight", "post_bias") if k in s]}


def _series(v):
    """the odd polynomial of every step applied to v's singular values: v (a + b v^T v + c (v^T v)^2), from the side with fewer products"""
    a, b, c = COEFFICIENTS
    v = v / (torch.linalg.norm(v) + NORM_EPS)
    for _ in range(STEPS):
        if v.shape[0] >= v.shape[1]:
            k = torch.matmul(v.transpose(0, 1).contiguous(), v)
            v = a * v + torch.matmul(v, b * k + c * torch.matmul(k, k))
        else:
            k = torch.matmul(v, v.transpose(0, 1).contiguous())
            v = a * v + torch.matmul(b * k + c * torch.matmul(k, k), v)
    return v


def _ortho_exact(case, s):
    return [_series(u.double()) for u in s["u"]]


def _muon_exact(case, s):
    out = {k: [] for k in ("p", "m", "copy") if k in s}
    for p, g, m in zip(s["p"], s["g"], s["m"]):
        m = MOMENTUM * m.double() + (1 - MOMENTUM) * g.double()
        o = _series(MOMENTUM * m + (1 - MOMENTUM) * g.double())
        q = p.double() - LR * DECAY * p.double() - LR * max(1.0, p.shape[0] / p.shape[1]) ** 0.5 * o
        for k, v in (("p", q), ("m", m), ("copy", q)):
            if k in out:
                out[k].append(v)
    return out


def _exact_weights(w, d_in, group):
    low, high = torch.remainder(w[0].double(), 16.0), torch.floor(w[0].double() / 16.0)
    c = torch.empty(w[0].shape[0], 2 * w[0].shape[1], dtype=torch.float64, device=DEV)
    c[:, 0::2], c[:, 1::2] = low, high
    c = torch.where(c >= 8.0, c - 16.0, c)[:, :d_in]
    return c * w[1].double()[:, torch.arange(d_in, device=DEV) // group]


def _low_exact(case, s):
    x = s["x"].double()
    if case["op"] == "product4":
        return {"y": torch.matmul(x, _exact_weights(s["w"], case["d_in"], case["group"]).transpose(0, 1))}
    g, u = (torch.matmul(x, _exact_weights(s[k], case["d_in"], case["group"]).transpose(0, 1)) for k in ("gate", "up"))
    name = case["act"]
    if name in CUBICS:
        a = sum(CUBICS[name][k] * g**k for k in range(4))
    else:
        a = torch.clamp(g, min=0.0) if name == "relu" else g * torch.sigmoid(g) if name == "silu" else g * torch.special.ndtr(g)
    return {"y": torch.matmul(a * u, _exact_weights(s["down"], case["d_hidden"], case["group"]).transpose(0, 1))}


# --------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    size = {"f32": 4, "bf16": 2, "f16": 2}
    e = size[case["type"]]
    if case["op"] == "norm":
        M, d, ew = case["rows"], case["d"], size[case["weights"]]
        vectors = sum({"none": 0, "rms": 1, "layer": 2}[case[k]] for k in ("pre", "post")) + (case["gate"] == "channel")
        rows = 3 + (case["pre"] != "none") + (case["gate"] == "element")  # x, f, gate; r, n
        flops = 20.0
        if case["train"]:
            rows += 5 + (case["pre"] != "none") + 2 * (case["gate"] == "element")  # x, f, dr, dn, gate; dx, df, dgate
            vectors *= 3
            flops += 50.0
        return {"bytes": M * d * e * rows + vectors * d * ew, "flops": flops * M * d}
    if case["op"] in ("ortho", "muon"):
        n = sum(r * c for r, c in _shapes(case))
        if case["op"] == "ortho":
            b = 2 * e * n
        else:
            b = n * (2 * e + size[case["grads"]] + 8 + (2 if case["copy"] else 0))
        return {"bytes": b, "flops": sum(_operations(*s) for s in _shapes(case))}

    def matrix(d_out, d_in):
        return d_out * (-(-d_in // 32) * 16 + -(-d_in // case["group"]) * e)

    M, K, O = case["rows"], case["d_in"], case["d_out"]
    if case["op"] == "product4":
        return {"bytes": matrix(O, K) + e * M * (K + O), "flops": 2.0 * M * K * O}
    H = case["d_hidden"]
    return {"bytes": 2 * matrix(H, K) + matrix(O, H) + e * M * (K + O), "flops": 2.0 * M * H * (2 * K + O)}
