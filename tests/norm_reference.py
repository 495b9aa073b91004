"""64-bit reference of the norms around a block with bounds of the kernels' rounding errors, written from the formulas, and the comparison
that the tests on the CPU stand-in and on the GPU share."""
import math

import torch

from paper_1911_11377_amd import training

ROUND = {torch.float32: 2.0**-24, torch.bfloat16: 2.0**-8, torch.float16: 2.0**-11}  # unit roundoff
TINY = {torch.float32: 2.0**-149, torch.bfloat16: 2.0**-133, torch.float16: 2.0**-25}  # half the smallest step, or more
U = 2.0**-24


def _norm(v, e_v, kind, w, b, eps):
    """N(v), h, s and bounds of the errors of N(v), h and (relative) s, for v known to e_v.  A sum over a row of d has at most d / 512 + 40
    additions one behind the other: 16 elements of a thread, 10 levels of lanes, 16 waves, or rounds of 512 threads"""
    d = v.shape[1]
    depth = d / 512 + 40
    mean = v.mean(1, keepdim=True) if kind == "layer" else torch.zeros_like(v[:, :1])
    e_mean = e_v.mean(1, keepdim=True) + (depth + 2) * U * v.abs().mean(1, keepdim=True) if kind == "layer" else torch.zeros_like(mean)
    c = v - mean
    s = 1.0 / torch.sqrt((c * c).mean(1, keepdim=True) + eps)
    h = c * s
    e_c = e_v + e_mean + U * c.abs()
    rel_s = s * (h.abs() * e_c).mean(1, keepdim=True) + (depth / 2 + 8) * U
    e_h = s * e_c + h.abs() * (rel_s + 2 * U)
    y = h * w + b
    return y, h, s, w.abs() * e_h + U * (h * w).abs() + U * y.abs(), e_h, rel_s


def _back(dy, e_dy, w, h, e_h, s, rel_s, kind):
    """gradient by v of h w + b and a bound of its error"""
    d = h.shape[1]
    depth = d / 512 + 40
    g, e_g = dy * w, e_dy * w.abs() + U * (dy * w).abs()
    m1 = (g * h).mean(1, keepdim=True)
    e_m1 = (g.abs() * e_h + e_g * h.abs()).mean(1, keepdim=True) + (depth + 3) * U * (g * h).abs().mean(1, keepdim=True)
    m0, e_m0 = torch.zeros_like(m1), torch.zeros_like(m1)
    if kind == "layer":
        m0 = g.mean(1, keepdim=True)
        e_m0 = e_g.mean(1, keepdim=True) + (depth + 3) * U * g.abs().mean(1, keepdim=True)
    t = g - m0 - h * m1
    e_t = e_g + e_m0 + h.abs() * e_m1 + m1.abs() * e_h + 3 * U * (g.abs() + m0.abs() + (h * m1).abs())
    return t * s, s * e_t + (t * s).abs() * (rel_s + 2 * U)


def residual_norm(x, f, gate, w, pre, post, eps, a, b, dr=None, dn=None):
    """{name: (value, bound before the last rounding)}; w: {"post_weight": .., ..}, missing ones are ones and zeros"""
    one, zero = torch.ones(1, x.shape[1], dtype=torch.float64), torch.zeros(1, x.shape[1], dtype=torch.float64)
    D = lambda t: t.double().cpu()  # noqa: E731
    x, dr, dn = D(x), D(dr) if dr is not None else torch.zeros_like(D(x)), D(dn) if dn is not None else torch.zeros_like(D(x))
    w = {k: D(w[k])[None] if w.get(k) is not None else (one if k.endswith("weight") else zero) for k in ("post_weight", "post_bias", "pre_weight", "pre_bias")}
    out, nothing = {}, torch.zeros_like(x)
    M = x.shape[0]
    if f is None:
        r, e_r = x, nothing
    else:
        f, e_y = D(f), nothing
        y = f
        if post:
            y, h1, s1, e_y, e_h1, rel1 = _norm(f, nothing, post, w["post_weight"], w["post_bias"], eps)
        g = D(gate).expand_as(x) if gate is not None else one.expand_as(x)
        e_u = e_y * g.abs() + U * (y * g).abs()
        r = a * x + b * y * g
        e_r = abs(b) * e_u + U * ((a * x).abs() + (b * y * g).abs() + r.abs())
        out["r"] = (r, e_r)
    e_dr, e_r_in = nothing, e_r
    if pre:
        n, h2, s2, e_n, e_h2, rel2 = _norm(r, e_r_in, pre, w["pre_weight"], w["pre_bias"], eps)
        out["n"] = (n, e_n)
        back, e_back = _back(dn, nothing, w["pre_weight"], h2, e_h2, s2, rel2, pre)
        out["dpre_weight"] = _columns(dn * h2, dn.abs() * e_h2)
        out["dpre_bias"] = _columns(dn, nothing)
        dr, e_dr = dr + back, e_back + U * (dr + back).abs()
    out["dx"] = (dr, e_dr) if f is None else (a * dr, abs(a) * e_dr + U * (a * dr).abs())
    if f is None:
        return out
    dg = b * dr * y
    e_dg = (b * y).abs() * e_dr + (b * dr).abs() * e_y + 2 * U * dg.abs()
    out["dgate"] = (dg, e_dg) if gate is not None and gate.dim() == 2 else _columns(dg, e_dg)
    dy = b * dr * g
    e_dy = (b * g).abs() * e_dr + 2 * U * dy.abs()
    out["df"] = (dy, e_dy)
    if post:
        out["dpost_weight"], out["dpost_bias"] = _columns(dy * h1, dy.abs() * e_h1 + e_dy * h1.abs()), _columns(dy, e_dy)
        out["df"] = _back(dy, e_dy, w["post_weight"], h1, e_h1, s1, rel1, post)
    assert M
    return out


def _columns(v, e):
    """sums over the rows: at most as many additions one behind the other as there are rows, and the groups'"""
    return v.sum(0), e.sum(0) + (v.shape[0] + 2) * U * v.abs().sum(0)


def within(got, want, dtype, name, before=None):
    v, bound = want
    if before is not None:
        v, bound = v + before, bound + U * (v + before).abs()
    bound = 1.25 * bound + (0 if dtype == torch.float32 else ROUND[dtype] * (v.abs() + 1.25 * bound)) + U * v.abs() + TINY[dtype]
    off = (got.double().cpu() - v).abs()
    assert bool((off <= bound).all()), (name, float((off - bound).max()), float((off / bound).max()))


class Case:
    """tensors of one call, made from a seed; `place` puts a tensor where it has to lie"""

    def __init__(self, rows, d, dtype, pre, post, gate, weight_dtype=None, with_f=True, lead=0, seed=1, weights=True, device="cpu", place=None):
        place = place or (lambda t: t)
        self.rows, self.d, self.dtype, self.pre, self.post, self.gate_kind = rows, d, dtype, pre, post, gate
        self.wt = weight_dtype or dtype
        gen = torch.Generator().manual_seed(seed)

        def normal(*shape, scale=1.0, at=0.0, t=dtype):
            return torch.randn(shape, generator=gen).mul(scale).add(at).to(t)

        def rowed(t):  # rows `lead` elements further apart than they are long
            if not lead:
                return place(t.to(device))
            wide = torch.full((rows, d + lead), math.nan, dtype=t.dtype)
            wide[:, :d] = t
            return place(wide.to(device))[:, :d]

        self.rowed = rowed
        self.vector = lambda t: place(t.to(device))
        self.x = rowed((torch.randn((rows, d), generator=gen) * torch.exp(torch.randn(d, generator=gen) * 0.7) + 0.3).to(dtype))
        self.f = rowed(normal(rows, d, scale=0.5, at=-0.2)) if with_f else None
        self.w = {}
        for k, kind in (("post", post), ("pre", pre)):
            if kind and weights and (with_f or k == "pre"):
                self.w[k + "_weight"] = self.vector(normal(d, scale=0.3, at=1.0, t=self.wt))
                if kind == "layer":
                    self.w[k + "_bias"] = self.vector(normal(d, scale=0.2, t=self.wt))
        self.gate = None
        if gate and with_f:
            self.gate = self.vector(normal(d, scale=0.5, t=self.wt)) if gate == "channel" else rowed(normal(rows, d, scale=0.5))
        self.dr, self.dn = rowed(normal(rows, d)), rowed(normal(rows, d)) if pre else None
        self.r = rowed(torch.full((rows, d), math.nan, dtype=dtype)) if with_f else None
        self.n = rowed(torch.full((rows, d), math.nan, dtype=dtype)) if pre else None

    def gradients(self, fill=math.nan):
        """buffers for the gradients of all that the call has"""
        out = {"dx": self.rowed(torch.full((self.rows, self.d), math.nan, dtype=self.dtype))}
        if self.f is not None:
            out["df"] = self.rowed(torch.full((self.rows, self.d), math.nan, dtype=self.dtype))
        if self.gate is not None:
            out["dgate"] = self.rowed(torch.full((self.rows, self.d), math.nan, dtype=self.dtype)) if self.gate.dim() == 2 else self.vector(torch.full((self.d,), fill, dtype=self.wt))
        for k in self.w:
            out["d" + k] = self.vector(torch.full((self.d,), fill, dtype=self.wt))
        return out


def check(ctx, case, place=None, device="cpu", eps=1e-5, a=0.9, b=-0.7, accumulate=False, dr=True, dn=True):
    """forward and backward of a case against 64 bits"""
    place = place or (lambda t: t)
    c = case
    plan = training.ResidualNorm(ctx, c.d, c.dtype, pre=c.pre, post=c.post, gate=c.gate_kind, weight_dtype=c.wt, eps=eps, residual_scale=a, block_scale=b)

    def room(n):
        return place(torch.full((max(n, 16),), 255, dtype=torch.uint8).to(device))

    saved = room(plan.saved_bytes(c.rows))
    plan.forward(c.x, c.f, c.r, c.n, gate=c.gate, saved=saved, **c.w)
    first = {k: t.clone() for k, t in (("r", c.r), ("n", c.n)) if t is not None}
    plan.forward(c.x, c.f, c.r, c.n, gate=c.gate, **c.w)  # nothing kept: the same bits
    for k, t in (("r", c.r), ("n", c.n)):
        assert t is None or torch.equal(t, first[k]), k
    dr, dn = c.dr if dr else None, c.dn if dn else None
    start = 0.5 if accumulate else math.nan
    grads = c.gradients(start)
    ws = room(plan.workspace_bytes(c.rows))
    plan.backward(c.x, c.f, saved, dr, dn, ws, gate=c.gate, accumulate=accumulate, **grads, **c.w)
    want = residual_norm(c.x, c.f, c.gate, c.w, c.pre, c.post, float(torch.tensor(eps, dtype=torch.float32)), float(torch.tensor(a, dtype=torch.float32)),
                         float(torch.tensor(b, dtype=torch.float32)), dr, dn)
    for k, t in (("r", c.r), ("n", c.n)):
        if t is not None:
            within(t, want[k], c.dtype, k)
    for k, t in grads.items():
        within(t, want[k], t.dtype, k, before=start if accumulate and t.dim() == 1 else None)
    again = c.gradients(start)
    plan.backward(c.x, c.f, saved, dr, dn, room(plan.workspace_bytes(c.rows)), gate=c.gate, accumulate=accumulate, **again, **c.w)
    for k in grads:
        assert torch.equal(again[k], grads[k]), ("a second call has other bits", k)


F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
# rows, d: one element to several pieces a thread, whole and ragged, groups within a wave and over waves, groups without a row
SIZES = [(1, 1), (5, 7), (33, 8), (70, 65), (3, 130), (9, 256), (6, 300), (2, 515), (5, 1021), (3, 1100), (2, 2056), (1, 4100)]
KINDS = [("rms", "rms", None), ("layer", "layer", "channel"), ("rms", None, "element"), (None, "layer", "element"), ("layer", "rms", None), (None, None, "channel"), (None, "rms", None)]
