"""64-bit references of the training operators and bounds of the kernels' rounding errors, written from the formulas."""
import math

import numpy as np
import torch

ROUND = {torch.float32: 2.0**-24, torch.bfloat16: 2.0**-8, torch.float16: 2.0**-11}  # unit roundoff
TINY = {torch.float32: 2.0**-149, torch.bfloat16: 2.0**-133, torch.float16: 2.0**-25}  # half the smallest step, or more
U32 = 2.0**-24


def act_parts(g, act):
    """act, act', act'' and the sum of the magnitudes that act is made of, at g (64 bits)"""
    if not isinstance(act, str):
        c = [float(np.float32(v)) for v in act]
        p = [g**k for k in range(4)]
        a = sum(c[k] * p[k] for k in range(4))
        d1 = c[1] + 2 * c[2] * g + 3 * c[3] * p[2]
        d2 = 2 * c[2] + 6 * c[3] * g
        return a, d1, d2, sum(abs(c[k]) * p[k].abs() for k in range(4)) + g.abs() * (abs(c[1]) + 2 * abs(c[2] * g) + 3 * abs(c[3]) * p[2])
    if act == "relu":
        on = (g > 0).double()
        return g * on, on, torch.zeros_like(g), g.abs()
    if act == "silu":
        q = torch.sigmoid(g)
        return g * q, q + g * q * (1 - q), q * (1 - q) * (2 + g * (1 - 2 * q)), g.abs() * (1 + g.abs())
    q, phi = torch.special.ndtr(g), torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
    return g * q, q + g * phi, phi * (2 - g * g), g.abs() * (1 + g * g)


def _rounded(v, dtype):
    return ROUND[dtype] * v.abs() + TINY[dtype]


def block(x, wg, wu, wd, act, dy=None, grad_dtype=None):
    """{name: (value, bound of |kernel - value|)} of the block's results.  The bound follows the kernel's order of steps to first
    order (times 1.25 for the rest): sums of n products in 32 bits lose at most (n + 8) 2^-24 of the sum of magnitudes in any
    order, h, dg and du are rounded to the element type (with f32 gradients of 16-bit operands to the sum of two f16 or three bf16
    where they enter the weights' gradients), act(g) and u act'(g) to 17 bits between the passes (f32 gradients: 24), results to their type; an activation loses
    at most 32 x 2^-24 of the magnitudes it is made of."""
    dtype = x.dtype
    grad_dtype = grad_dtype or dtype
    x, wg, wu, wd = (t.double() for t in (x, wg, wu, wd))
    M, K = x.shape
    H, O = wg.shape[0], wd.shape[0]
    g, u = x @ wg.t().contiguous(), x @ wu.t().contiguous()
    eg = (K + 8) * U32 * (x.abs() @ wg.abs().t().contiguous())
    eu = (K + 8) * U32 * (x.abs() @ wu.abs().t().contiguous())
    a, d1, d2, mag = act_parts(g, act)
    d1_near = d1.abs() + d2.abs() * eg
    if act == "relu":
        d1_near = torch.maximum(d1_near, (g.abs() <= eg).double())
    ea = d1_near * eg + 32 * U32 * mag
    h = a * u
    fine = dtype != torch.float32 and grad_dtype == torch.float32
    parts = (3 if dtype == torch.bfloat16 else 2) if fine else 1

    def paired(v):
        return ROUND[dtype] ** parts * v.abs() + TINY[dtype]

    eh0 = ea * u.abs() + a.abs() * eu + ea * eu + 4 * U32 * h.abs()
    eh = eh0 + _rounded(h, dtype)
    y = h @ wd.t().contiguous()
    wda = wd.abs()
    ey = eh @ wda.t().contiguous() + (H + 8) * U32 * (h.abs() @ wda.t().contiguous())
    out = {"y": (y, 1.25 * (ey + _rounded(y, dtype)))}
    if dy is None:
        return out
    dy = dy.double()
    dh = dy @ wd
    edh = (O + 8) * U32 * (dy.abs() @ wda)
    ed1 = d2.abs() * eg + 32 * U32 * (1 + mag)
    if not isinstance(act, str):
        ed1 = ed1 + 6 * abs(float(act[3])) * eg * eg
    if act == "relu":
        ed1 = ed1 + (g.abs() <= eg).double()
    keep = 2.0**-17 if dtype != torch.float32 and not fine else U32
    ea_kept = ea + keep * a.abs()
    ep_kept = ed1 * u.abs() + d1.abs() * eu + ed1 * eu + (keep + 2 * U32) * (u * d1).abs()
    dg, du = dh * u * d1, dh * a
    edg0 = edh * (u * d1).abs() + dh.abs() * ep_kept + 2 * U32 * dg.abs()
    edu0 = edh * a.abs() + dh.abs() * ea_kept + 2 * U32 * du.abs()
    edg, edu = edg0 + _rounded(dg, dtype), edu0 + _rounded(du, dtype)
    dx = dg @ wg + du @ wu
    edx = edg @ wg.abs() + edu @ wu.abs() + (2 * H + 8) * U32 * (dg.abs() @ wg.abs() + du.abs() @ wu.abs())
    out["dx"] = (dx, 1.25 * (edx + _rounded(dx, dtype)))

    def weights(l, el, r, er):
        lt, elt = l.t().contiguous(), el.t().contiguous()
        v = lt @ r
        e = elt @ r.abs() + (parts * M + 8) * U32 * (lt.abs() @ r.abs())
        if er is not None:
            e = e + lt.abs() @ er
        return v, 1.25 * (e + _rounded(v, grad_dtype))

    out["dwg"] = weights(dg, edg0 + paired(dg), x, None)
    out["dwu"] = weights(du, edu0 + paired(du), x, None)
    out["dwd"] = weights(dy, torch.zeros_like(dy), h, eh0 + paired(h))
    return out


# ---------------------------------------------------------------- AdamW, one operation at a time in 32 bits (numpy rounds each)
M32 = 0xFFFFFFFF


def mix(h):
    h = np.asarray(h, dtype=np.uint64) & np.uint64(M32)
    h ^= h >> np.uint64(16)
    h = (h * np.uint64(0x6A09E667)) & np.uint64(M32)
    h ^= h >> np.uint64(15)
    h = (h * np.uint64(0xBB67AE85)) & np.uint64(M32)
    return h ^ (h >> np.uint64(16))


def random_words(seed, tensor, n):
    key = mix(mix(seed & M32) + np.uint64((seed >> 32) & M32))
    key = mix(key + np.uint64(tensor))
    i = np.arange(n, dtype=np.uint64)
    b, j = i >> np.uint64(8), i & np.uint64(255)
    bkey = mix(mix(key + (b & np.uint64(M32))) + (b >> np.uint64(32)))
    return mix(bkey + j * np.uint64(0x9E3779B9))


def code_table(fraction):
    """what the codes without sign stand for, in units"""
    one = 1 << fraction
    return np.array([c if c < one else (one + (c & (one - 1))) << ((c >> fraction) - 1) for c in range(16 * one)], dtype=np.float64)


def read_codes(codes, units, fraction):
    """float32 values of 8-bit states"""
    t = code_table(fraction).astype(np.float32)
    u = np.repeat(np.asarray(units, dtype=np.float32), 256)[: len(codes)]
    if fraction == 3:
        return np.where(codes & 128, -t[codes & 127], t[codes & 127]) * u
    return t[codes] * u


def write_codes(x, rnd16, fraction):
    """codes and units of float32 values (finite): the largest code whose value is below |x| in units plus a random part, 16 bits, of the
    gap above it"""
    n, blocks = len(x), -(-len(x) // 256)
    t = code_table(fraction)
    pad = np.zeros(blocks * 256, dtype=np.float32)
    pad[:n] = np.abs(x)
    with np.errstate(all="ignore"):
        units = pad.reshape(blocks, 256).max(1) * np.float32(1.0 / t[-1])
        units = np.where(units >= np.float32(1e-36), units, np.float32(0))
        inv = np.where(units > 0, np.float32(1) / units, np.float32(0)).astype(np.float32)
    z = (pad.reshape(blocks, 256) * inv[:, None]).reshape(-1)[:n].astype(np.float64)
    # below the smallest doubling the kernel adds it to z in 32 bits before it cuts
    one = float(1 << fraction)
    z = np.where(z < one, (z.astype(np.float32) + np.float32(one)).astype(np.float64) - one, z)
    c = np.searchsorted(t, np.minimum(z, t[-1]), side="right") - 1
    gap = np.where(c + 1 < len(t), t[np.minimum(c + 1, len(t) - 1)] - t[c], 1.0)
    up = (z - t[c]) / gap + rnd16.astype(np.float64) / 65536.0 >= 1.0
    c = np.minimum(c + up, len(t) - 1)
    if fraction == 4:
        c = np.where((z > 0) & (c == 0), 1, c)
    c = c.astype(np.uint8)
    if fraction == 3:
        c = np.where(x < 0, c | 128, c).astype(np.uint8)
    return c, units.astype(np.float32)


def adamw_f32(p, g, m, v, lr, betas, eps, wd, step, scale=1.0):
    """p, m, v after a step on float32 arrays"""
    f = np.float32
    b1, b2 = betas
    with np.errstate(all="ignore"):
        g = (g * f(scale)).astype(f)
        m = (m * f(b1)) + (g * f(1.0 - b1))
        v = (v * f(b2)) + (g * g) * f(1.0 - b2)
        p = p * f(1.0 - lr * wd) - (m / (np.sqrt(v) * f(1.0 / math.sqrt(1.0 - b2**step)) + f(eps))) * f(lr / (1.0 - b1**step))
    return p, m, v
