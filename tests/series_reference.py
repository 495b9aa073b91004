"""Orthogonalised directions in 64 bits, and how far rounding takes them: the polynomials raise errors of weak directions by up to
3.4^steps, so a bound from norms alone says nothing beyond a few rows.  `rounded` takes the steps in 64 bits with every value that the kernels
hold rounded as they hold it, and every sum moved at random by what sums in 32 bits lose; its distance from the exact
direction, over some seeds, is what the kernels are allowed twice."""
import math

import numpy as np
import torch

COEFFICIENTS = (3.4445, -4.7750, 2.0315)
ROUND = {torch.float32: 2.0**-24, torch.bfloat16: 2.0**-8, torch.float16: 2.0**-11}
TINY = {torch.float32: 2.0**-149, torch.bfloat16: 2.0**-133, torch.float16: 2.0**-25}


def start(u, eps):
    size = float(torch.linalg.norm(u)) + eps
    return u / size if size else u


def exact(u, eps=1e-7, steps=5, coefficients=COEFFICIENTS):
    """from the definition: the polynomial of the singular values"""
    a, b, c = coefficients
    x = start(u.double().cpu(), eps)
    for _ in range(steps):
        k = x @ x.t() if x.shape[0] <= x.shape[1] else x.t() @ x
        p = b * k + c * (k @ k)
        x = a * x + (p @ x if x.shape[0] <= x.shape[1] else x @ p)
    return x


def _upper(x):
    return x.to(torch.float16).double()


def _two(x):
    return _upper(x) + _upper(x - _upper(x))


def rounded(u, parts, seed, eps=1e-7, steps=5, coefficients=COEFFICIENTS):
    a, b, c = coefficients
    gen = torch.Generator().manual_seed(seed)
    x = u.double().cpu()
    tall = x.shape[0] > x.shape[1]
    if tall:
        x = x.t()
    m, n = x.shape
    S = 2.0 ** min(14, round(0.5 * math.log2(m * n)))
    held = _upper if parts == 1 else _two

    def product(p, q):
        k = p.shape[1]
        loss = 2.0**-24 * math.sqrt(k / 32 * (1 if parts == 1 else 3) + 12)
        return p @ q + loss * (torch.rand((m, q.shape[1]), generator=gen, dtype=torch.float64) * 2 - 1) * (p.abs() @ q.abs())

    def near(v):  # some operations in 32 bits
        return v * (1 + 4 * 2.0**-24 * (torch.rand(v.shape, generator=gen, dtype=torch.float64) * 2 - 1))

    off = 1 - torch.eye(m, dtype=torch.float64)
    x = _two(near(start(x, eps) * S))
    for _ in range(steps):
        h = held(x)
        k = product(h, h.t()) / S**2
        k = torch.tril(k) + torch.tril(k, -1).t()
        d, o = near(k.diagonal()), held(near(k * off * 256)) / 256
        square = product(o, o)
        square = torch.tril(square) + torch.tril(square, -1).t()
        rest = near(b * o + c * ((d[:, None] + d[None, :]) * o + square))
        e = near(a + b * d + c * (d * d + square.diagonal()))
        x = near(e[:, None] * x + product(held(rest * off * 256) / 256, h))
        x = _two(x)
    x = x / S
    return x.t() if tall else x


def allowed(u, parts, eps=1e-7, steps=5, coefficients=COEFFICIENTS):
    """the exact direction, and bounds of an error's Frobenius norm and of its largest element"""
    v = exact(u, eps, steps, coefficients)
    off = [rounded(u, parts, s, eps, steps, coefficients) - v for s in range(3)]
    return v, 2 * max(float(torch.linalg.norm(o)) for o in off), 3 * max(float(o.abs().max()) for o in off)


def check(got, u, parts, **kw):
    v, norm, most = allowed(u, parts, **kw)
    d = (got.double().cpu() - v).abs()
    r, t = ROUND[got.dtype], TINY[got.dtype]
    assert bool(torch.isfinite(got).all())
    last = r * v.abs() + t + r * most
    assert float(torch.linalg.norm(d)) <= norm + float(torch.linalg.norm(last)), (float(torch.linalg.norm(d)), norm, float(torch.linalg.norm(last)))
    assert bool((d <= most + last).all()), (float((d - last).max()), most)


def momentum(m, g, beta, grad_scale, nesterov):
    """m after the step and what is orthogonalised, one 32-bit operation at a time"""
    f = np.float32
    m, g = m.float().cpu().numpy(), g.float().cpu().numpy() * f(grad_scale)
    m = m * f(beta) + g * f(1.0 - beta)
    return torch.from_numpy(m), torch.from_numpy(m * f(beta) + g * f(1.0 - beta)) if nesterov else torch.from_numpy(m)


def check_step(p, p0, u, parts, lr, scale, decay, copy=None):
    """parameters after a step of lr * scale along the direction of u"""
    v, _, most = allowed(u, parts)
    keep = float(np.float32(1.0 - lr * decay))
    size = abs(lr * scale)
    want = p0.double().cpu() * keep - lr * scale * v
    bound = size * most + 3 * 2.0**-24 * (p0.double().cpu().abs() + size * v.abs())
    for t in (p, copy):
        if t is not None:
            off = (t.double().cpu() - want).abs()
            last = 0 if t.dtype == torch.float32 else ROUND[t.dtype] * (want.abs() + bound) + TINY[t.dtype]
            assert bool((off <= bound + last).all()), float((off - bound - last).max())


def matrix(rows, cols, seed, kind="normal", dtype=torch.float32, scale=1.0):
    """normal numbers; a few strong directions above noise; directions that fall off over five decades; rank 3 and next to nothing else"""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((rows, cols), generator=g, dtype=torch.float64)
    if kind == "strong":
        x = 0.3 * x + sum(0.8 * 0.7**k * torch.randn((rows, 1), generator=g, dtype=torch.float64) * torch.randn((1, cols), generator=g, dtype=torch.float64) for k in range(4))
    elif kind == "falling":
        x = x * torch.logspace(0, -5, rows, dtype=torch.float64)[:, None]
    elif kind == "rank3":
        x = torch.randn((rows, 3), generator=g, dtype=torch.float64) @ torch.randn((3, cols), generator=g, dtype=torch.float64) + 1e-3 * x
    return (x * scale).to(dtype)


F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
# one element, rows and columns, sides that are multiples of nothing, of 8, beyond one tile of 32 and of 128
SIZES = [(1, 1), (1, 40), (37, 1), (2, 9), (8, 8), (5, 31), (33, 16), (40, 64), (70, 41), (130, 67), (20, 300)]
