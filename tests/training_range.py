"""f32 gradients of 16-bit operands over the range of f32: inputs, what 64 bits give and how far f32 operands would be from it."""
import math

import torch

from paper_1911_11377_amd import training

U32 = 2.0**-24
# (scale of x, scale of dy): a mean loss's gradients from a batch of thousand rows down to f16's smallest numbers, and products beyond f16's largest
SCALES = [(1.0, 1.0), (1.0, 2.0**-10), (1.0, 2.0**-17), (1.0, 2.0**-22), (2.0**-8, 2.0**-17), (8.0, 300.0)]


def check(ctx, device, place, rows, dtype, scales, seed=1, d_in=8, d_hidden=16, d_out=8):
    """the weights' gradients of a squared gate in f32.  g, u and dh are sums of n products in 32 bits (n + 8 roundings of the sum of
    magnitudes at most), a = g^2 and the products after it a few more; dg, du and h enter the gradients in 24 bits, as sums of
    three bf16 parts each half a place of 8 bits, what is left out of five products being 2^-24 of the whole: at most 5 rows + 8 + 4 roundings"""
    g = torch.Generator().manual_seed(seed)

    def normal(shape, scale):
        return place((torch.randn(shape, generator=g) * scale).to(dtype).to(device))

    x, dy = normal((rows, d_in), scales[0]), normal((rows, d_out), scales[1])
    wg, wu, wd = normal((d_hidden, d_in), d_in**-0.5), normal((d_hidden, d_in), d_in**-0.5), normal((d_out, d_hidden), d_hidden**-0.5)
    ff = training.GatedFF(ctx, d_in, d_hidden, d_out, dtype, "square", torch.float32)
    y, dx = place(torch.zeros(rows, d_out, dtype=dtype, device=device)), place(torch.zeros(rows, d_in, dtype=dtype, device=device))
    dw = [place(torch.full(w.shape, math.nan, device=device)) for w in (wg, wu, wd)]
    ws, saved = [place(torch.full((max(16, n),), 255, dtype=torch.uint8, device=device)) for n in (ff.workspace_bytes(rows, backward=True), ff.saved_bytes(rows))]
    ff.forward(x, wg, wu, wd, y, ws, saved=saved)
    assert bool(torch.isfinite(y).all())
    ff.backward(x, wg, wu, wd, saved, dy, dx, *dw, ws)
    x, dy, wg, wu, wd = (t.double().cpu() for t in (x, dy, wg, wu, wd))

    def gradients(x, dy, wg, wu, wd):
        g, u, dh = x @ wg.t(), x @ wu.t(), dy @ wd
        dg, du = dh * u * 2 * g, dh * g * g
        return dg.t() @ x, du.t() @ x, dy.t() @ (g * g * u)

    want = gradients(x, dy, wg, wu, wd)
    magnitudes = gradients(*(t.abs() for t in (x, dy, wg, wu, wd)))
    roundings = (d_out + 8) + 3 * (d_in + 8) + 8 + (5 * rows + 8) + 4
    for name, got, v, mag in zip(("dwg", "dwu", "dwd"), dw, want, magnitudes):
        off = (got.double().cpu() - v).abs()
        assert bool((off <= 1.25 * roundings * U32 * mag).all()), (name, float((off / mag).max()), 1.25 * roundings * U32)
