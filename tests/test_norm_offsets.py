"""Layer norms of rows whose numbers are nearly equal and far from zero; on the CPU stand-in and on the GPU."""
import math

import pytest
import torch

import train_emu_support as emu
from paper_1911_11377_amd import ckksmi, training

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


@pytest.fixture(scope="module", params=["stand-in", pytest.param("gpu", marks=pytest.mark.gpu)])
def where(request):
    if request.param == "gpu":
        c = ckksmi.Context(4, 3, 20, 1, 21, 1, device=0)
        yield c, "cuda:0"
        c.close()
        return
    if not emu.available:
        pytest.skip("no host compiler with 16-bit float types")
    c = emu.EmuContext()
    yield c, "cpu"
    assert c.errors() == 0
    c.close()


# rows that a group of 8 .. 1024 threads holds, and longer ones
WIDTHS = [7, 100, 333, 1021, 3000, 9000, 17000]
VALUES = [0.1, 123.456, 12345.678, -1e6]


@pytest.mark.parametrize("d", WIDTHS)
def test_a_row_of_equal_numbers_has_nothing_left(where, d):
    """both norms; the sum of what the mean leaves is off by less than 2^-24 (d + 2) of itself, so the mean is rounded to the number itself"""
    ctx, device = where
    for dtype in (F32, BF16, F16):
        plan = training.ResidualNorm(ctx, d, dtype, pre="layer", post="layer", weight_dtype=F32)
        b1, b2 = torch.zeros(d, device=device), torch.linspace(-1, 1, d).to(device)
        x = torch.tensor([v for v in VALUES if abs(v) < torch.finfo(dtype).max])[:, None].expand(-1, d).to(dtype).contiguous().to(device)
        f = (-x).contiguous()
        r, n = torch.full_like(x, math.nan), torch.full_like(x, math.nan)
        plan.forward(x, f, r, n, post_bias=b1, pre_bias=b2)
        assert torch.equal(r, x)  # N(f) = 0
        assert torch.equal(n, b2.to(dtype).expand_as(n))


@pytest.mark.parametrize("d", WIDTHS)
def test_a_row_of_nearly_equal_numbers(where, d):
    """some last places apart: the mean is off by its own rounding, 2^-24 of it, and what comes of that is at most 1 / size of the row times as much; the sums
    themselves by d 2^-24 at most (of squares twice), the rest is a few roundings"""
    ctx, device = where
    plan = training.ResidualNorm(ctx, d, F32, pre="layer", post=None)
    g = torch.Generator().manual_seed(d)
    for value in VALUES:
        step = 2.0 ** (math.floor(math.log2(abs(value))) - 23)
        x = (torch.full((3, d), value) + step * torch.randint(-3, 4, (3, d), generator=g)).to(device)
        n = torch.full_like(x, math.nan)
        plan.forward(x, None, None, n)
        v = x.double().cpu()
        eps = float(torch.tensor(1e-5))
        c = v - v.mean(1, keepdim=True)
        size = torch.sqrt((c * c).mean(1, keepdim=True) + eps)
        want = c / size
        off = 2.0**-24 * abs(value) / size + want.abs() * 2.0**-24 * (3 * d + 16)
        # (a mean that is off by e moves the sum of squares by d e^2, which is taken out again)
        assert bool(((n.double().cpu() - want).abs() <= 1.01 * off).all()), (value, float(((n.double().cpu() - want).abs() / off).max()))
