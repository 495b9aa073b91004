"""Products with 4-bit matrices at the ends of their types' ranges: NaN of any payload; on the CPU stand-in and
on the GPU."""
import pytest
import torch

import train_emu_support as emu
from lowbit_reference import F32
from paper_1911_11377_amd import ckksmi, lowbit


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


def matrix4(plan, code, scale, device):
    """every element code * scale"""
    codes = torch.full(plan.codes_shape, (code & 15) * 17, dtype=torch.uint8, device=device)
    return codes, torch.full(plan.scales_shape, scale, dtype=plan.dtype, device=device)


def room(n, device):
    return torch.zeros(max(16, n), dtype=torch.uint8, device=device)


@pytest.mark.parametrize("word", [0x7F800001, 0x7FC00000, 0x7F80FFFF, 0xFF800001, 0xFFFFFFFF])
@pytest.mark.parametrize("rows", [2, 20, 60])
def test_every_nan_makes_its_row_nan(where, word, rows):
    """one whose payload is in the lower half of its word too"""
    ctx, device = where
    for d_in, at in ((40, 33), (300, 7)):
        x = torch.ones(rows, d_in)
        x.view(torch.int32)[1, at] = word - 2**32 if word >= 2**31 else word
        x = x.to(device)
        plan = lowbit.Product4(ctx, d_in, 9, F32, 32)
        y = torch.zeros(rows, 9, device=device)
        plan.forward(x, *matrix4(plan, 3, 0.5, device), y)
        block = lowbit.GatedFF4(ctx, d_in, 5, 9, F32, "linear", 32)
        z, ws = torch.zeros(rows, 9, device=device), room(block.workspace_bytes(rows), device)
        into = matrix4(block.into, 1, 0.01, device)
        block.forward(x, into, into, matrix4(block.out, 1, 1.0, device), z, ws)
        for r in (y, z):
            assert bool(torch.isnan(r[1]).all()) and bool(torch.isfinite(r[torch.arange(rows) != 1]).all())
