"""Answers from 4-bit matrices on the GPU, against 64 bits."""
import math

import pytest
import torch

import lowbit_reference as lr
from lowbit_reference import BF16, F16, F32
from paper_1911_11377_amd import ckksmi, lowbit

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def ctx():
    c = ckksmi.Context(4, 3, 20, 1, 21, 1, device=0)
    yield c
    c.close()


def off_alignment(t):
    """values one element behind a whole 16 bytes, between NaN; codes where they have to be"""
    if t.dtype == torch.uint8:
        return t.clone()
    buf = torch.full((t.numel() + 24,), math.nan, dtype=t.dtype, device=DEV)
    v = buf[1:1 + t.numel()].view(t.shape)
    v.copy_(t)
    return v


LARGER = [(1, 1024, 4096, 128), (7, 999, 2731, 32), (64, 1000, 517, 64), (16, 4100, 300, 1024), (33, 513, 1024, 256), (130, 700, 65, 128), (1, 9000, 40, 32), (2, 70000, 33, 256)]


@pytest.mark.parametrize("size", lr.SIZES + LARGER, ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=["f32", "bf16", "f16"])
def test_products(ctx, size, dtype):
    lr.check_product(ctx, *size, dtype, off_alignment, DEV)


@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=["f32", "f16", "bf16"])
def test_products_of_strided_rows(ctx, dtype):
    lr.check_product(ctx, 5, 77, 19, 32, dtype, off_alignment, DEV, lead=3)
    lr.check_product(ctx, 5, 128, 24, 32, dtype, torch.clone, DEV, lead=8)


@pytest.mark.parametrize("rows,sizes,group,act", lr.BLOCKS + [(1, (1024, 4096, 1024), 128, "silu"), (7, (999, 2731, 501), 32, "poly3"), (64, (300, 1000, 200), 64, "gelu")], ids=str)
@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=["f32", "bf16", "f16"])
def test_blocks(ctx, rows, sizes, group, act, dtype):
    lr.check_block(ctx, rows, sizes, group, dtype, act, off_alignment, DEV)


@pytest.mark.parametrize("dtype,wt", [(F32, F32), (BF16, F32), (F16, BF16), (BF16, F16)], ids=str)
@pytest.mark.parametrize("rows,cols,group", [(1, 1, 32), (5, 75, 32), (300, 1300, 128), (40, 5000, 1024)])
def test_packing(ctx, rows, cols, group, dtype, wt):
    w = torch.randn((rows, cols), generator=torch.Generator().manual_seed(3)) * torch.logspace(-3, 1, cols)
    w[0, : min(cols, 40)] = 0.0
    w = off_alignment(w.to(wt).to(DEV))
    plan = lowbit.Product4(ctx, cols, rows, dtype, group)
    codes, scales = torch.full(plan.codes_shape, 255, dtype=torch.uint8, device=DEV), torch.full(plan.scales_shape, math.nan, dtype=dtype, device=DEV)
    plan.pack(w, codes, scales)
    want = lr.nearest(w, group, dtype)
    assert torch.equal(codes.cpu(), want[0]) and torch.equal(scales.cpu(), want[1])
    back = torch.full((rows, cols), math.nan, device=DEV)
    plan.unpack(codes, scales, back)
    c, s = lr.values((codes, scales), cols, group)
    assert torch.equal(back.cpu(), (c * s).float())


@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=["f32", "bf16", "f16"])
def test_values_that_are_not_finite_stay_in_their_row(ctx, dtype):
    plan = lowbit.Product4(ctx, 40, 16, dtype, 32)
    w = lr.weights(16, 40, 32, dtype, 5, lambda t: t.to(DEV), fill=0x53)
    x = torch.ones(3, 40, dtype=dtype, device=DEV)
    y, clean = torch.zeros(3, 16, dtype=dtype, device=DEV), torch.zeros(3, 16, dtype=dtype, device=DEV)
    plan.forward(x, *w, clean)
    x[1, 7] = math.inf
    plan.forward(x, *w, y)
    assert torch.equal(y[1].float(), torch.sign(w[1][:, 0].float()) * math.inf) and torch.equal(y[0], clean[0]) and torch.equal(y[2], clean[2])
    x[1, 7] = math.nan
    plan.forward(x, *w, y)
    assert bool(torch.isnan(y[1]).all()) and torch.equal(y[0], clean[0])
    x[1, 7] = torch.finfo(dtype).max / 64
    plan.forward(x, *w, y)
    assert bool(torch.isfinite(y[1]).all())


def test_equal_calls_give_equal_bits_on_any_stream_and_in_graphs(ctx):
    plan, x, w, y, ws = lr.check_block(ctx, 5, (1024, 2048, 512), 128, BF16, "silu", torch.clone, DEV)
    first = y.clone()
    side = torch.cuda.Stream()
    y.fill_(math.nan)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        plan.forward(x, *w, y, ws)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(y, first)
    graph = torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        plan.forward(x, *w, y, ws)
    for _ in range(3):
        y.fill_(math.nan)
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, first)


def test_a_trained_block_in_4_bits_answers_like_itself(ctx):
    """packed weights, read back, through the block in full width: the two differ by their own rounding alone"""
    from paper_1911_11377_amd import training

    g = torch.Generator().manual_seed(2)
    sizes = (200, 300, 100)
    w = [(torch.randn(s, generator=g) * s[1] ** -0.5).to(DEV) for s in ((300, 200), (300, 200), (100, 300))]
    x = torch.randn((9, 200), generator=g).to(DEV)
    low = lowbit.GatedFF4(ctx, *sizes, F32, "silu", 64)
    packed, wide = [], []
    for t, plan in zip(w, (low.into, low.into, low.out)):
        pair = torch.empty(plan.codes_shape, dtype=torch.uint8, device=DEV), torch.empty(plan.scales_shape, device=DEV)
        plan.pack(t, *pair)
        packed.append(pair)
        wide.append(torch.empty_like(t))
        plan.unpack(*pair, wide[-1])
    y, z = torch.empty(9, 100, device=DEV), torch.empty(9, 100, device=DEV)
    low.forward(x, *packed, y, torch.empty(low.workspace_bytes(9), dtype=torch.uint8, device=DEV))
    full = training.GatedFF(ctx, *sizes, F32, "silu")
    full.forward(x, *wide, z, torch.empty(full.workspace_bytes(9), dtype=torch.uint8, device=DEV))
    v, bound = lr.block(x, *packed, "silu", sizes, 64, F32)
    assert bool(((y.double().cpu() - v).abs() <= 1.25 * bound + lr.U * v.abs()).all())
    # the wide product's bound has the same terms, over d_in and d_hidden instead of groups
    wider, other = lr.ref.block(x.cpu(), *(t.cpu() for t in wide), "silu")["y"]
    assert bool(((y.double().cpu() - z.double().cpu()).abs() <= 1.25 * bound + other + lr.U * v.abs()).all()) and float((wider - v).abs().max()) < 1e-6


def test_as_many_rows_as_a_call_takes(ctx):
    """2^21 rows, 16-row tiles 64 rows a workgroup: every 2^17-th row is as in a call on 64 rows (the same kernel)"""
    plan = lowbit.Product4(ctx, 40, 24, BF16, 32)
    w = [t.to(DEV) for t in lr.weights(24, 40, 32, BF16, 1)]
    x = torch.randn(2**21, 40, device=DEV, generator=torch.Generator(DEV).manual_seed(2)).to(BF16)
    y = torch.full((2**21, 24), math.nan, dtype=BF16, device=DEV)
    plan.forward(x, *w, y)
    some = x[2**17 - 1::2**17].repeat(4, 1)
    want = torch.empty(64, 24, dtype=BF16, device=DEV)
    plan.forward(some, *w, want)
    assert torch.equal(y[2**17 - 1::2**17], want[:16]) and bool(torch.isfinite(y).all())
