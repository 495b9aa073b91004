"""Answers from 4-bit matrices on the CPU stand-in: every operand ends against a page that cannot be touched.  Small sizes; refusals."""
import math

import pytest
import torch

import lowbit_reference as lr
import train_emu_support as emu
from lowbit_reference import BF16, F16, F32
from paper_1911_11377_amd import ckksmi, lowbit

pytestmark = pytest.mark.skipif(not emu.available, reason="no host compiler with 16-bit float types")


@pytest.fixture(scope="module")
def ctx():
    c = emu.EmuContext()
    yield c
    assert c.errors() == 0
    c.close()


@pytest.mark.parametrize("size", lr.SIZES, ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=["f32", "bf16", "f16"])
def test_products(ctx, size, dtype):
    lr.check_product(ctx, *size, dtype, ctx.guarded)


@pytest.mark.parametrize("dtype", [F32, F16], ids=["f32", "f16"])
def test_products_of_strided_rows(ctx, dtype):
    lr.check_product(ctx, 5, 77, 19, 32, dtype, ctx.guarded, lead=3)


@pytest.mark.parametrize("rows,sizes,group,act", lr.BLOCKS, ids=str)
@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=["f32", "bf16", "f16"])
def test_blocks(ctx, rows, sizes, group, act, dtype):
    lr.check_block(ctx, rows, sizes, group, dtype, act, ctx.guarded)


@pytest.mark.parametrize("dtype,wt", [(F32, F32), (BF16, F32), (F16, BF16), (BF16, F16)], ids=str)
@pytest.mark.parametrize("rows,cols,group", [(1, 1, 32), (5, 75, 32), (3, 300, 128), (2, 1500, 1024)])
def test_packing(ctx, rows, cols, group, dtype, wt):
    w = torch.randn((rows, cols), generator=torch.Generator().manual_seed(3)) * torch.logspace(-3, 1, cols)
    w[0, : min(cols, 40)] = 0.0
    w = ctx.guarded(w.to(wt))
    plan = lowbit.Product4(ctx, cols, rows, dtype, group)
    codes, scales = ctx.guarded(torch.full(plan.codes_shape, 255, dtype=torch.uint8)), ctx.guarded(torch.full(plan.scales_shape, math.nan, dtype=dtype))
    plan.pack(w, codes, scales)
    want = lr.nearest(w, group, dtype)
    assert torch.equal(codes, want[0]) and torch.equal(scales, want[1])
    back = ctx.guarded(torch.full((rows, cols), math.nan))
    plan.unpack(codes, scales, back)
    c, s = lr.values((codes, scales), cols, group)
    assert torch.equal(back, (c * s).float())  # 4 bits times up to 24 have 27 (f32 scales): rounded once
    # no code is further than half a scale from its weight (the scale's own rounding moves the largest by 7/2 of its last place more)
    reach = s * (0.5 + 7 * lr.ref.ROUND[dtype] + 1e-6) + 2 * lr.ref.TINY[dtype] * 7
    assert bool(((back.double() - w.double()).abs() <= reach).all())


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_scales_whose_inverse_f32_does_not_hold(ctx, dtype):
    """weights of 1e-39 with zeros between them: zeros stay zeros, the others within half a scale (and what the scale's rounding adds)"""
    w = torch.zeros(2, 64)
    w[:, ::2] = torch.linspace(-7e-39, 7e-39, 32)
    plan = lowbit.Product4(ctx, 64, 2, dtype, 64)
    codes, scales, back = torch.zeros(plan.codes_shape, dtype=torch.uint8), torch.zeros(plan.scales_shape, dtype=dtype), torch.ones(2, 64)
    plan.pack(w, codes, scales)
    plan.unpack(codes, scales, back)
    s = scales.double().amax()
    assert 0.9e-39 < float(s) < 1.1e-39 and bool((back[:, 1::2] == 0).all())
    # (a bf16 denormal near 1e-39 has steps of 2^-133, 9e-41: the largest weight is seven times half of that off)
    off = s * 0.5 + (7 * 2.0**-134 if dtype == BF16 else 7 * 2.0**-149)
    assert bool(((back.double() - w.double()).abs() <= off).all())
    want = lr.nearest(w, 64, dtype)
    assert torch.equal(codes, want[0]) and torch.equal(scales, want[1])


def test_groups_without_a_finite_scale(ctx):
    w = torch.ones(4, 64)
    w[0, 3], w[1, 40], w[2, 5] = math.inf, math.nan, 1e38
    largest, one = lowbit.Product4(ctx, 64, 4, F32, 32), torch.zeros(1, 64)
    codes, scales = torch.zeros(largest.codes_shape, dtype=torch.uint8), torch.zeros(largest.scales_shape)
    largest.pack(torch.full((4, 64), 3.4e38), codes, scales)  # scales whose sixteenfold f32 does not hold
    back, y = torch.zeros(4, 64), torch.zeros(1, 4)
    largest.unpack(codes, scales, back)
    one[0, 40] = 0.5
    largest.forward(one, codes, scales, y)
    assert bool(((back / 3.4e38 - 1).abs() < 1e-6).all()) and bool(((y / 1.7e38 - 1).abs() < 1e-6).all())
    plan = lowbit.Product4(ctx, 64, 4, F16, 32)
    codes, scales = torch.zeros(plan.codes_shape, dtype=torch.uint8), torch.zeros(plan.scales_shape, dtype=F16)
    plan.pack(w, codes, scales)
    want = lr.nearest(w, 32, F16)
    assert torch.equal(codes, want[0]) and torch.equal(torch.isnan(scales), torch.isnan(want[1]))
    assert torch.isnan(scales).tolist() == [[True, False], [False, True], [True, False], [False, False]]


@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=["f32", "bf16", "f16"])
def test_values_that_are_not_finite_stay_in_their_row(ctx, dtype):
    """an infinity times a code that is not zero, and next to large values"""
    plan = lowbit.Product4(ctx, 40, 16, dtype, 32)
    w = lr.weights(16, 40, 32, dtype, 5, ctx.guarded, fill=0x53)  # codes 3 and 5
    x = torch.ones(3, 40, dtype=dtype)
    y, clean = torch.zeros(3, 16, dtype=dtype), torch.zeros(3, 16, dtype=dtype)
    plan.forward(ctx.guarded(x), *w, clean)
    x[1, 7] = math.inf
    plan.forward(ctx.guarded(x), *w, y)
    sign = torch.sign(w[1][:, 0].float())
    assert torch.equal(y[1].float(), sign * math.inf) and torch.equal(y[0], clean[0]) and torch.equal(y[2], clean[2])
    x[1, 7] = math.nan
    plan.forward(ctx.guarded(x), *w, y)
    assert bool(torch.isnan(y[1]).all()) and torch.equal(y[0], clean[0])
    x[1, 7] = torch.finfo(dtype).max / 64
    plan.forward(ctx.guarded(x), *w, y)
    assert bool(torch.isfinite(y[1]).all())


def test_no_rows_and_fewer_rows(ctx):
    plan = lowbit.GatedFF4(ctx, 40, 24, 16, BF16, "square", 32)
    w = [lr.weights(24, 40, 32, BF16, 1), lr.weights(24, 40, 32, BF16, 2), lr.weights(16, 24, 32, BF16, 3)]
    none = torch.empty(0, 40, dtype=BF16)
    plan.forward(none, *w, torch.empty(0, 16, dtype=BF16), torch.empty(0, dtype=torch.uint8))
    plan.into.forward(none, *w[0], torch.empty(0, 24, dtype=BF16))
    sizes = [plan.workspace_bytes(n) for n in (0, 1, 2, 17, 64, 100)]
    assert sizes == sorted(sizes)


# ---------------------------------------------------------------- refusals
def refused(code, call, *args, **kw):
    with pytest.raises(ckksmi.CkksmiError) as e:
        call(*args, **kw)
    assert e.value.code == code, e.value


def test_plans_that_are_refused(ctx):
    for group in (16, 48, 2048):
        plan = lowbit.Product4(ctx, 64, 8, BF16, group)
        refused(ckksmi.EINVAL, plan.forward, torch.zeros(1, 64, dtype=BF16), *lr.weights(8, 64, group, BF16, 1), torch.zeros(1, 8, dtype=BF16))
    for group in (0, -32):
        refused(ckksmi.EINVAL, lowbit.GatedFF4(ctx, 64, 8, 8, BF16, "silu", group).workspace_bytes, 1)
    refused(ckksmi.EINVAL, lowbit.GatedFF4(ctx, 2**20 + 1, 8, 8, BF16, "silu").workspace_bytes, 1)
    refused(ckksmi.EINVAL, lowbit.GatedFF4(ctx, 64, 8, 8, BF16, "silu").workspace_bytes, 2**21 + 1)
    with pytest.raises(ValueError):
        lowbit.Product4(ctx, 64, 8, torch.float64)
    with pytest.raises(KeyError):
        lowbit.GatedFF4(ctx, 64, 8, 8, BF16, "tanh")


def test_products_that_are_refused(ctx):
    plan, x, w, y = lr.check_product(ctx, 3, 64, 16, 32, BF16, lambda t: t)
    for args in ((x.float(), *w, y), (x[:, :32], *w, y), (x, w[0][:, :16], w[1], y), (x, w[0].to(torch.int8), w[1], y), (x, w[0], w[1].float(), y), (x, *w, y[:2]), (x[:1].expand(3, 64), *w, y)):
        with pytest.raises(ValueError):
            plan.forward(*args)
    both = torch.zeros(3 * 64 + 3 * 16, dtype=BF16)
    refused(ckksmi.EINVAL, plan.forward, both[:192].view(3, 64), *w, both[160:208].view(3, 16))
    off = torch.zeros(w[0].numel() + 8, dtype=torch.uint8)[8:].view(w[0].shape)
    refused(ckksmi.EINVAL, plan.forward, x, off, w[1], y)
    with pytest.raises(ValueError):
        plan.pack(torch.zeros(16, 63), *w)
    flat = torch.zeros(16 * 64, dtype=BF16)
    refused(ckksmi.EINVAL, plan.pack, flat.view(16, 64), w[0], flat[:32].view(16, 2))


def test_blocks_that_are_refused(ctx):
    plan, x, w, y, ws = lr.check_block(ctx, 2, (64, 32, 16), 32, BF16, "silu", lambda t: t)
    refused(ckksmi.EWORKSPACE, plan.forward, x, *w, y, ws[:-1])
    refused(ckksmi.EINVAL, plan.forward, x, *w, y, torch.zeros(ws.numel() + 8, dtype=torch.uint8)[8:])
    refused(ckksmi.EINVAL, plan.forward, x, *w, ws[:64].view(BF16).view(2, 16), ws)
    refused(ckksmi.EINVAL, plan.forward, x, *w, x[:, :16], ws)
    with pytest.raises(ValueError):
        plan.forward(x, w[0], w[1], w[0], y, ws)
