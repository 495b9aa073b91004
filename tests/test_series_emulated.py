"""Orthogonalised directions and steps along them on the CPU stand-in: small sizes of each kernel, and refusals."""
import ctypes as C
import math

import pytest
import torch

import series_reference as sr
import train_emu_support as emu
from paper_1911_11377_amd import ckksmi, training
from series_reference import BF16, F16, F32

pytestmark = pytest.mark.skipif(not emu.available, reason="no host compiler with 16-bit float types")


@pytest.fixture(scope="module", params=["small", "tiles"])
def ctx(request):
    """matrices in one workgroup's LDS where they fit; and in tiles whatever their size"""
    c = emu.EmuContext()
    c._L.emu_series_small.argtypes = [C.c_size_t]
    c.kind = request.param
    c._L.emu_series_small(2**63 if c.kind == "small" else 0)
    yield c
    c._L.emu_series_small(2**63)
    assert c.errors() == 0
    c.close()


def room(ctx, n):
    return ctx.guarded(torch.full((max(n, 16),), 255, dtype=torch.uint8))


def direct(ctx, u, out=None, **kw):
    out = ctx.guarded(torch.full(u.shape, math.nan, dtype=u.dtype)) if out is None else out
    plan = training.Orthogonalise(ctx, [u], [out])
    plan.run(room(ctx, plan.workspace_bytes()), **kw)
    return out


@pytest.mark.parametrize("rows,cols", sr.SIZES, ids=str)
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_sizes(ctx, rows, cols, dtype):
    u = ctx.guarded(sr.matrix(rows, cols, rows + cols, dtype=dtype))
    sr.check(direct(ctx, u), u, 1 if dtype == BF16 else 2)


@pytest.mark.parametrize("kind", ["strong", "falling", "rank3"])
@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=["f32", "bf16", "f16"])
def test_spectra(ctx, kind, dtype):
    u = ctx.guarded(sr.matrix(24, 40, 3, kind, dtype))
    sr.check(direct(ctx, u), u, 1 if dtype == BF16 else 2)


@pytest.mark.parametrize("size,tile,dtype", [((140, 70), 0, F32), ((140, 70), 1, F32), ((200, 140), 0, BF16), ((200, 140), 1, F32), ((200, 140), -1, BF16), ((300, 290), 0, BF16)], ids=str)
def test_large_tiles(ctx, size, tile, dtype):
    """tiles of 128 x 128 and 256 x 256, whole and ragged, below and on the diagonal"""
    if ctx.kind == "small":
        pytest.skip("matrices that are none for one workgroup: the same kernels as the other way")
    ctx._L.emu_enough_tiles(1)
    ctx._L.emu_series_tile(tile)
    try:
        u = ctx.guarded(sr.matrix(*size, 5, "strong", dtype))
        sr.check(direct(ctx, u, steps=1), u, 1 if dtype == BF16 else 2, steps=1)
    finally:
        ctx._L.emu_enough_tiles(192)
        ctx._L.emu_series_tile(-1)


def test_a_split_k_axis(ctx):
    """in parts of the smallest tiles; and, with many steps and enough tiles, of 128 x 128 ones"""
    u = ctx.guarded(sr.matrix(20, 1100, 5, "strong"))
    sr.check(direct(ctx, u, steps=2), u, 2, steps=2)


def test_in_place_zeros_and_small_numbers(ctx):
    u = ctx.guarded(sr.matrix(12, 30, 4, dtype=F32))
    want = direct(ctx, u)
    start = u.clone()
    assert torch.equal(direct(ctx, u, out=u), want)
    z = ctx.guarded(torch.zeros(9, 20))
    assert bool((direct(ctx, z) == 0).all()) and bool((direct(ctx, z, eps=0.0) == 0).all())
    for scale in (1e-30, 1e30):  # squares that f32 does not hold
        v = ctx.guarded(start * scale)
        sr.check(direct(ctx, v, eps=0.0), v, 2, eps=0.0)
    # eps is part of the size
    sr.check(direct(ctx, ctx.guarded(start), eps=5.0), start, 2, eps=5.0)


def test_values_that_are_not_finite(ctx):
    for bad in (math.nan, math.inf):
        u, v = sr.matrix(10, 20, 6), sr.matrix(8, 30, 7)
        u[3, 4] = bad
        outs = [ctx.guarded(torch.zeros_like(t)) for t in (u, v)]
        plan = training.Orthogonalise(ctx, [ctx.guarded(u), ctx.guarded(v)], outs)
        plan.run(room(ctx, plan.workspace_bytes()))
        assert bool(torch.isnan(outs[0]).any()) and not bool((outs[0][torch.isfinite(outs[0])] != 0).any())
        sr.check(outs[1], v, 2)


@pytest.mark.parametrize("rows,cols", [(64, 380), (1050, 16), (48, 400), (17, 33), (64, 64)], ids=str)
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_the_largest_that_fit_one_workgroup(ctx, rows, cols, dtype):
    u = ctx.guarded(sr.matrix(rows, cols, 5, "strong", dtype))
    plan = training.Orthogonalise(ctx, [u], [ctx.guarded(torch.zeros_like(u))])
    assert (plan.workspace_bytes() == 0) == (ctx.kind == "small")
    sr.check(direct(ctx, u, steps=2), u, 1 if dtype == BF16 else 2, steps=2)


def test_other_polynomials_and_numbers_of_steps(ctx):
    u = ctx.guarded(sr.matrix(9, 21, 8))
    for steps, k in ((1, sr.COEFFICIENTS), (4, sr.COEFFICIENTS), (8, (1.5, -0.5, 0.0)), (3, (2.0, -1.5, 0.5))):
        sr.check(direct(ctx, u, steps=steps, coefficients=k), u, 2, steps=steps, coefficients=k)


def test_derived_properties(ctx):
    """after enough steps of 1.5 s - 0.5 s^3 the rows are orthonormal"""
    u = ctx.guarded(sr.matrix(6, 40, 2))
    o = direct(ctx, u, steps=20, coefficients=(1.5, -0.5, 0.0)).double()
    assert float((o @ o.t() - torch.eye(6)).abs().max()) < 1e-5


@pytest.mark.parametrize("dtype,gt,copy", [(F32, BF16, BF16), (F32, F32, None), (BF16, BF16, None), (F16, F32, F16)], ids=str)
@pytest.mark.parametrize("nesterov", [True, False])
def test_steps(ctx, dtype, gt, copy, nesterov):
    """several matrices of one call, more than one launch's table holds, among them empty ones"""
    sizes = [(16, 40), (40, 16), (0, 7), (1, 9), (33, 33), (5, 0)] + [(3, 4)] * 22
    p0 = [sr.matrix(*s, i, scale=0.1, dtype=dtype) for i, s in enumerate(sizes)]
    g = [ctx.guarded(sr.matrix(*s, 100 + i, scale=10.0 ** (-i % 5), dtype=gt)) for i, s in enumerate(sizes)]
    m0 = [sr.matrix(*s, 200 + i, scale=10.0 ** (-i % 5)) for i, s in enumerate(sizes)]
    p, m = [ctx.guarded(t) for t in p0], [ctx.guarded(t) for t in m0]
    copies = [ctx.guarded(torch.zeros(s, dtype=copy)) for s in sizes] if copy else None
    opt = training.Muon(ctx, p, g, m, copies=copies)
    opt.step(0.02, 0.9, room(ctx, opt.workspace_bytes()), weight_decay=0.1, nesterov=nesterov, grad_scale=0.5)
    for i, (r, c) in enumerate(sizes):
        if not r * c:
            continue
        wm, u = sr.momentum(m0[i], g[i], 0.9, 0.5, nesterov)
        assert torch.equal(m[i], wm)
        sr.check_step(p[i], p0[i], u, 2 if dtype == F32 else 1, 0.02, max(1.0, r / c) ** 0.5, 0.1, copies[i] if copies else None)


def test_a_step_that_is_skipped(ctx):
    p0, g, m0 = sr.matrix(9, 20, 1), sr.matrix(9, 20, 2), sr.matrix(9, 20, 3)
    p, m = ctx.guarded(p0), ctx.guarded(m0)
    opt = training.Muon(ctx, [p], [ctx.guarded(g)], [m])
    ws = room(ctx, opt.workspace_bytes())
    opt.step(0.1, 0.9, ws, skip=ctx.guarded(torch.ones(1, dtype=torch.int32)))
    assert torch.equal(p, p0) and torch.equal(m, m0)
    opt.step(0.1, 0.9, ws, skip=ctx.guarded(torch.zeros(1, dtype=torch.int32)))
    assert not torch.equal(p, p0) and not torch.equal(m, m0)


def test_nothing_to_do(ctx):
    plan = training.Orthogonalise(ctx, [], [])
    plan.run(room(ctx, plan.workspace_bytes()))
    opt = training.Muon(ctx, [torch.zeros(0, 4)], [torch.zeros(0, 4)], [torch.zeros(0, 4)])
    opt.step(0.1, 0.9, room(ctx, opt.workspace_bytes()))


# ---------------------------------------------------------------- refusals
def refused(code, call, *args, **kw):
    with pytest.raises(ckksmi.CkksmiError) as e:
        call(*args, **kw)
    assert e.value.code == code, e.value


def test_polynomials_that_leave_the_range_are_refused(ctx):
    u = sr.matrix(70, 80, 1)
    plan = training.Orthogonalise(ctx, [u], [torch.zeros_like(u)])
    ws = room(ctx, plan.workspace_bytes())
    for kw in (dict(steps=0), dict(steps=33), dict(eps=-1.0), dict(eps=math.nan), dict(coefficients=(3.0, 0.0, 0.0)), dict(coefficients=(1.0, math.inf, 0.0)),
               dict(coefficients=(0.0, 0.0, 120.0)), dict(coefficients=(1.5, 0.0, 0.0), steps=3)):
        refused(ckksmi.EINVAL, plan.run, ws, **kw)
    plan.run(ws, steps=3)
    refused(ckksmi.EWORKSPACE, plan.run, ws[:-1])
    refused(ckksmi.EINVAL, plan.run, ctx.guarded(torch.zeros(ws.numel() + 8, dtype=torch.uint8))[8:])


def test_plans_that_are_refused(ctx):
    u = torch.zeros(4, 6)
    for args in (([u], [torch.zeros(4, 5)]), ([u], [torch.zeros(4, 6, dtype=BF16)]), ([u], []), ([torch.zeros(6)], [torch.zeros(6)]), ([u, u], [torch.zeros(4, 6)] * 2)):
        with pytest.raises(ValueError):
            training.Orthogonalise(ctx, *args)
    with pytest.raises(ValueError):
        training.Orthogonalise(ctx, [u.t()], [torch.zeros(6, 4)])  # not contiguous
    with pytest.raises(ValueError):
        training.Orthogonalise(ctx, [u, torch.zeros(4, 6)], [torch.zeros(4, 6), u])  # written while the other reads it
    for kw in (dict(m=[torch.zeros(4, 6, dtype=BF16)]), dict(grads=[torch.zeros(6, 4)]), dict(m=[u]), dict(copies=[torch.zeros(4, 6, dtype=torch.float64)]), dict(scales=[1.0, 2.0])):
        with pytest.raises(ValueError):
            training.Muon(ctx, **{**dict(params=[u], grads=[torch.zeros(4, 6)], m=[torch.zeros(4, 6)]), **kw})
    wide = torch.zeros(2**16 + 1, 1)
    refused(ckksmi.EINVAL, training.Orthogonalise(ctx, [wide], [torch.zeros_like(wide)]).workspace_bytes)


def test_steps_that_are_refused(ctx):
    p, g, m = sr.matrix(70, 80, 1), sr.matrix(70, 80, 2), sr.matrix(70, 80, 3)
    opt = training.Muon(ctx, [p], [g], [m])
    ws = room(ctx, opt.workspace_bytes())
    for a, kw in (((math.nan, 0.9), {}), ((0.1, 1.0), {}), ((0.1, -0.1), {}), ((0.1, 0.9), dict(weight_decay=math.inf)), ((0.1, 0.9), dict(grad_scale=math.nan)),
                  ((0.1, 0.9), dict(steps=0))):
        refused(ckksmi.EINVAL, opt.step, *a, ws, **kw)
    refused(ckksmi.EWORKSPACE, opt.step, 0.1, 0.9, ws[:16])
    with pytest.raises(ValueError):
        opt.step(0.1, 0.9, ws, skip=torch.zeros(1))
    bad = training.Muon(ctx, [p], [g], [m], scales=[math.inf])
    refused(ckksmi.EINVAL, bad.workspace_bytes)
    both = torch.zeros(ws.numel() + 4096, dtype=torch.uint8)
    inside = both[1024:1024 + 4 * 5600].view(torch.float32).view(70, 80)
    refused(ckksmi.EINVAL, training.Muon(ctx, [inside], [g], [m]).step, 0.1, 0.9, both)
