"""Norms around a block on the CPU stand-in: every operand ends against a page that cannot be touched.  Small sizes of each kernel; refusals."""
import math

import pytest
import torch

import norm_reference as nr
import train_emu_support as emu
from norm_reference import BF16, F16, F32
from paper_1911_11377_amd import ckksmi, training

pytestmark = pytest.mark.skipif(not emu.available, reason="no host compiler with 16-bit float types")


@pytest.fixture(scope="module")
def ctx():
    c = emu.EmuContext()
    yield c
    assert c.errors() == 0
    c.close()


@pytest.mark.parametrize("rows,d", nr.SIZES, ids=lambda v: str(v))
@pytest.mark.parametrize("dtype,wt", [(F32, None), (BF16, F32), (F16, None)], ids=["f32", "bf16", "f16"])
def test_sizes(ctx, rows, d, dtype, wt):
    pre, post, gate = nr.KINDS[(rows + d) % 2]
    nr.check(ctx, nr.Case(rows, d, dtype, pre, post, gate, wt, place=ctx.guarded), ctx.guarded)


@pytest.mark.parametrize("pre,post,gate", nr.KINDS, ids=str)
@pytest.mark.parametrize("dtype,wt", [(BF16, None), (F32, None), (F16, F32)], ids=["bf16", "f32", "f16"])
def test_kinds(ctx, pre, post, gate, dtype, wt):
    nr.check(ctx, nr.Case(7, 75, dtype, pre, post, gate, wt, lead=3, place=ctx.guarded), ctx.guarded, accumulate=True)


@pytest.mark.parametrize("pre", ["rms", "layer"])
def test_the_first_norm_has_no_block_before_it(ctx, pre):
    nr.check(ctx, nr.Case(5, 90, BF16, pre, None, None, with_f=False, place=ctx.guarded), ctx.guarded)
    nr.check(ctx, nr.Case(5, 90, F32, pre, "layer", "channel", with_f=False, weights=False, place=ctx.guarded), ctx.guarded)


def test_weights_may_be_left_out(ctx):
    nr.check(ctx, nr.Case(5, 33, F32, "layer", "layer", "channel", weights=False, place=ctx.guarded), ctx.guarded)


@pytest.mark.parametrize("dr,dn", [(False, True), (True, False), (False, False)])
def test_gradients_that_are_not_there(ctx, dr, dn):
    nr.check(ctx, nr.Case(5, 40, F32, "rms", "rms", "channel", place=ctx.guarded), ctx.guarded, dr=dr, dn=dn)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("pre,post,gate", [("layer", "layer", "element"), ("rms", None, "channel"), (None, "rms", None)], ids=str)
def test_rows_longer_than_registers_hold(ctx, dtype, pre, post, gate):
    """8193 columns: the backward pass reads rows several times; 16385: the forward pass too"""
    nr.check(ctx, nr.Case(3, 8193, dtype, pre, post, gate, F32, place=ctx.guarded), ctx.guarded)
    nr.check(ctx, nr.Case(2, 16385, dtype, pre, post, gate, F32, place=ctx.guarded), ctx.guarded, accumulate=True)


@pytest.mark.parametrize("d", [40, 16390])
def test_the_sum_may_overwrite_x(ctx, d):
    c = nr.Case(3, d, BF16, "layer", "rms", "channel", F32, place=ctx.guarded)
    plan = training.ResidualNorm(ctx, d, BF16, "layer", "rms", "channel", F32)
    plan.forward(c.x, c.f, c.r, c.n, gate=c.gate, **c.w)
    n = torch.empty_like(c.n)
    plan.forward(c.x, c.f, c.x, n, gate=c.gate, **c.w)
    assert torch.equal(c.x, c.r) and torch.equal(n, c.n)
    # and a sum that nobody reads need not be written
    plan.forward(c.r, c.f, None, n, gate=c.gate, **c.w)


@pytest.mark.parametrize("d", [16, 8200])
def test_large_means_and_magnitudes(ctx, d):
    """a mean a thousand times the spread, rows whose squares are near the ends of the range of f32, a row of zeros"""
    c = nr.Case(4, d, F32, "layer", "layer", None, place=ctx.guarded)
    c.x[0] += 1000.0
    c.f[1] = c.f[1] * 1e15
    c.x[2] = c.x[2] * 1e-12
    c.f[2] = c.f[2] * 1e-12
    c.f[3] = 0.0
    nr.check(ctx, c, ctx.guarded)


def test_values_that_are_not_finite_stay_in_their_row(ctx):
    """what the formulas give: an infinity makes the finite elements of an rms row zeros and itself NaN; other rows keep their bits"""
    for kind in ("rms", "layer"):
        c = nr.Case(3, 20, BF16, kind, None, None, F32, place=ctx.guarded)
        plan = training.ResidualNorm(ctx, 20, BF16, kind, None, None, F32)
        plan.forward(c.x, c.f, c.r, c.n, **c.w)
        before = c.n.clone()
        c.x[1, 3] = math.inf
        plan.forward(c.x, c.f, c.r, c.n, **c.w)
        assert torch.equal(c.n[0], before[0]) and torch.equal(c.n[2], before[2])
        assert math.isinf(float(c.r[1, 3])) and bool(torch.isnan(c.n[1, 3]))
        others = torch.cat([c.n[1, :3], c.n[1, 4:]])
        if kind == "rms":
            assert bool((others == 0).all())
        else:
            assert bool(torch.isnan(others).all())
        c.x[1, 3] = math.nan
        plan.forward(c.x, c.f, c.r, c.n, **c.w)
        assert bool(torch.isnan(c.n[1]).all()) and torch.equal(c.n[0], before[0])


def test_no_rows(ctx):
    """nothing to do forward; the sums of no rows are zeros, or what was there"""
    plan = training.ResidualNorm(ctx, 12, BF16, "layer", "rms", "channel", F32)
    none = torch.empty(0, 12, dtype=BF16)
    plan.forward(none, none, none, none, gate=torch.ones(12), post_weight=torch.ones(12), saved=torch.empty(0, dtype=torch.uint8))
    for accumulate in (True, False):
        g = {k: ctx.guarded(torch.full((12,), 3.0)) for k in ("dpost_weight", "dpre_weight", "dpre_bias", "dgate")}
        plan.backward(none, none, torch.empty(0, dtype=torch.uint8), none, none, None, gate=torch.ones(12), accumulate=accumulate, **g)
        assert all(bool((t == (3.0 if accumulate else 0.0)).all()) for t in g.values())


def test_a_workspace_serves_fewer_rows(ctx):
    for d in (8, 64, 200, 1021, 8192, 8200):
        plan = training.ResidualNorm(ctx, d, BF16)
        sizes = [plan.workspace_bytes(rows) for rows in (0, 1, 2, 5, 31, 64, 100, 1000, 1024, 1030, 5000, 100000)]
        assert sizes == sorted(sizes)


def test_gradients_against_differences(ctx):
    """the derivative along a direction, from the 64-bit forward reference at two points h apart: the differences' own error is
    of the order h^2 times a third derivative (here below 1e-6), the gradients' is bounded by the test above"""
    c = nr.Case(4, 12, F32, "layer", "layer", "element", place=ctx.guarded)
    plan = training.ResidualNorm(ctx, 12, F32, "layer", "layer", "element", eps=1e-3, residual_scale=0.9, block_scale=-0.7)
    saved, ws = ctx.guarded(torch.zeros(plan.saved_bytes(4), dtype=torch.uint8)), ctx.guarded(torch.zeros(plan.workspace_bytes(4), dtype=torch.uint8))
    plan.forward(c.x, c.f, c.r, c.n, gate=c.gate, saved=saved, **c.w)
    grads = c.gradients()
    plan.backward(c.x, c.f, saved, c.dr, c.dn, ws, gate=c.gate, **grads, **c.w)
    at = {"x": c.x, "f": c.f, "gate": c.gate, **c.w}

    def value(moved):
        t = {k: v.double() for k, v in {**at, **moved}.items()}
        w = {k: t[k] for k in c.w}
        o = nr.residual_norm(t["x"], t["f"], t["gate"], w, "layer", "layer", 1e-3, 0.9, -0.7)
        return float((o["r"][0] * c.dr.double()).sum() + (o["n"][0] * c.dn.double()).sum())

    for k, t in at.items():
        to = torch.randn(t.shape, generator=torch.Generator().manual_seed(9), dtype=torch.float64)
        h = 1e-4
        slope = (value({k: t.double() + h * to}) - value({k: t.double() - h * to})) / (2 * h)
        mine = float((grads["d" + k].double() * to).sum())
        assert abs(mine - slope) <= 1e-4 * max(1.0, abs(slope)), (k, mine, slope)


# ---------------------------------------------------------------- refusals
def refused(code, call, *args, **kw):
    with pytest.raises(ckksmi.CkksmiError) as e:
        call(*args, **kw)
    assert e.value.code == code, e.value


def test_plans_that_make_no_sense(ctx):
    with pytest.raises(ValueError):
        training.ResidualNorm(ctx, 8, BF16, pre="batch")
    with pytest.raises(ValueError):
        training.ResidualNorm(ctx, 8, torch.float64)
    for kw in (dict(d=0), dict(d=2**20 + 1), dict(eps=-1.0), dict(eps=math.nan), dict(residual_scale=math.inf), dict(block_scale=math.nan), dict(dtype=BF16, weight_dtype=F16)):
        kw = {"d": 8, "dtype": F32, **kw}
        d, dtype = kw.pop("d"), kw.pop("dtype")
        refused(ckksmi.EINVAL, training.ResidualNorm(ctx, d, dtype, **kw).workspace_bytes, 4)
    refused(ckksmi.EINVAL, training.ResidualNorm(ctx, 8, F32).saved_bytes, -1)
    assert training.ResidualNorm(ctx, 8, F32).saved_bytes(2**30) == 2**34
    refused(ckksmi.EINVAL, training.ResidualNorm(ctx, 8, F32).saved_bytes, 2**30 + 1)


def test_forward_calls_that_are_refused(ctx):
    c = nr.Case(4, 16, BF16, "rms", "layer", "channel", F32)
    plan = training.ResidualNorm(ctx, 16, BF16, "rms", "layer", "channel", F32)
    ok = dict(x=c.x, f=c.f, r=c.r, n=c.n, gate=c.gate, **c.w)
    plan.forward(**ok)
    bad = [dict(gate=None), dict(n=None), dict(pre_bias=c.w["post_bias"]), dict(f=None), dict(f=None, r=None, gate=None), dict(r=c.f), dict(n=c.x), dict(n=c.r),
           dict(r=None, n=c.f), dict(saved=torch.zeros(65, dtype=torch.uint8)[1:])]
    for change in bad:
        refused(ckksmi.EINVAL, plan.forward, **{**ok, **change})
    wide = torch.zeros(4, 40, dtype=BF16)
    refused(ckksmi.EINVAL, plan.forward, **{**ok, "x": wide[:, :16], "r": wide[:, 8:24]})  # one over the other
    for change in (dict(x=c.x.float()), dict(x=c.x[:, :8]), dict(n=c.n[:3]), dict(post_weight=c.w["post_weight"].to(BF16)), dict(gate=torch.zeros(8)),
                   dict(x=c.x[:1].expand(4, 16)), dict(saved=torch.zeros(63, dtype=torch.uint8))):
        with pytest.raises(ValueError):
            plan.forward(**{**ok, **change})
    none = training.ResidualNorm(ctx, 16, BF16, None, None, None)
    refused(ckksmi.EINVAL, none.forward, c.x, c.f, None, None)  # nothing to write
    refused(ckksmi.EINVAL, none.forward, c.x, c.f, c.r, c.n)


def test_backward_calls_that_are_refused(ctx):
    c = nr.Case(4, 16, BF16, "layer", "layer", "channel", F32)
    plan = training.ResidualNorm(ctx, 16, BF16, "layer", "layer", "channel", F32)
    saved, ws = torch.zeros(64, dtype=torch.uint8), torch.zeros(plan.workspace_bytes(4), dtype=torch.uint8)
    plan.forward(c.x, c.f, c.r, c.n, gate=c.gate, saved=saved, **c.w)
    g = c.gradients()
    ok = dict(x=c.x, f=c.f, saved=saved, dr=c.dr, dn=c.dn, ws=ws, gate=c.gate, **g, **c.w)
    plan.backward(**ok)
    refused(ckksmi.EWORKSPACE, plan.backward, **{**ok, "ws": ws[:-1]})
    for change in (dict(ws=None), dict(dx=c.dr), dict(df=c.f), dict(dx=g["df"]), dict(dgate=g["dpre_bias"]), dict(gate=None), dict(f=None)):
        refused(ckksmi.EINVAL, plan.backward, **{**ok, **change})
    with pytest.raises(ValueError):
        plan.backward(**{**ok, "saved": None})
    # without sums no workspace is needed
    plan.backward(**{**ok, "ws": None, **{k: None for k in g if k not in ("dx", "df")}})
    rms = training.ResidualNorm(ctx, 16, BF16, "rms", None, None, F32)
    for change in (dict(dpre_bias=g["dpre_bias"]), dict(dpost_weight=g["dpost_weight"]), dict(dgate=g["dgate"])):
        refused(ckksmi.EINVAL, rms.backward, c.x, c.f, saved, c.dr, c.dn, ws, **change)
