"""The training kernels on the CPU stand-in (tests/emu/train_emu.cpp): every operand ends against a page that cannot be touched,
loads to LDS arrive no earlier than they are waited for, LDS accesses stay in the kernel's array.  Small sizes of each kernel."""
import math

import numpy as np
import pytest
import torch

import train_emu_support as emu
import training_reference as ref
from paper_1911_11377_amd import ckksmi, training

pytestmark = pytest.mark.skipif(not emu.available, reason="no host compiler with 16-bit float types")
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def ctx():
    c = emu.EmuContext()
    yield c
    assert c.errors() == 0
    c.close()


def normal(seed, *shape, scale=1.0, dtype=F32):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * scale).to(dtype)


def nan_bytes(ctx, n):
    return ctx.guarded(torch.full((max(n, 16),), 255, dtype=torch.uint8))


def run_block(ctx, rows, d_in, d_hidden, d_out, dtype, act="poly3", grad_dtype=None, misaligned=False, accumulate=False):
    cubic = training.CUBICS.get(act, act)
    ff = training.GatedFF(ctx, d_in, d_hidden, d_out, dtype, act, grad_dtype)
    gt = grad_dtype or dtype

    def place(t):
        if not misaligned:
            return ctx.guarded(t)
        flat = ctx.guarded(torch.cat([t.reshape(-1)[:1], t.reshape(-1)]))  # one element behind 16-byte alignment, or in front of it
        return flat[1:].view(t.shape)

    x = place(normal(1, rows, d_in, dtype=dtype))
    wg, wu = place(normal(2, d_hidden, d_in, scale=d_in**-0.5, dtype=dtype)), place(normal(3, d_hidden, d_in, scale=d_in**-0.5, dtype=dtype))
    wd, dy = place(normal(4, d_out, d_hidden, scale=d_hidden**-0.5, dtype=dtype)), place(normal(5, rows, d_out, dtype=dtype))
    y, dx = place(torch.full((rows, d_out), math.nan, dtype=dtype)), place(torch.full((rows, d_in), math.nan, dtype=dtype))
    dw = [place(torch.full(w.shape, 0.0 if accumulate else math.nan, dtype=gt)) for w in (wg, wu, wd)]
    saved = nan_bytes(ctx, ff.saved_bytes(rows))
    ff.forward(x, wg, wu, wd, y, nan_bytes(ctx, ff.workspace_bytes(rows)), saved=saved)
    first = y.clone()
    ff.forward(x, wg, wu, wd, y, nan_bytes(ctx, ff.workspace_bytes(rows)))
    assert torch.equal(y, first)
    ff.backward(x, wg, wu, wd, saved, dy, dx, *dw, nan_bytes(ctx, ff.workspace_bytes(rows, backward=True)), accumulate=accumulate)
    want = ref.block(x, wg, wu, wd, cubic, dy, gt)
    for name, got in (("y", y), ("dx", dx), ("dwg", dw[0]), ("dwu", dw[1]), ("dwd", dw[2])):
        v, bound = want[name]
        assert bool(((got.double() - v).abs() <= bound).all()), (name, float(((got.double() - v).abs() - bound).max()))
    assert ctx.errors() == 0


@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=["f32", "bf16", "f16"])
@pytest.mark.parametrize("size", [(1, 1, 1, 1), (1, 200, 24, 16), (3, 5, 7, 9), (17, 40, 24, 1), (33, 70, 33, 20), (65, 33, 9, 31), (70, 136, 72, 40)], ids=lambda s: "x".join(map(str, s)))
def test_block(ctx, size, dtype):
    run_block(ctx, *size, dtype)


@pytest.mark.parametrize("size,dtype,grads,act", [((9, 24, 16, 8), BF16, F32, "silu"), ((70, 40, 24, 17), F16, F32, "gelu"), ((40, 16, 136, 8), BF16, None, "relu"),
                                                   ((1, 107, 8, 19), F32, None, "silu"), ((70, 33, 40, 7), F32, None, "gelu")],
                         ids=["fine", "fine16", "relu", "silu-f32", "gelu-f32"])
def test_block_with_other_gradients_and_activations(ctx, size, dtype, grads, act):
    run_block(ctx, *size, dtype, act, grads)


@pytest.mark.parametrize("size", [(5, 16, 8, 8), (66, 24, 16, 8)], ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_block_off_alignment(ctx, size, dtype):
    run_block(ctx, *size, dtype, misaligned=True, accumulate=True)


@pytest.mark.parametrize("hidden", [2100, 4200])
def test_few_rows_in_one_workgroup(ctx, hidden):
    """64 rows and so many columns that a workgroup takes 32 of the rows, or all of them"""
    run_block(ctx, 64, 8, hidden, 8, BF16, "square")


def test_a_split_k_axis(ctx):
    """weights' gradients of a narrow block over many rows: the rows in parts"""
    run_block(ctx, 1100, 8, 16, 3, BF16, "square", F32)


@pytest.mark.parametrize("size,dtype,grads,enough", [((130, 72, 140, 136), BF16, None, 3), ((260, 24, 70, 129), F16, F32, 3), ((200, 40, 140, 130), F32, None, 1),
                                                     ((300, 136, 140, 72), BF16, None, 1), ((270, 72, 260, 33), F16, F32, 1)],
                         ids=["128", "128-fine", "128-f32", "256", "256-fine"])
def test_large_tiles(ctx, size, dtype, grads, enough):
    """tiles of 128 x 128 and 256 x 256 with ragged edges, k axes of one to five steps, sums of several products"""
    ctx._L.emu_enough_tiles(enough)
    try:
        run_block(ctx, *size, dtype, "square", grads)
    finally:
        ctx._L.emu_enough_tiles(192)


# ---------------------------------------------------------------- AdamW
@pytest.mark.parametrize("lead", [0, 1])
@pytest.mark.parametrize("bits,pt,gt,copy", [(32, F32, F32, BF16), (32, BF16, F16, None), (8, F32, BF16, F16), (8, BF16, BF16, None)], ids=str)
def test_adamw(ctx, bits, pt, gt, copy, lead):
    numels = [1, 255, 257, 4096, 5003, 0, 9000] + [3] * 50  # more than a table of tensors holds

    def place(t):
        return ctx.guarded(torch.cat([t[:1].expand(lead), t]) if t.numel() else t)[lead if t.numel() else 0:]

    p = [place(normal(10 + i, n, dtype=pt)) for i, n in enumerate(numels)]
    g = [place(normal(100 + i, n, scale=10.0 ** (-i % 4), dtype=gt)) for i, n in enumerate(numels)]
    m0 = [normal(200 + i, n, scale=0.3).numpy() for i, n in enumerate(numels)]
    v0 = [(normal(300 + i, n) ** 2 + 0.01).numpy() for i, n in enumerate(numels)]
    cp = [place(torch.zeros(n, dtype=copy)) for n in numels] if copy else None
    seed, mu, vu = 0xABCDEF0123, None, None
    if bits == 8:
        rnd = [ref.random_words(7, i, n) >> np.uint64(16) for i, n in enumerate(numels)]
        mc = [ref.write_codes(a, r, 3) if len(a) else (np.zeros(0, np.uint8), np.zeros(0, np.float32)) for a, r in zip(m0, rnd)]
        vc = [ref.write_codes(a, r, 4) if len(a) else (np.zeros(0, np.uint8), np.zeros(0, np.float32)) for a, r in zip(v0, rnd)]
        m, v = [place(torch.from_numpy(c)) for c, _ in mc], [place(torch.from_numpy(c)) for c, _ in vc]
        mu, vu = [ctx.guarded(torch.from_numpy(u)) for _, u in mc], [ctx.guarded(torch.from_numpy(u)) for _, u in vc]
        m0, v0 = [ref.read_codes(c, u, 3) for c, u in mc], [ref.read_codes(c, u, 4) for c, u in vc]
    else:
        m, v = [place(torch.from_numpy(a)) for a in m0], [place(torch.from_numpy(a)) for a in v0]
    hp = dict(lr=2e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.1, step=3)
    want = [ref.adamw_f32(a.float().numpy(), b.float().numpy(), c, d, hp["lr"], hp["betas"], hp["eps"], hp["weight_decay"], hp["step"]) for a, b, c, d in zip(p, g, m0, v0)]
    opt = training.AdamW(ctx, p, g, m, v, mu, vu, cp)
    opt.step(**hp, seed=seed)
    for i, n in enumerate(numels):
        wp, wm, wv = want[i]
        assert torch.equal(p[i], torch.from_numpy(wp).to(pt))
        if copy:
            assert torch.equal(cp[i], torch.from_numpy(wp).to(copy))
        if bits == 32:
            assert np.array_equal(m[i].numpy(), wm) and np.array_equal(v[i].numpy(), wv)
        elif n:
            w = ref.random_words(seed, i, n)
            for got, unit, x, r, f in ((m[i], mu[i], wm, w >> np.uint64(16), 3), (v[i], vu[i], wv, w & np.uint64(0xFFFF), 4)):
                c, u = ref.write_codes(x, r, f)
                assert np.array_equal(got.numpy(), c) and np.array_equal(unit.numpy(), u)
    if bits == 8:
        mo, vo = [place(torch.zeros(n)) for n in numels], [place(torch.zeros(n)) for n in numels]
        opt.read_states(mo, vo)
        for i, n in enumerate(numels):
            if n:
                assert np.array_equal(mo[i].numpy(), ref.read_codes(m[i].numpy(), mu[i].numpy(), 3)) and np.array_equal(vo[i].numpy(), ref.read_codes(v[i].numpy(), vu[i].numpy(), 4))


def test_workspace_that_is_too_small_is_refused(ctx):
    """for sizes that take each tile and part rule: one byte less than what is asked for"""
    for rows, d_in, d_hidden, d_out in ((5, 64, 64, 64), (300, 700, 520, 130), (128, 4096, 4096, 4096), (256, 2048, 8192, 2048), (2048, 1024, 4096, 1024)):
        ff = training.GatedFF(ctx, d_in, d_hidden, d_out, BF16, "square")
        s = ff._s
        a = 1 << 40  # addresses that nothing is done with: the size is refused first
        for backward in (False, True):
            n = ff.workspace_bytes(rows, backward=backward)
            s.rows = rows
            args = [a, 2 * a, 3 * a, 4 * a] + ([5 * a, 6 * a, 7 * a, 8 * a, 9 * a, 10 * a, 0] if backward else [5 * a, None])
            fn = ctx._L.ckksmi_gated_ff_backward if backward else ctx._L.ckksmi_gated_ff_forward
            assert fn(ctx._h, ff._r, *args, 11 * a, n - 1, None) == ckksmi.EWORKSPACE


def test_sizes_that_no_grid_holds_are_refused(ctx):
    ff = training.GatedFF(ctx, 2**20, 2**20, 2**20, BF16, "square")
    with pytest.raises(ckksmi.CkksmiError) as e:
        ff.workspace_bytes(2**31 - 1000)
    assert e.value.code == ckksmi.EUNSUPPORTED
    with pytest.raises(ckksmi.CkksmiError) as e:
        ff.workspace_bytes(2**31 - 256)
    assert e.value.code == ckksmi.EINVAL
    ff = training.GatedFF(ctx, 2**19, 2**19, 2**19, BF16, "square")
    assert ff.workspace_bytes(4096) > 2**40  # the weights' padded copies alone
