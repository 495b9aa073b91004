"""Many matrices of different sizes and both orientations in one call: every one of them against 64 bits, and its bits move with it to another
place of its size in a launch.  A wrong entry of a launch's table is off by the size of a direction; rounding is by at most 2^-24 of 12 times what an f32 evaluation rounds, raised
by at most |a| in every later step: 12 * 2^-24 * (3.4445 + .. + 3.4445^5) < 5e-4, and half a step of the type."""
import ctypes as C
import math
import random

import pytest
import torch

import series_reference as sr
import train_emu_support as emu
from paper_1911_11377_amd import ckksmi, training
from series_reference import BF16, F32


@pytest.fixture(scope="module")
def ctx():
    c = ckksmi.Context(4, 3, 20, 1, 21, 1, device=0)
    yield c
    c.close()


def exact(u):
    """in 64 bits on u's device"""
    a, b, c = sr.COEFFICIENTS
    x = u.double()
    x = x.t().contiguous() if x.shape[0] > x.shape[1] else x
    x = x / (torch.linalg.norm(x) + 1e-7)
    for _ in range(5):
        k = x @ x.t().contiguous()
        x = a * x + (b * k + c * (k @ k)) @ x
    return x.t() if u.shape[0] > u.shape[1] else x


def near(got, want, dtype, what):
    assert float((got.double() - want).norm()) <= (5e-4 + sr.ROUND[dtype]) * float(want.norm()), (what, float((got.double() - want).norm() / want.norm()))


def check_calls(ctx, sizes, dtype, device):
    us = [sr.matrix(*s, i, "strong", dtype).to(device) for i, s in enumerate(sizes)]
    wants = [exact(u) for u in us]
    order = list(range(len(us)))
    kept = {}
    for turn in range(2):  # the second time every matrix stands in another place of its size
        outs = [torch.full_like(u, math.nan) for u in us]
        plan = training.Orthogonalise(ctx, [us[i] for i in order], [outs[i] for i in order])
        plan.run(torch.full((max(16, plan.workspace_bytes()),), 255, dtype=torch.uint8, device=device))
        for i, (o, w) in enumerate(zip(outs, wants)):
            near(o, w, dtype, (turn, i, sizes[i]))
            if turn:
                assert torch.equal(o, kept[i]), (i, sizes[i])
            kept[i] = o
        places = {}
        for i, s in enumerate(sizes):
            places.setdefault((s, i // 16), []).append(i)  # (sixteen matrices share a launch, and its choice of tiles)
        for same in places.values():
            moved = same[:]
            random.Random(3).shuffle(moved)
            for a, b in zip(same, moved):
                order[a] = b
    # steps along them, from zeros: the same tables with momentum, parameters and copies
    p, m, copies = [torch.zeros(s, device=device) for s in sizes], [torch.zeros(s, device=device) for s in sizes], [torch.zeros(s, dtype=BF16, device=device) for s in sizes]
    opt = training.Muon(ctx, p, us, m, copies=copies, scales=[1.0 + i for i in range(len(us))])
    opt.step(0.5, 0.0, torch.full((max(16, opt.workspace_bytes()),), 255, dtype=torch.uint8, device=device), nesterov=False)
    for i, w in enumerate(wants):
        near(p[i], -0.5 * (1 + i) * w, F32, ("p", i, sizes[i]))
        near(copies[i], -0.5 * (1 + i) * w, BF16, ("copy", i, sizes[i]))
        assert torch.equal(m[i], us[i].float())


MIXED = [(264, 520), (520, 264), (100, 300), (300, 100), (7, 33), (64, 64), (257, 129)]


@pytest.mark.gpu
@pytest.mark.parametrize("sizes", [[MIXED[i % 7] for i in range(52)], [(60, 90), (90, 60), (1, 70), (33, 33)] * 13, [(256, 1024), (1024, 256)] * 9,
                                   [(1024, 1030), (1030, 1024)] * 8, [(900, 1030), (1030, 900), (1030, 900)] * 5], ids=["mixed", "small", "wide", "large", "fifteen"])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_every_matrix_of_a_call(ctx, sizes, dtype):
    check_calls(ctx, sizes, dtype, "cuda:0")


@pytest.mark.skipif(not emu.available, reason="no host compiler with 16-bit float types")
@pytest.mark.parametrize("small", [True, False])
def test_every_matrix_of_a_call_on_the_stand_in(small):
    c = emu.EmuContext()
    c._L.emu_series_small.argtypes = [C.c_size_t]
    c._L.emu_series_small(2**63 if small else 0)
    try:
        check_calls(c, [(5, 12), (12, 5), (3, 3), (1, 9), (17, 8)] * 5 + [(5, 12)] * 2, F32, "cpu")
    finally:
        c._L.emu_series_small(2**63)
    assert c.errors() == 0
    c.close()


@pytest.mark.gpu
def test_operations_that_the_profile_counts(ctx):
    """three products of each kind a step, half of the symmetric ones: the same count in tiles and in one workgroup, under the kernel that ran"""
    for (m, n), name in (((60, 90), "series_small_kernel"), ((256, 512), "gemm_kernel")):
        u = sr.matrix(m, n, 1).to("cuda:0")
        plan = training.Orthogonalise(ctx, [u], [torch.empty_like(u)])
        ws = torch.empty(max(16, plan.workspace_bytes()), dtype=torch.uint8, device="cuda:0")
        ctx.profile_enable(True)
        plan.run(ws, steps=4)
        torch.cuda.synchronize()
        ran = ctx.profile_read()
        ctx.profile_enable(False)
        assert ran[name][1] == (1 if m == 60 else 12) and ran[name][2] == 4 * 3.0 * (m * m * n + m**3 + 2 * m * m * n), ran
        assert ("gemm_kernel" in ran) == (m == 256)
