"""How near orthogonalised directions come to 64 bits, judged by what arithmetic in 32 bits loses and by nothing that the kernels do: matrices of any
spectrum, of low and exact rank, of equal elements, with rows and columns of very different sizes; on the CPU stand-in and on the GPU.

`loss` evaluates the steps in 64 bits with every value moved that an f32 evaluation would round: by up to 2^-24 of itself, each element by itself or all
of a matrix alike (matrices of equal elements round alike).  The kernels' operands are f16 pairs of 22 bits, off by 2^-22, four times as much, and
each product has two of them and leaves out the product of the second parts, another 2^-22: 3 * 4 = 12 times that loss is allowed.  What is below f16's numbers adds an absolute
error: 2^-25 of a second part's unit, held 2^11 times larger, in X (units of 2^-14), A outside its diagonal (2^-13) and the polynomial (2^-12 for the usual
coefficients; |b| + 4 |c| times A's); a later step raises it by at most |a| (the largest slope of the polynomials here).  The last rounding is
monotone, so an element lies between the rounded ends of what is allowed."""
import ctypes as C
import math

import pytest
import torch

import series_reference as sr
import train_emu_support as emu
from paper_1911_11377_amd import ckksmi, training
from series_reference import BF16, F16, F32

F64 = torch.float64


def loss(u, steps, seed, alike):
    a, b, c = sr.COEFFICIENTS
    gen = torch.Generator().manual_seed(seed)

    def moved(v):
        by = torch.rand(() if alike else v.shape, generator=gen, dtype=F64) * 2 - 1
        return v * (1 + 2.0**-24 * (torch.sign(by) if alike else by))

    x = u.double().cpu()
    tall = x.shape[0] > x.shape[1]
    x = moved(sr.start(x.t() if tall else x, 1e-7))
    for _ in range(steps):
        k = moved(x @ x.t())
        p = moved(b * k + c * moved(k @ k))
        x = moved(a * x + moved(p @ x))
    return x.t() if tall else x


def allowed(u, steps):
    """the exact direction and the largest error of each element: of its row's and its column's, whichever is less"""
    want = sr.exact(u, steps=steps)
    off = torch.stack([(loss(u, steps, s, s % 2 == 1) - want).abs() for s in range(8)]).amax(0)
    off = torch.minimum(off.amax(1, keepdim=True), off.amax(0, keepdim=True))
    a, b, c = (abs(k) for k in sr.COEFFICIENTS)
    floor = 2.0**-36 * (2.0**-14 + min(u.shape) ** 0.5 * (2.0**-12 + (b + 4 * c) * 2.0**-13))
    return want, 12 * off + floor * sum(a**k for k in range(1, steps + 1)) * 2


def check(got, u, steps, what=""):
    want, off = allowed(u, steps)
    got = got.cpu()
    low, high = (want - off).to(got.dtype), (want + off).to(got.dtype)
    bad = ~((got >= low) & (got <= high))
    assert not bool(bad.any()), (what, int(bad.sum()), float(((got.double() - want).abs() / off)[bad].max()), float((got.double() - want).norm() / want.norm()))


def outer(m, n, rank, seed, whole=False, sign=False):
    g = torch.Generator().manual_seed(seed)
    p, q = torch.randn((m, rank), generator=g, dtype=F64), torch.randn((rank, n), generator=g, dtype=F64)
    if whole:
        p, q = torch.round(4 * p), torch.round(4 * q)
    return torch.sign(p) @ torch.sign(q) if sign else p @ q


def graded(m, n, rows=True, cols=False):
    """rows (columns) of sizes 1, 1e-4, 1e-6, 1e-8 in turn"""
    x = sr.matrix(m, n, 11).double()
    if rows:
        x = x * (10.0 ** torch.tensor([0.0, -4.0, -6.0, -8.0], dtype=F64))[torch.arange(m) % 4][:, None]
    if cols:
        x = x * (10.0 ** torch.tensor([0.0, -4.0, -6.0, -8.0], dtype=F64))[torch.arange(n) % 4]
    return x


def matrices(m, n):
    one = graded(m, n)
    one[1:] = one[1:].sign() * 1e-6
    return {
        "normal": sr.matrix(m, n, 1),
        "strong": sr.matrix(m, n, 2, "strong"),
        "falling": sr.matrix(m, n, 3, "falling"),
        "rank 3 and noise": sr.matrix(m, n, 4, "rank3"),
        "rank 1 and noise": outer(m, n, 1, 5) + 1e-4 * sr.matrix(m, n, 6).double(),
        "rank 1": outer(m, n, 1, 7, whole=True),
        "rank 2 of signs": outer(m, n, 2, 8, sign=True),
        "rank 4": outer(m, n, 4, 9),
        "ones": torch.ones(m, n),
        "identity": torch.eye(m, n),
        "graded rows": graded(m, n),
        "graded columns": graded(m, n, False, True),
        "both graded": graded(m, n, True, True),
        "one strong row": one,
    }


KINDS = list(matrices(2, 2))


@pytest.fixture(scope="module", params=["small", "tiles"])
def stand_in(request):
    if not emu.available:
        pytest.skip("no host compiler with 16-bit float types")
    c = emu.EmuContext()
    c._L.emu_series_small.argtypes = [C.c_size_t]
    c._L.emu_series_small(2**63 if request.param == "small" else 0)
    yield c
    c._L.emu_series_small(2**63)
    assert c.errors() == 0
    c.close()


@pytest.fixture(scope="module")
def ctx():
    c = ckksmi.Context(4, 3, 20, 1, 21, 1, device=0)
    yield c
    c.close()


def direct(ctx, u, steps, device="cpu"):
    u = u.to(device)
    out = torch.full_like(u, math.nan)
    plan = training.Orthogonalise(ctx, [u], [out])
    plan.run(torch.full((max(16, plan.workspace_bytes()),), 255, dtype=torch.uint8, device=device), steps=steps)
    return out


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("size,dtype,steps", [((24, 40), F32, 5), ((24, 40), BF16, 5), ((31, 17), F16, 5), ((24, 40), F32, 12), ((40, 24), BF16, 8)], ids=str)
def test_on_the_stand_in(stand_in, kind, size, dtype, steps):
    u = matrices(*size)[kind].to(dtype)
    check(direct(stand_in, u, steps), u, steps, kind)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("size", [(24, 90), (64, 100), (100, 140), (330, 200), (300, 1021)], ids=str)
@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=["f32", "bf16", "f16"])
def test_against_the_loss_of_32_bits(ctx, kind, size, dtype):
    u = matrices(*size)[kind].to(dtype)
    for steps in (5, 8, 12):
        check(direct(ctx, u, steps, "cuda:0"), u, steps, (kind, steps))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("kind", ["normal", "rank 1", "ones", "graded rows"])
def test_tiles_of_every_size(ctx, kind, dtype):
    """sixteen of 256 x 1100: 128 x 128 tiles and larger; one of 1100 x 1030: 32 x 128 and 128 x 128, some with their k axes in parts"""
    us = [matrices(256, 1100)[kind].to(dtype).to("cuda:0")] * 16
    outs = [torch.full_like(u, math.nan) for u in us]
    plan = training.Orthogonalise(ctx, us, outs)
    plan.run(torch.full((plan.workspace_bytes(),), 255, dtype=torch.uint8, device="cuda:0"))
    check(outs[0], us[0], 5)
    assert all(torch.equal(o, outs[0]) for o in outs)
    u = matrices(1100, 1030)[kind].to(dtype)
    check(direct(ctx, u, 5, "cuda:0"), u, 5)


def check_from_zeros(ctx, dtype, gt, device):
    """parameters that were zeros show the direction itself, 16-bit ones too: p = -lr scale direction, each product and sum rounded once to 32 bits"""
    for kind in ("rank 1", "rank 3 and noise", "ones"):
        g = matrices(24, 40)[kind].to(gt).to(device)
        p, m = torch.zeros(24, 40, dtype=dtype, device=device), torch.zeros(24, 40, device=device)
        opt = training.Muon(ctx, [p], [g], [m], scales=[1.0])
        opt.step(0.5, 0.0, torch.zeros(max(16, opt.workspace_bytes()), dtype=torch.uint8, device=device), nesterov=False)
        want, off = allowed(g.float(), 5)
        want, off = -0.5 * want, 0.5 * off + 2 * 2.0**-24 * want.abs()
        assert bool(((p.cpu() >= (want - off).to(dtype)) & (p.cpu() <= (want + off).to(dtype))).all()), kind


STEPS = [(F32, BF16), (BF16, BF16), (F16, F32)]


@pytest.mark.parametrize("dtype,gt", STEPS, ids=str)
def test_steps_from_zeros_on_the_stand_in(stand_in, dtype, gt):
    check_from_zeros(stand_in, dtype, gt, "cpu")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,gt", STEPS, ids=str)
def test_steps_from_zeros(ctx, dtype, gt):
    check_from_zeros(ctx, dtype, gt, "cuda:0")
