"""Training operators on the GPU: ranges, workspaces and sizes beside those of test_training_gpu.py."""
import pytest
import torch

import training_range
import training_reference as ref
from paper_1911_11377_amd import ckksmi, head, training

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def ctx():
    c = ckksmi.Context(4, 3, 20, 1, 21, 1, device=0)
    yield c
    c.close()


@pytest.mark.parametrize("dtype", [F16, BF16], ids=["f16", "bf16"])
@pytest.mark.parametrize("rows", [1, 20, 70, 600])
@pytest.mark.parametrize("scales", training_range.SCALES, ids=str)
def test_f32_gradients_of_16_bit_operands_have_the_range_of_f32(ctx, scales, rows, dtype):
    training_range.check(ctx, DEV, lambda t: t, rows, dtype, scales)


@pytest.mark.parametrize("dtype", [F16, BF16], ids=["f16", "bf16"])
@pytest.mark.parametrize("size", [(3000, 256, 512, 256), (1500, 250, 511, 131), (300, 1500, 1500, 1500)], ids=lambda s: "x".join(map(str, s)))
def test_f32_gradients_of_16_bit_operands_in_many_tiles(ctx, size, dtype):
    training_range.check(ctx, DEV, lambda t: t, size[0], dtype, (1.0, 2.0**-17), d_in=size[1], d_hidden=size[2], d_out=size[3])


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_steps_on_a_stream_of_their_own(ctx, dtype):
    """a head trained on a side stream, whose losses are torch operations, ends with the bits of one trained on the current stream"""
    ends = []
    for side in (None, torch.cuda.Stream()):
        g = torch.Generator().manual_seed(4)
        weights = [(torch.randn(s, generator=g) * s[1] ** -0.5).to(DEV) for s in ((256, 512), (256, 512), (64, 256))]
        x, target = torch.randn(1000, 512, generator=g).to(DEV).to(dtype), torch.randn(1000, 64, generator=g).to(DEV)
        h = head.GatedHead(ctx, 1000, weights, "square", dtype, lambda shape, t: torch.zeros(shape, dtype=t, device=DEV))
        torch.cuda.synchronize()

        def loss(y, dy):
            off = y.float() - target[: y.shape[0]]
            for _ in range(20):  # a loss of many launches
                off = off + 0.0
            dy.copy_(off * (2.0 / off.numel()))
            return off.square().mean()

        losses = [h.step(x[:rows], loss, 1e-3, stream=side and side.cuda_stream) for rows in (1000, 1000, 700, 1000, 30, 1000)]
        torch.cuda.synchronize()
        ends.append(weights + losses)
    assert all(torch.equal(a, b) for a, b in zip(*ends))


def block(dtype, rows, d_in, d_hidden, d_out, grads=None, seed=1):
    """operands and zeroed results"""
    g = torch.Generator(DEV).manual_seed(seed)

    def normal(shape, scale=1.0):
        return (torch.randn(shape, generator=g, device=DEV) * scale).to(dtype)

    x, dy = normal((rows, d_in)), normal((rows, d_out))
    w = [normal((d_hidden, d_in), d_in**-0.5), normal((d_hidden, d_in), d_in**-0.5), normal((d_out, d_hidden), d_hidden**-0.5)]
    y, dx = torch.zeros(rows, d_out, dtype=dtype, device=DEV), torch.zeros(rows, d_in, dtype=dtype, device=DEV)
    return x, dy, w, y, dx, [torch.zeros(t.shape, dtype=grads or dtype, device=DEV) for t in w]


def room(n):
    return torch.full((max(16, n),), 255, dtype=torch.uint8, device=DEV)


@pytest.mark.parametrize("size", [(2049, 4001, 4000, 3990), (1100, 8192, 4096, 8200)], ids=lambda s: "x".join(map(str, s)))
def test_f32_blocks_of_many_large_tiles(ctx, size):
    """512 tiles of 128 x 128 and more in every product: operands along k, along rows and both, ragged edges"""
    x, dy, w, y, dx, dw = block(F32, *size)
    ff = training.GatedFF(ctx, *size[1:], F32, "poly3")
    saved, ws = room(ff.saved_bytes(size[0])), room(ff.workspace_bytes(size[0], backward=True))
    ff.forward(x, *w, y, ws, saved=saved)
    ff.backward(x, *w, saved, dy, dx, *dw, ws)
    want = ref.block(x, *w, training.CUBICS["poly3"], dy)
    for name, got in (("y", y), ("dx", dx), ("dwg", dw[0]), ("dwu", dw[1]), ("dwd", dw[2])):
        v, bound = want.pop(name)
        assert bool(((got.double() - v).abs() <= bound).all()), (name, float(((got.double() - v).abs() / bound).max()))
        # the bound allows for every rounding's worst case; roundings that do not conspire come to some square root of it
        assert float((got.double() - v).norm() / v.norm()) < 1e-5, name


@pytest.mark.parametrize("dtype,widths", [(BF16, (1024, 4096, 1024)), (F32, (3136, 256, 2)), (F16, (517, 1021, 129))], ids=["bf16", "f32", "f16"])
def test_fewer_rows_than_a_workspace_was_made_for(ctx, dtype, widths):
    """the answers and gradients of a workspace that was made for just these rows"""
    ff = training.GatedFF(ctx, *widths, dtype, "square")
    made_for = 1537
    ws, saved = room(ff.workspace_bytes(made_for, backward=True)), room(ff.saved_bytes(made_for))
    for rows in (1537, 1536, 512, 65, 7, 1):
        x, dy, w, y, dx, dw = block(dtype, rows, *widths, seed=rows)
        results = []
        for s, k in ((saved, ws), (room(ff.saved_bytes(rows)), room(ff.workspace_bytes(rows, backward=True)))):
            ff.forward(x, *w, y, k, saved=s)
            ff.backward(x, *w, s, dy, dx, *dw, k)
            results.append([t.clone() for t in (y, dx, *dw)])
        assert all(torch.equal(a, b) and bool(torch.isfinite(a).all()) for a, b in zip(*results)), rows


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("rows", [3, 70, 2000])
def test_infinite_sums(ctx, rows, dtype):
    """max(g, 0) of gate sums that pass the type's range downwards is 0; an infinite row's answers and gradients are infinite, no NaN from what
    pads rows of 517 hidden units"""
    inf = float("inf")
    x, dy, w, y, dx, dw = block(dtype, rows, 24, 517, 40)
    ff = training.GatedFF(ctx, 24, 517, 40, dtype, "relu")
    saved, ws = room(ff.saved_bytes(rows)), room(ff.workspace_bytes(rows, backward=True))
    w = [t.abs() + 0.25 for t in w]
    w[1] *= 2.0**-120
    x[0], x[1], x[2] = -3e38, inf, 1.0
    dy[0], dy[2] = 1.0, inf
    ff.forward(x, *w, y, ws, saved=saved)
    ff.backward(x, *w, saved, dy, dx, *dw, ws)
    assert bool((y[0] == 0).all()) and bool((y[1] == inf).all()) and bool(torch.isfinite(y[2:]).all())
    assert bool((dx[0] == 0).all()) and bool((dx[2] == inf).all()) and bool(torch.isfinite(dx[3:]).all())
