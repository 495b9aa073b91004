"""Training operators on the GPU: ranges, workspaces and sizes beside those of test_training_gpu.py."""
import pytest
import torch

import training_range
from paper_1911_11377_amd import ckksmi, head

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
