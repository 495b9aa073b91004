"""Training operators on the GPU: ranges, workspaces and sizes beside those of test_training_gpu.py."""
import pytest
import torch

import training_range
from paper_1911_11377_amd import ckksmi

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
