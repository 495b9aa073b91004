"""Calls of one head beside each other: answers within a step's loss, answers of several streams with workspaces of their own."""
import math

import pytest
import torch

import train_emu_support as emu
from paper_1911_11377_amd import ckksmi, head
from test_residual_head import BF16, F32, empty_on, some, weights


@pytest.fixture(scope="module", params=["stand-in", pytest.param("gpu", marks=pytest.mark.gpu)])
def where(request):
    if request.param == "gpu":
        c = ckksmi.Context(4, 3, 20, 1, 21, 1, device=0)
        yield c, "cuda:0"
        c.close()
        return
    if not emu.available:
        pytest.skip("no host compiler with 16-bit float types")
    c = emu.EmuContext()
    yield c, "cpu"
    assert c.errors() == 0
    c.close()


@pytest.mark.parametrize("kind", [head.GatedHead, head.ResidualHead])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_an_answer_within_the_loss_leaves_the_step_as_it_is(where, kind, dtype):
    ctx, device = where
    rows, d = 24, 16
    x, other = some(7, rows, d).to(dtype).to(device), some(9, rows - 3, d).to(dtype).to(device)

    def step(asked):
        h = kind(ctx, rows, weights(d, 20, device), "poly3", dtype, empty_on(device))
        answer = torch.full((rows - 3, d), math.nan, dtype=dtype, device=device)

        def loss(y, dy):
            if asked:
                h.answer(other, answer)
            dy.copy_(y)

        h.step(x, loss, 0.02)
        block = h.block if kind is head.ResidualHead else h
        return block.grads + block.weights + list(h.vectors.values() if kind is head.ResidualHead else []), answer

    with_answer, answer = step(True)
    without, _ = step(False)
    assert all(torch.equal(a, b) for a, b in zip(with_answer, without))
    h = kind(ctx, rows, weights(d, 20, device), "poly3", dtype, empty_on(device))
    alone = torch.full_like(answer, math.nan)
    h.answer(other, alone)
    assert torch.equal(answer, alone)


def test_4_bit_answers_with_workspaces_of_their_own(where):
    ctx, device = where
    low = head.LowBitHead(ctx, 8, weights(16, 40, device), "silu", BF16, empty_on(device), group=32)
    xs = [some(20 + i, 8, 16).to(BF16).to(device) for i in range(4)]
    want = [torch.zeros(8, 16, dtype=BF16, device=device) for _ in xs]
    for x, y in zip(xs, want):
        low.answer(x, y)
    got, spaces = [torch.full_like(y, math.nan) for y in want], [torch.full((low.workspace_bytes(8),), 255, dtype=torch.uint8, device=device) for _ in xs]
    if device == "cpu":
        for x, y, ws in zip(xs, got, spaces):
            low.answer(x, y, ws=ws)
    else:
        streams = [torch.cuda.Stream() for _ in xs]
        torch.cuda.synchronize()
        for _ in range(10):
            for x, y, ws, s in zip(xs, got, spaces, streams):
                low.answer(x, y, stream=s.cuda_stream, ws=ws)
        torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert all(bool((ws != 255).any()) for ws in spaces)


def test_answers_of_more_rows_than_a_step_has(where):
    """as far as the steps' workspace goes"""
    ctx, device = where
    d, more = 15, 27
    w = weights(d, 21, device)
    h = head.GatedHead(ctx, 24, w, "square", BF16, empty_on(device))
    wide = head.GatedHead(ctx, more, weights(d, 21, device), "square", BF16, empty_on(device))
    assert h.answer_ws.numel() < h.ff.workspace_bytes(more) <= h.ws.numel()
    x = some(3, more, d).to(BF16).to(device)
    y, want = torch.zeros(more, d, dtype=BF16, device=device), torch.ones(more, d, dtype=BF16, device=device)
    h.answer(x, y)
    wide.answer(x, want)
    assert torch.equal(y, want)
