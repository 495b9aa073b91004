"""The example from training to encrypted answers (examples/encrypted_head.py), on the CPU stand-ins and on the GPU."""
import os
import sys

import numpy as np
import pytest
import torch

import parity_cases as pc
import train_emu_support as emu
from paper_1911_11377_amd import head

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import encrypted_head as example  # noqa: E402


def check_encrypted(be, shape, act, weights, x, tolerance):
    ctx = be.context(*shape)

    def to_dev(a):
        a = np.ascontiguousarray(a)
        return be.to_dev(a, dtype=a.dtype)

    got = example.encrypted(ctx, weights, act, x, to_dev, be.empty, be.to_host, be.ws, stream=be.stream)
    want = example.clear(weights, act, x)
    ctx.close()
    # scale 2^45 in, 2^30 or more where a cubic's products leave it; the same bound as the framework's other decrypted answers
    assert np.abs(got - want).max() < tolerance, np.abs(got - want).max()


def some_weights(d_in, d_hidden, seed=3):
    g = np.random.default_rng(seed)
    return [g.normal(0, 0.5, s).astype(np.float32) for s in ((d_hidden, d_in), (d_hidden, d_in), (2, d_hidden))]


@pytest.mark.parametrize("act,primes", [("linear", 4), ("square", 5), ("poly2", 6), ("poly3", 6)])
def test_encrypted_answers_are_the_clear_ones(act, primes):
    x, _ = example.features(16, 4, 1)
    check_encrypted(pc.EmuBackend(), (5, primes, 50, 1, 51, 1), act, some_weights(4, 3), x, 1e-3)


def test_heads_that_cannot_be_planned():
    with pytest.raises(ValueError):
        head.plan(*some_weights(4, 3), "silu", [2**50] * 8, 8, 2.0**45)
    with pytest.raises(ValueError):
        head.plan(*some_weights(4, 3), "square", [2**50] * 4, 4, 2.0**45)


@pytest.mark.skipif(not emu.available, reason="no host compiler with 16-bit float types")
def test_training_on_the_stand_in():
    ctx = emu.EmuContext()
    weights, first, last = example.train(ctx, "cpu", "square", torch.bfloat16, rows=32, steps=40)
    assert np.isfinite(last) and last < 0.8 * first, (first, last)
    assert ctx.errors() == 0
    ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("act,dtype", [("square", torch.bfloat16), ("linear", torch.float32)], ids=["square-bf16", "linear-f32"])
def test_from_training_to_encrypted_answers(act, dtype):
    be = pc.GpuBackend()
    ctx = be.context(4, 3, 20, 1, 21, 1)
    weights, first, last = example.train(ctx, "cuda:0", act, dtype)
    ctx.close()
    assert last < 0.5 * first, (first, last)
    x, target = example.features(512, 8, 5)
    assert np.mean(np.sign(example.clear(weights, act, x)) == target) > 0.85
    check_encrypted(be, (10, 6, 50, 1, 51, 1), act, weights, x, 1e-3)
