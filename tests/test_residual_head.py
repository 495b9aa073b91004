"""Norms, block, orthogonalised steps and 4-bit answers together: a residual head trained in the clear, evaluated in the clear, from 4-bit matrices and
under encryption; on the CPU stand-ins and on the GPU."""
import os
import sys

import numpy as np
import pytest
import torch

import norm_reference as nr
import parity_cases as pc
import series_reference as sr
import train_emu_support as emu
import training_reference as ref
from paper_1911_11377_amd import ckksmi, head

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import encrypted_head as example  # noqa: E402

F32, BF16 = torch.float32, torch.bfloat16


def some(seed, *shape, scale=1.0):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * scale


def weights(d, d_hidden, device, dtype=F32):
    return [some(i, *s, scale=s[1] ** -0.5).to(dtype).to(device) for i, s in enumerate(((d_hidden, d), (d_hidden, d), (d, d_hidden)))]


def empty_on(device):
    return lambda shape, t: torch.zeros(shape, dtype=t, device=device)


def check_step(ctx, device, norm, optimizer, rows=24, d=16, d_hidden=20):
    """one step in f32: answers, the gradients of every matrix and vector and the moved matrices against 64 bits (autograd of the formulas).  The
    tolerance is a thousandth of each tensor's size: chained operators whose own bounds, at these sizes, are each below 1e-5 of theirs;
    a wrong sign, factor or operand is off by its whole size"""
    w = weights(d, d_hidden, device)
    start = [t.clone() for t in w]
    h = head.ResidualHead(ctx, rows, w, "poly3", F32, empty_on(device), norm=norm, residual_scale=0.9, block_scale=0.8, optimizer=optimizer)
    g = {k: some(50 + i, d, scale=0.2) + (0.0 if k.endswith("bias") else 1.0) for i, k in enumerate(h.vectors)}
    for k, v in h.vectors.items():
        v.copy_(g[k])
    x, target = some(7, rows, d).to(device), some(8, rows, d).to(device)

    def loss(r, dr):
        off = r.float() - target
        dr.copy_(off * (2.0 / off.numel()))
        return off.square().mean()

    value = h.step(x, loss, 0.02, weight_decay=0.1)
    at = {k: v.double().requires_grad_() for k, v in g.items()}
    m = [t.double().cpu().requires_grad_() for t in start]

    def normed(v, side):
        mean = v.mean(1, keepdim=True) if norm == "layer" else 0.0
        return (v - mean) / torch.sqrt(((v - mean) ** 2).mean(1, keepdim=True) + float(torch.tensor(1e-5))) * at[side + "_weight"] + at.get(side + "_bias", 0.0)

    X = x.double().cpu()
    n = normed(X, "pre")
    gate = n @ m[0].t()
    a = 0.5 + 0.25 * gate - 0.02 * gate**3
    r = 0.9 * X + 0.8 * at["gate"] * normed((a * (n @ m[1].t())) @ m[2].t(), "post")
    want = (r - target.double().cpu()).square().mean()
    want.backward()
    assert abs(float(value) - float(want.detach())) < 1e-5 * float(want.detach())

    def near(got, v, what):
        assert float((got.double().cpu() - v).abs().max()) <= 1e-3 * float(v.abs().max()), what

    near(h.r, r.detach(), "r")
    for k, v in at.items():
        near(h.grads[k], v.grad, k)
    for t, grad, s, name in zip(w, m, start, ("gate", "up", "down")):
        near(h.block.grads[("gate", "up", "down").index(name)], grad.grad, name)
        if optimizer == "muon":
            # direction of the gradients that the step had (its own are within the bound above)
            _, u = sr.momentum(torch.zeros_like(grad).float().detach(), h.block.grads[("gate", "up", "down").index(name)], 0.9, 1.0, True)
            sr.check_step(t, s, u, 2, 0.02, max(1.0, t.shape[0] / t.shape[1]) ** 0.5, 0.1)
    return h, x


@pytest.mark.skipif(not emu.available, reason="no host compiler with 16-bit float types")
@pytest.mark.parametrize("norm", ["rms", "layer"])
@pytest.mark.parametrize("optimizer", ["muon", "adamw"])
def test_a_step_on_the_stand_in(norm, optimizer):
    ctx = emu.EmuContext()
    check_step(ctx, "cpu", norm, optimizer)
    assert ctx.errors() == 0
    ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("norm", ["rms", "layer"])
@pytest.mark.parametrize("optimizer", ["muon", "adamw"])
def test_a_step(norm, optimizer):
    ctx = ckksmi.Context(4, 3, 20, 1, 21, 1, device=0)
    check_step(ctx, "cuda:0", norm, optimizer)
    check_step(ctx, "cuda:0", norm, optimizer, rows=300, d=100, d_hidden=260)
    ctx.close()


@pytest.mark.skipif(not emu.available, reason="no host compiler with 16-bit float types")
def test_heads_that_make_no_sense():
    ctx = emu.EmuContext()
    with pytest.raises(ValueError):
        head.GatedHead(ctx, 4, weights(8, 8, "cpu"), "square", F32, empty_on("cpu"), optimizer="sgd")
    with pytest.raises(ValueError):
        head.ResidualHead(ctx, 4, [some(1, 6, 8), some(2, 6, 8), some(3, 4, 6)], "square", F32, empty_on("cpu"))
    ctx.close()


def train(ctx, device, dtype, rows=64, d=8, steps=30):
    w = weights(d, 16, device)
    h = head.ResidualHead(ctx, rows, w, "square", dtype, empty_on(device))
    for t in range(steps):
        x = some(100 + t % 4, rows, d)
        x[:, -1] = 1.0
        target = (x + 0.5 * torch.sign(x[:, :1] * x[:, 1:2])).to(device)

        def loss(r, dr):
            off = r.float() - target
            dr.copy_(off * (2.0 / off.numel()))
            return off.square().mean()

        value = h.step(x.to(dtype).to(device), loss, 0.02)
    assert bool(torch.isfinite(value))
    return h, w


def check_low_bits(ctx, h, w, device, dtype):
    """answers from 4-bit matrices are those of the block with the matrices that the codes stand for"""
    low = head.LowBitHead(ctx, 8, w, "square", dtype, empty_on(device), group=32)
    x = some(5, 8, 8).to(dtype).to(device)
    y = torch.zeros(8, 8, dtype=dtype, device=device)
    low.answer(x, y)
    wide = [torch.zeros_like(t, dtype=F32) for t in w]
    for t, pair, plan in zip(wide, low.matrices, (low.ff.into, low.ff.into, low.ff.out)):
        plan.unpack(*pair, t)
        assert float((t - w[[i for i, v in enumerate(wide) if v is t][0]]).abs().max()) <= float(t.abs().max()) * (0.5 / 7 + 0.01)
    want, bound = ref.block(x.cpu(), *(t.cpu() for t in wide), [0.0, 0.0, 1.0, 0.0])["y"]
    off = (y.double().cpu() - want).abs()
    # (the bound is of one rounding less of h: 2^-17 of it, and of products in other orders)
    assert bool((off <= 1.25 * bound + 2 * nr.ROUND[dtype] * want.abs() + 1e-5).all())


def check_encrypted(be, h, w, device, rows=6):
    """whoever holds the key norms, encrypts, decrypts and joins: the clear answers"""
    x = some(9, rows, 8)
    x[:, -1] = 1.0
    x = x.to(device)
    n, r, clear = (torch.zeros(rows, 8, device=device) for _ in range(3))
    h.normed(x, n)
    h.answer(x, clear)
    ctx = be.context(10, 6, 50, 1, 51, 1) if device != "cpu" else be.context(5, 6, 50, 1, 51, 1)

    def to_dev(a):
        a = np.ascontiguousarray(a)
        return be.to_dev(a, dtype=a.dtype)

    f = example.encrypted(ctx, [t.cpu().numpy() for t in w], "square", n.cpu().numpy().astype(np.float64), to_dev, be.empty, be.to_host, be.ws, stream=be.stream)
    ctx.close()
    h.joined(x, torch.from_numpy(f).float().to(device), r)
    # decrypted answers are off by at most 1e-3 (the framework's other ones' bound); the norm of 8 values around them passes an error on
    # by at most its inverse size
    f32 = torch.from_numpy(f)
    size = float((f32.square().mean(1) + 1e-5).rsqrt().max())
    gain = float(h.vectors["gate"].abs().max() * h.vectors["post_weight"].abs().max())
    assert float((r - clear).abs().max()) <= 2 * 1e-3 * size * gain * 8**0.5 + 1e-5


@pytest.mark.skipif(not emu.available, reason="no host compiler with 16-bit float types")
def test_from_training_to_encrypted_answers_on_the_stand_in():
    ctx = emu.EmuContext()
    h, w = train(ctx, "cpu", F32, rows=16, steps=6)
    check_low_bits(ctx, h, w, "cpu", BF16)
    check_encrypted(pc.EmuBackend(), h, w, "cpu")
    assert ctx.errors() == 0
    ctx.close()


@pytest.mark.gpu
def test_from_training_to_encrypted_answers():
    be = pc.GpuBackend()
    ctx = ckksmi.Context(4, 3, 20, 1, 21, 1, device=0)
    train(ctx, "cuda:0", BF16)
    h, w = train(ctx, "cuda:0", F32)
    check_low_bits(ctx, h, w, "cuda:0", BF16)
    check_encrypted(be, h, w, "cuda:0")
    ctx.close()


@pytest.mark.gpu
def test_a_step_on_another_stream_and_in_a_graph():
    """the same bits on torch's current stream, on another one and replayed, and what the steps leave in between"""
    ctx = ckksmi.Context(4, 3, 20, 1, 21, 1, device=0)
    x = some(3, 40, 24).to(BF16).to("cuda:0")

    def run(how, steps=3):
        w = weights(24, 40, "cuda:0")
        h = head.ResidualHead(ctx, 40, w, "square", BF16, empty_on("cuda:0"))

        def one(stream=None):
            h.step(x, lambda r, dr: dr.copy_(r), 0.02, stream=stream)

        side = torch.cuda.Stream()
        torch.cuda.synchronize()
        if how == "graph":  # (a step's number is the host's: captured, it stays the first's)
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                one()
            for _ in range(steps):
                graph.replay()
                torch.cuda.synchronize()
        else:
            for _ in range(steps):
                h.block.steps = 0 if how.endswith("first") else h.block.steps
                one(side.cuda_stream if how.startswith("side") else None)
        torch.cuda.synchronize()
        return w + list(h.vectors.values()) + [h.r]

    here, there = run("here"), run("side")
    assert all(torch.equal(a, b) for a, b in zip(here, there))
    here, replayed = run("here, always the first"), run("graph")
    assert all(torch.equal(a, b) for a, b in zip(here, replayed))
    ctx.close()
