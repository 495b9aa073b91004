"""Training operators on the GPU: the gated feed-forward block and the AdamW step against references in 64 bits (block) and in
operation-by-operation 32 bits (AdamW, equal bits), at the sizes, strides and values where they could go wrong."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

import training_reference as ref
from paper_1911_11377_amd import ckksmi, training

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def ctx():
    c = ckksmi.Context(4, 3, 20, 1, 21, 1, device=0)
    yield c
    c.close()


def gen(seed):
    return torch.Generator(DEV).manual_seed(seed)


def normal(g, *shape, scale=1.0, dtype=F32):
    return (torch.randn(shape, generator=g, device=DEV) * scale).to(dtype)


def framed(t, lead=0, gap=0):
    """t inside a larger buffer of NaN: rows `gap` elements further apart, `lead` elements behind the buffer's start"""
    rows, cols = t.shape
    buf = torch.full((lead + rows * (cols + gap) + 64,), math.nan, dtype=t.dtype, device=DEV)
    v = buf[lead:lead + rows * (cols + gap)].view(rows, cols + gap)[:, :cols]
    v.copy_(t)
    return v, buf


class Block:
    def __init__(self, ctx, rows, d_in, d_hidden, d_out, dtype, act, grad_dtype=None, seed=0):
        g = gen(seed)
        self.act = training.CUBICS.get(act, act) if isinstance(act, str) else act
        self.ff = training.GatedFF(ctx, d_in, d_hidden, d_out, dtype, act, grad_dtype)
        self.rows, self.shape, self.dtype, self.gt = rows, (d_in, d_hidden, d_out), dtype, grad_dtype or dtype
        self.x = normal(g, rows, d_in, dtype=dtype)
        self.wg, self.wu = normal(g, d_hidden, d_in, scale=d_in**-0.5, dtype=dtype), normal(g, d_hidden, d_in, scale=d_in**-0.5, dtype=dtype)
        self.wd = normal(g, d_out, d_hidden, scale=d_hidden**-0.5, dtype=dtype)
        self.dy = normal(g, rows, d_out, dtype=dtype)
        self.y, self.dx = torch.full((rows, d_out), math.nan, dtype=dtype, device=DEV), torch.full((rows, d_in), math.nan, dtype=dtype, device=DEV)
        self.dw = [torch.full(w.shape, math.nan, dtype=self.gt, device=DEV) for w in (self.wg, self.wu, self.wd)]
        # workspaces hold NaN: what a call reads before it writes shows
        self.ws = torch.full((max(16, self.ff.workspace_bytes(rows, backward=True)),), 255, dtype=torch.uint8, device=DEV)
        self.saved = torch.full((max(16, self.ff.saved_bytes(rows)),), 255, dtype=torch.uint8, device=DEV)

    def forward(self, saved=True, **kw):
        self.ff.forward(self.x, self.wg, self.wu, self.wd, self.y, self.ws, saved=self.saved if saved else None, **kw)

    def backward(self, dx=True, **kw):
        self.ff.backward(self.x, self.wg, self.wu, self.wd, self.saved, self.dy, self.dx if dx else None, *self.dw, self.ws, **kw)

    def results(self):
        return {"y": self.y, "dx": self.dx, "dwg": self.dw[0], "dwu": self.dw[1], "dwd": self.dw[2]}

    def check(self, names=("y", "dx", "dwg", "dwu", "dwd"), skip=()):
        want = ref.block(self.x, self.wg, self.wu, self.wd, self.act, self.dy, self.gt)
        got = self.results()
        for n in names:
            v, bound = want[n]
            off = (got[n].double() - v).abs()
            worst = float((off - bound).max()) if off.numel() else 0.0
            assert worst <= 0, "%s: off by %g where %g is allowed" % (n, float(off.flatten()[(off - bound).argmax()]), float(bound.flatten()[(off - bound).argmax()]))


SIZES = [(1, 1, 1, 1), (1, 64, 64, 64), (1, 1000, 72, 8), (2, 8, 8, 8), (3, 5, 7, 9), (7, 999, 131, 50), (16, 64, 128, 16), (17, 40, 24, 1), (31, 130, 65, 33),
         (32, 256, 264, 40), (33, 72, 200, 100), (64, 784, 256, 2), (100, 33, 1, 31), (129, 257, 129, 65), (300, 520, 264, 136), (512, 128, 512, 256)]


@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=["f32", "bf16", "f16"])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_block_against_64_bits(ctx, size, dtype):
    b = Block(ctx, *size, dtype, "poly3", seed=sum(size))
    b.forward()
    b.backward()
    b.check()
    y = b.y.clone()
    b.y.fill_(math.nan)
    b.forward(saved=False)  # answering requests: the same bits
    assert torch.equal(b.y, y)


@pytest.mark.parametrize("act", ["linear", "square", "poly2", "poly3", "relu", "silu", "gelu", (0.3, -0.7, 0.2, 0.05)], ids=str)
@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=["f32", "bf16", "f16"])
def test_activations(ctx, act, dtype):
    b = Block(ctx, 70, 96, 80, 24, dtype, act, seed=5)
    b.forward()
    b.backward()
    b.check()


@pytest.mark.parametrize("act", ["poly3", "relu", "silu", "gelu"])
@pytest.mark.parametrize("rows", [1, 40, 130])
def test_answers_do_not_depend_on_what_is_saved(ctx, act, rows):
    b = Block(ctx, rows, 107, 72, 19, F32, act, seed=21)
    b.forward()
    y = b.y.clone()
    b.y.fill_(math.nan)
    b.forward(saved=False)
    assert torch.equal(b.y, y)


@pytest.mark.parametrize("size", [(4100, 72, 1600, 2000), (2048, 1024, 4096, 1024), (5000, 1100, 1030, 1536)], ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("dtype", [BF16, F16], ids=["bf16", "f16"])
def test_block_of_many_tiles(ctx, size, dtype):
    b = Block(ctx, *size, dtype, "silu", F32 if size[0] == 4100 else None, seed=9)
    b.forward()
    b.backward()
    b.check()


def test_many_rows_of_a_narrow_block(ctx):
    b = Block(ctx, 70001, 24, 16, 3, BF16, "square", F32, seed=3)
    b.forward()
    b.backward()
    b.check()


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("lead,gap", [(0, 8), (0, 3), (1, 0), (5, 24)])
def test_rows_apart_and_off_alignment(ctx, dtype, lead, gap):
    """strided and misaligned x, y, dy, dx between NaN: nothing beside them is read or written"""
    b = Block(ctx, 45, 64, 72, 40, dtype, "poly3", seed=8)
    frames = {}
    for n in ("x", "dy", "y", "dx"):
        v, buf = framed(getattr(b, n), lead, gap)
        setattr(b, n, v)
        frames[n] = buf
    for i in range(3):
        b.dw[i] = framed(b.dw[i].reshape(1, -1), lead)[0].reshape(b.dw[i].shape)
    for n in ("wg", "wu", "wd"):
        w = getattr(b, n)
        setattr(b, n, framed(w.reshape(1, -1), lead)[0].reshape(w.shape))
    b.forward()
    b.backward()
    b.check()
    for n in ("y", "dx"):
        t = getattr(b, n)
        assert int(torch.isfinite(frames[n]).sum()) == t.numel()


@pytest.mark.parametrize("size", [(1, 64, 96, 40), (33, 40, 24, 17), (300, 136, 264, 136)], ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("gt", [F32, BF16], ids=["f32", "bf16"])
def test_gradients_are_added_where_asked(ctx, size, gt):
    b = Block(ctx, *size, BF16, "square", gt, seed=4)
    b.forward()
    b.backward()
    once = [d.clone() for d in b.dw]
    base = [normal(gen(40 + i), *d.shape, scale=3.0, dtype=gt) for i, d in enumerate(b.dw)]
    want = [(s.double(), base_.double()) for s, base_ in zip(once, base)]
    for d, s in zip(b.dw, base):
        d.copy_(s)
    b.dx.fill_(math.nan)
    dx_before = b.dx.clone()
    b.backward(dx=False, accumulate=True)
    assert torch.equal(b.dx.isnan(), dx_before.isnan())  # no dx asked, none written
    for d, (s, base_) in zip(b.dw, want):
        # the sum before its one rounding differs from the stored gradient by that gradient's rounding
        tol = ref.ROUND[gt] * (s.abs() * 1.01 + (s + base_).abs() * 1.01) + 2.0**-23 * (s.abs() + base_.abs())
        assert bool(((d.double() - s - base_).abs() <= tol).all())


def test_no_rows(ctx):
    b = Block(ctx, 0, 24, 16, 8, BF16, "silu", F32)
    b.forward()
    b.backward()
    assert all(bool((d == 0).all()) for d in b.dw)
    for d in b.dw:
        d.fill_(2.0)
    b.backward(accumulate=True)
    assert all(bool((d == 2).all()) for d in b.dw)


@pytest.mark.parametrize("size", [(5, 40, 32, 24), (70, 96, 80, 24), (260, 136, 264, 136)], ids=lambda s: "x".join(map(str, s)))
def test_what_is_not_finite_stays_in_its_row(ctx, size):
    b = Block(ctx, *size, BF16, "poly3", seed=6)
    b.forward()
    b.backward()
    y, dx = b.y.clone(), b.dx.clone()
    r = size[0] // 2
    b.x[r, size[1] // 2] = math.inf
    b.dy[r, 0] = math.nan
    b.forward()
    b.backward()
    keep = torch.arange(size[0], device=DEV) != r
    assert torch.equal(b.y[keep], y[keep]) and torch.equal(b.dx[keep], dx[keep])
    assert bool(torch.isnan(b.y[r]).any()) and bool(torch.isnan(b.dx[r]).all())
    assert all(bool(torch.isnan(d).any()) for d in b.dw)


@pytest.mark.parametrize("act", ["linear", "square", "poly3"])
def test_gradients_are_differences(ctx, act):
    """The answer is a polynomial of the step along any direction of x or of one weight matrix, of degree at most 4: differences at
    steps of 1/2 and 1 (and their combination that leaves out the third power) give its derivative without truncation"""
    b = Block(ctx, 37, 40, 48, 24, F32, act, seed=12)
    b.forward()
    b.backward()
    b.check()

    def loss():
        b.forward(saved=False)
        return float((b.y.double() * b.dy.double()).sum())

    bound_y = ref.block(b.x, b.wg, b.wu, b.wd, b.act)["y"][1]
    for name, grad in (("x", b.dx), ("wg", b.dw[0]), ("wu", b.dw[1]), ("wd", b.dw[2])):
        t = getattr(b, name)
        keep = t.clone()
        d = normal(gen(77), *t.shape, scale=0.25 * float(t.double().pow(2).mean().sqrt()))
        vals = {}
        slack = 0.0
        for s in (-1.0, -0.5, 0.5, 1.0):
            t.copy_(keep + s * d)
            real = (t.double() - keep.double()) - s * d.double()  # what rounding the point to 32 bits moved it by
            vals[s] = loss()
            want = ref.block(b.x, b.wg, b.wu, b.wd, b.act)["y"]
            slack += float((want[1] * b.dy.double().abs()).sum())
            slack += float((grad.double().abs() * real.abs()).sum()) * 4
        t.copy_(keep)
        full, half = (vals[1.0] - vals[-1.0]) / 2, vals[0.5] - vals[-0.5]
        slope = (4 * half - full) / 3
        along = float((grad.double() * d.double()).sum())
        gb = {"x": "dx", "wg": "dwg", "wu": "dwu", "wd": "dwd"}[name]
        gbound = float((ref.block(b.x, b.wg, b.wu, b.wd, b.act, b.dy)[gb][1] * d.double().abs()).sum())
        assert abs(slope - along) <= gbound + 2 * slack, (name, slope, along, gbound, slack)


def test_equal_calls_give_equal_bits_on_any_stream_and_in_graphs(ctx):
    b = Block(ctx, 333, 517, 1021, 129, BF16, "poly3", F32, seed=2)
    b.forward()
    b.backward()
    first = {k: v.clone() for k, v in b.results().items()}
    side = torch.cuda.Stream()
    for v in b.results().values():
        v.fill_(math.nan)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        b.forward()
        b.backward()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(v, first[k]) for k, v in b.results().items())
    graph = torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        b.forward()
        b.backward()
    for _ in range(3):
        for v in b.results().values():
            v.fill_(math.nan)
        b.ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(v, first[k]) for k, v in b.results().items())


def refused(code, call, *args, **kw):
    with pytest.raises(ckksmi.CkksmiError) as e:
        call(*args, **kw)
    assert e.value.code == code


def test_block_refusals(ctx):
    b = Block(ctx, 10, 24, 16, 8, BF16, "silu", F32)
    L, h = ctx._L, ctx._h

    def fwd(shape=b.ff._s, x=b.x, y=b.y, ws=b.ws, n=None, saved=None, wg=b.wg):
        p = ckksmi._ptr
        return L.ckksmi_gated_ff_forward(h, C.byref(shape), p(x), p(wg), p(b.wu), p(b.wd), p(y), p(saved), p(ws), b.ws.numel() if n is None else n, None)

    def shape(**kw):
        s = ckksmi.GatedFFShape.from_buffer_copy(b.ff._s)
        s.rows, s.ld_x, s.ld_y = 10, 0, 0
        for k, v in kw.items():
            setattr(s, k, v)
        return s

    assert fwd(shape()) == ckksmi.OK
    for bad in (dict(dtype=3), dict(dtype=-1), dict(grad_dtype=ckksmi.F16), dict(act=4), dict(act=-1), dict(rows=-1), dict(rows=2**31), dict(d_in=0), dict(d_hidden=0),
                dict(d_out=-3), dict(d_in=2**20 + 1), dict(ld_x=23), dict(ld_y=7), dict(ld_x=2**20 + 8)):
        assert fwd(shape(**bad)) == ckksmi.EINVAL, bad
    assert fwd(shape(), x=None) == ckksmi.EINVAL and fwd(shape(), y=None) == ckksmi.EINVAL and fwd(shape(), ws=None) == ckksmi.EINVAL
    assert fwd(shape(), x=b.x.data_ptr() + 1) == ckksmi.EINVAL and fwd(shape(), ws=b.ws.data_ptr() + 8) == ckksmi.EINVAL
    assert fwd(shape(), saved=b.saved.data_ptr() + 2) == ckksmi.EINVAL
    assert fwd(shape(), y=b.x) == ckksmi.EINVAL and fwd(shape(), y=b.wg.data_ptr() + 32) == ckksmi.EINVAL and fwd(shape(), saved=b.ws) == ckksmi.EINVAL
    need = b.ff.workspace_bytes(10)
    assert fwd(shape(), n=need - 1) == ckksmi.EWORKSPACE and fwd(shape(), n=need) == ckksmi.OK
    assert L.ckksmi_gated_ff_forward(h, None, None, None, None, None, None, None, None, 0, None) == ckksmi.EINVAL
    assert L.ckksmi_gated_ff_forward(None, C.byref(shape()), None, None, None, None, None, None, None, 0, None) == ckksmi.EDEVICE
    n = C.c_size_t(0)
    assert L.ckksmi_gated_ff_workspace_bytes(h, C.byref(shape(d_in=0)), 0, C.byref(n)) == ckksmi.EINVAL
    assert L.ckksmi_gated_ff_saved_bytes(None, C.byref(shape()), C.byref(n)) == ckksmi.EINVAL
    # backward
    keep = b.dx, b.dw[0], b.saved
    b.forward()
    b.dx = b.x
    refused(ckksmi.EINVAL, b.backward)
    b.dx = keep[0]
    b.dw[1] = b.dw[0]
    refused(ckksmi.EINVAL, b.backward)
    b.dw[1] = torch.empty_like(keep[1])
    small = b.ws
    b.ws = b.ws[: b.ff.workspace_bytes(10, backward=True) - 256]
    refused(ckksmi.EWORKSPACE, b.backward)
    b.ws = small
    b.backward()
    b.check()
    # the binding's own checks
    with pytest.raises(ValueError):
        b.ff.forward(b.x.float(), b.wg, b.wu, b.wd, b.y, b.ws)
    with pytest.raises(ValueError):
        b.ff.forward(b.x, b.wu.t(), b.wu, b.wd, b.y, b.ws)
    with pytest.raises(ValueError):
        b.ff.forward(b.x[:, :8], b.wg, b.wu, b.wd, b.y, b.ws)
    with pytest.raises(ValueError):
        b.ff.forward(b.x, b.wg, b.wu, b.wd, b.y, b.ws, saved=b.saved[:64])
    with pytest.raises(ValueError):
        training.GatedFF(ctx, 8, 8, 8, BF16, (1.0, 2.0))
    with pytest.raises(ValueError):
        training.GatedFF(ctx, 8, 8, 8, torch.float64, "silu")


# ---------------------------------------------------------------- AdamW
HP = dict(lr=3e-3, betas=(0.9, 0.99), eps=1e-8, weight_decay=0.1, step=4, grad_scale=0.5)


class Step:
    """tensors of a step with states in 8 or 32 bits, each behind `lead` elements of a buffer that nothing else may touch"""

    def __init__(self, ctx, numels, bits, pt=F32, gt=F32, copy=None, lead=0, seed=0):
        g = gen(seed)
        self.numels, self.bits, self.seed = numels, bits, 0x1234567890 + seed

        def place(t):
            buf = torch.full((lead + t.numel() + 9,), 77, dtype=t.dtype, device=DEV)
            buf[lead:lead + t.numel()] = t
            self.frames.append((buf, lead, t.numel()))
            return buf[lead:lead + t.numel()]

        self.frames = []
        self.p = [place(normal(g, n, dtype=pt)) for n in numels]
        self.g = [place(normal(g, n, scale=10.0 ** (-i % 5), dtype=gt)) for i, n in enumerate(numels)]
        m = [normal(g, n, scale=0.3) for n in numels]
        v = [normal(g, n).square_() + 0.01 for n in numels]
        self.mu = self.vu = None
        if bits == 8:
            rm = [ref.random_words(1, i, n) >> np.uint64(16) for i, n in enumerate(numels)]
            mc = [ref.write_codes(a.cpu().numpy(), r, 3) for a, r in zip(m, rm)]
            vc = [ref.write_codes(a.cpu().numpy(), r, 4) for a, r in zip(v, rm)]
            m, v = [torch.from_numpy(c).to(DEV) for c, _ in mc], [torch.from_numpy(c).to(DEV) for c, _ in vc]
            self.mu, self.vu = [place(torch.from_numpy(u).to(DEV)) for _, u in mc], [place(torch.from_numpy(u).to(DEV)) for _, u in vc]
        self.m, self.v = [place(t) for t in m], [place(t) for t in v]
        self.copy = [place(torch.zeros(n, dtype=copy, device=DEV)) for n in numels] if copy is not None else None
        self.opt = training.AdamW(ctx, self.p, self.g, self.m, self.v, self.mu, self.vu, self.copy)

    def host(self, t):
        return t.float().cpu().numpy() if t.dtype != torch.uint8 else t.cpu().numpy()

    def expect(self, **kw):
        """per tensor: dict of arrays after a step"""
        hp = dict(HP, **kw)
        out = []
        for i, n in enumerate(self.numels):
            p, g = self.host(self.p[i]), self.host(self.g[i])
            m, v = self.host(self.m[i]), self.host(self.v[i])
            if self.bits == 8:
                m, v = ref.read_codes(m, self.host(self.mu[i]), 3), ref.read_codes(v, self.host(self.vu[i]), 4)
            p, m, v = ref.adamw_f32(p, g, m, v, hp["lr"], hp["betas"], hp["eps"], hp["weight_decay"], hp["step"], hp["grad_scale"])
            d = {"p": p, "m": m, "v": v}
            if self.bits == 8:
                w = ref.random_words(self.seed, i, n)
                d["mc"], d["mu"] = ref.write_codes(m, w >> np.uint64(16), 3)
                d["vc"], d["vu"] = ref.write_codes(v, w & np.uint64(0xFFFF), 4)
            out.append(d)
        return out

    def step(self, **kw):
        self.opt.step(**dict(HP, seed=self.seed, **kw))

    def check(self, want):
        for i, d in enumerate(want):
            p = torch.from_numpy(np.ascontiguousarray(d["p"])).to(self.p[i].dtype)
            assert torch.equal(self.p[i].cpu(), p), ("p", i)
            if self.copy is not None:
                assert torch.equal(self.copy[i].cpu(), torch.from_numpy(np.ascontiguousarray(d["p"])).to(self.copy[i].dtype)), ("copy", i)
            if self.bits == 32:
                assert np.array_equal(self.host(self.m[i]), d["m"]) and np.array_equal(self.host(self.v[i]), d["v"]), ("states", i)
            else:
                assert np.array_equal(self.host(self.mu[i]), d["mu"]) and np.array_equal(self.host(self.vu[i]), d["vu"]), ("units", i)
                assert np.array_equal(self.host(self.m[i]), d["mc"]) and np.array_equal(self.host(self.v[i]), d["vc"]), ("codes", i)
        for buf, lead, n in self.frames:
            assert bool((buf[:lead] == 77).all()) and bool((buf[lead + n:] == 77).all()), "written beside a tensor"


NUMELS = [1, 2, 255, 256, 257, 1023, 4095, 4096, 4097, 70001, 0, 3, 8191]


@pytest.mark.parametrize("lead", [0, 1, 4])
@pytest.mark.parametrize("pt,gt,copy", [(F32, F32, None), (F32, BF16, BF16), (F32, F16, F16), (BF16, BF16, None), (F16, F16, None), (BF16, F32, None)])
@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_bits(ctx, bits, pt, gt, copy, lead):
    s = Step(ctx, NUMELS, bits, pt, gt, copy, lead, seed=lead)
    want = s.expect()
    s.step()
    s.check(want)
    want = s.expect(step=5)  # and from the state it left
    s.step(step=5)
    s.check(want)


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_more_tensors_than_a_table_holds(ctx, bits):
    s = Step(ctx, [(37 * i) % 600 for i in range(150)], bits, seed=3)
    want = s.expect()
    s.step()
    s.check(want)


def test_adamw_against_64_bits(ctx):
    """32-bit results lose at most a few roundings of their parts"""
    s = Step(ctx, [5000], 32, seed=5)
    p, g, m, v = (t[0].double() for t in (s.p, s.g, s.m, s.v))
    s.step()
    g = g * HP["grad_scale"]
    b1, b2 = HP["betas"]
    m1, v1 = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
    up = HP["lr"] * (m1 / (1 - b1**4)) / (torch.sqrt(v1 / (1 - b2**4)) + HP["eps"])
    em = 4 * ref.U32 * ((b1 * m).abs() + ((1 - b1) * g).abs())
    assert bool(((s.m[0].double() - m1).abs() <= em).all()) and bool(((s.v[0].double() - v1).abs() <= 6 * ref.U32 * v1).all())
    ep = HP["lr"] * (em / (1 - b1**4)) / torch.sqrt(v1 / (1 - b2**4)) + 16 * ref.U32 * up.abs() + 4 * ref.U32 * p.abs()
    assert bool(((s.p[0].double() - (p - HP["lr"] * HP["weight_decay"] * p - up)).abs() <= 1.1 * ep).all())


def test_adamw_values_that_are_not_finite(ctx):
    for bits in (32, 8):
        s = Step(ctx, [1024], bits, seed=6)
        s.g[0][300], s.g[0][700] = math.nan, math.inf
        s.step()
        bad = torch.tensor([300, 700], device=DEV)
        if bits == 32:
            assert not bool(torch.isfinite(s.m[0][bad]).any()) and int((~torch.isfinite(s.m[0])).sum()) == 2
        else:
            # the states of a block with such a value are lost and say so; other blocks and other elements' parameters are not
            assert torch.isnan(s.mu[0]).tolist() == [False, True, True, False] and torch.isnan(s.vu[0]).tolist() == [False, True, True, False]
            m, v = [torch.empty(1024, device=DEV)], [torch.empty(1024, device=DEV)]
            s.opt.read_states(m, v)
            assert torch.isnan(m[0]).reshape(4, 256).all(1).tolist() == [False, True, True, False]
        assert int((~torch.isfinite(s.p[0])).sum()) == 2


def test_adamw_zeros_and_tiny_values(ctx):
    for bits in (32, 8):
        s = Step(ctx, [600], bits, seed=7)
        for t in (s.m, s.v) + ((s.mu, s.vu) if bits == 8 else ()):
            t[0].zero_()
        s.g[0].zero_()
        s.g[0][300:] = 1e-36  # magnitudes below what a block's unit can hold
        want = s.expect()
        s.step()
        s.check(want)
        assert bool(torch.isfinite(s.p[0]).all())


def test_adamw_skip(ctx):
    s = Step(ctx, [3000], 8, BF16, BF16, seed=8)
    before = [t.clone() for t in (s.p[0], s.m[0], s.v[0], s.mu[0], s.vu[0])]
    flag = torch.ones(1, dtype=torch.int32, device=DEV)
    s.step(skip=flag)
    assert all(torch.equal(a, b) for a, b in zip(before, (s.p[0], s.m[0], s.v[0], s.mu[0], s.vu[0])))
    flag.zero_()
    want = s.expect()
    s.step(skip=flag)
    s.check(want)


def test_states_read_back(ctx):
    """every code, in blocks of an odd tensor"""
    n = 256 * 3 + 77
    codes = torch.arange(n, device=DEV).to(torch.uint8)
    units = torch.tensor([1.0, 0.25, 3.0, 1e-3], device=DEV)
    z = torch.zeros(n, device=DEV)
    opt = training.AdamW(ctx, [z], [z.clone()], [codes], [codes.clone()], [units], [units.clone()])
    m, v = [torch.full((n,), math.nan, device=DEV)], [torch.full((n,), math.nan, device=DEV)]
    opt.read_states(m, v)
    c, u = codes.cpu().numpy(), units.cpu().numpy()
    assert np.array_equal(m[0].cpu().numpy(), ref.read_codes(c, u, 3))
    assert np.array_equal(v[0].cpu().numpy(), ref.read_codes(c, u, 4))


def test_rounding_of_states_has_no_bias(ctx):
    """A mean that moves by less than half a code a step follows its gradients: 400 steps of a constant gradient from zero states.  A
    step rounds a value to a code at a distance of at most 1/8 (m) or 1/16 (v) of it: standard deviation at most half of that.  Of
    an error that is made at one step, beta^k is left k steps later: the sum of 400 has at most 1/sqrt(1 - beta^2) times one's
    deviation, the mean of 65536 elements 1/256 of that.  The random bits are cut at 16: up to 2^-16 of a gap a step downwards"""
    n = 65536
    g = normal(gen(1), n).abs_() + 0.5
    p = torch.zeros(n, device=DEV)
    m, v = torch.zeros(n, dtype=torch.uint8, device=DEV), torch.zeros(n, dtype=torch.uint8, device=DEV)
    mu, vu = torch.zeros(256, device=DEV), torch.zeros(256, device=DEV)
    opt = training.AdamW(ctx, [p], [g], [m], [v], [mu], [vu])
    for t in range(1, 401):
        opt.step(1e-3, (0.99, 0.999), 1e-8, 0.0, t, seed=t)
    a, b = [torch.empty(n, device=DEV)], [torch.empty(n, device=DEV)]
    opt.read_states(a, b)
    for got, of, beta, gap in ((a[0], g, 0.99, 1 / 8), (b[0], g * g, 0.999, 1 / 16)):
        want = 1 - beta**400
        dev = want * gap / 2 / math.sqrt(1 - beta**2) / 256
        cut = want * gap * 2.0**-16 / (1 - beta)
        assert abs(float((got.double() / of.double()).mean()) - want) < 6 * dev + cut


def test_adamw_trains_alike_with_8_and_32_bit_states(ctx):
    """a least-squares problem solved from zero states: both end near the answer"""
    g = gen(11)
    a = normal(g, 512, 64, scale=1 / 8)
    want = normal(g, 64)
    b = a @ want
    ends = []
    for bits in (32, 8):
        p, gr = torch.zeros(64, device=DEV), torch.zeros(64, device=DEV)
        if bits == 32:
            opt = training.AdamW(ctx, [p], [gr], [torch.zeros(64, device=DEV)], [torch.zeros(64, device=DEV)])
        else:
            z = [torch.zeros(64, dtype=torch.uint8, device=DEV) for _ in range(2)]
            opt = training.AdamW(ctx, [p], [gr], [z[0]], [z[1]], [torch.zeros(1, device=DEV)], [torch.zeros(1, device=DEV)])
        for t in range(1, 601):
            gr.copy_(a.t() @ (a @ p - b))
            opt.step(0.05 * (1 - t / 601), (0.9, 0.99), 1e-8, 0.0, t, seed=t)
        ends.append(float((p - want).norm() / want.norm()))
    assert ends[0] < 0.02 and ends[1] < 0.05, ends


def test_adamw_refusals(ctx):
    s = Step(ctx, [100], 8, seed=9)
    for bad in (dict(step=0), dict(betas=(1.0, 0.9)), dict(betas=(0.9, -0.1)), dict(eps=-1.0), dict(lr=math.nan), dict(grad_scale=math.inf), dict(weight_decay=math.inf),
                dict(betas=(math.nan, 0.9))):
        refused(ckksmi.EINVAL, s.step, **bad)
    L, h = ctx._L, ctx._h
    o, t = s.opt._o, s.opt._t
    s.step()

    def call(n=1, params=o, **kw):
        x = ckksmi.AdamWTensor.from_buffer_copy(t[0])
        for k, v in kw.items():
            setattr(x, k, v)
        return L.ckksmi_adamw_step(h, C.byref(params), C.byref(x), n, None)

    assert call() == ckksmi.OK and call(n=0) == ckksmi.OK
    for k in ("p", "grad", "m", "v", "m_unit", "v_unit"):
        assert call(**{k: None}) == ckksmi.EINVAL, k
    for k in ("p", "grad", "m_unit", "v_unit"):
        assert call(**{k: getattr(t[0], k) + 1}) == ckksmi.EINVAL, k
    assert call(n=-1) == ckksmi.EINVAL and L.ckksmi_adamw_step(h, C.byref(o), None, 1, None) == ckksmi.EINVAL
    assert call(n=1) == ckksmi.OK
    x = ckksmi.AdamWTensor.from_buffer_copy(t[0])
    x.n = -1
    assert L.ckksmi_adamw_step(h, C.byref(o), C.byref(x), 1, None) == ckksmi.EINVAL
    x.n = 2**40
    assert L.ckksmi_adamw_step(h, C.byref(o), C.byref(x), 1, None) == ckksmi.EINVAL
    for k, v in (("p_dtype", 3), ("grad_dtype", -1), ("state_bits", 16), ("skip", s.p[0].data_ptr() + 1)):
        q = ckksmi.AdamWParams.from_buffer_copy(o)
        setattr(q, k, v)
        assert call(params=q) == ckksmi.EINVAL, k
    q = ckksmi.AdamWParams.from_buffer_copy(o)
    q.copy_dtype = ckksmi.F32
    assert call(params=q, copy=s.g[0].data_ptr()) == ckksmi.EINVAL
    assert L.ckksmi_adamw_read_states(h, t, 1, None, None, None) == ckksmi.EINVAL
    assert L.ckksmi_adamw_step(None, C.byref(o), t, 1, None) == ckksmi.EDEVICE
    z = [torch.zeros(5, device=DEV)]
    with pytest.raises(ValueError):
        training.AdamW(ctx, z, z, z, [torch.zeros(4, device=DEV)])
    with pytest.raises(ValueError):
        training.AdamW(ctx, z, z, z, z, m_units=z)
    with pytest.raises(ValueError):
        training.AdamW(ctx, z, z, [torch.zeros(5, dtype=BF16, device=DEV)], z)
