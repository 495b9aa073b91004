"""Plans of training.py and head.py on the CPU stand-in: what they refuse, what they ask for and what a call is given."""
import ctypes as C

import pytest
import torch

import train_emu_support as emu
import training_range
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


class Calls:
    """a context that counts the calls and makes none"""

    _h = None

    def __init__(self):
        self.made = []

    def _call(self, name, *args):
        self.made.append(name)

    @staticmethod
    def _stream(stream):
        return None


@pytest.mark.parametrize("width", [1, 8])
@pytest.mark.parametrize("which", ["x", "y", "dy", "dx"])
def test_rows_that_lie_on_each_other_are_refused(which, width):
    """a row repeated by expand() and rows closer than their width: a distance of 0 means dense rows to the library"""
    rows = 5
    ff = training.GatedFF(Calls(), width, 16, width, F32, "square")
    w = [torch.zeros(16, width), torch.zeros(16, width), torch.zeros(width, 16)]
    dw = [torch.zeros_like(t) for t in w]
    room = torch.zeros(1 << 16, dtype=torch.uint8)
    overlapping = [torch.zeros(1, width).expand(rows, width)]
    if width > 1:
        overlapping.append(torch.zeros(64).as_strided((rows, width), (width - 1, 1)))
    for bad in overlapping:
        t = {k: torch.zeros(rows, width) for k in ("x", "y", "dy", "dx")}
        t[which] = bad
        with pytest.raises(ValueError):
            ff.forward(t["x"], *w, t["y"], room)
            ff.backward(t["x"], *w, room, t["dy"], t["dx"], *dw, room)
    # one row has no distance, and rows further apart are taken as they are
    ff.forward(torch.zeros(1, width).expand(1, width), *w, torch.zeros(1, width), room)
    ff.forward(torch.zeros(rows, width + 3)[:, :width], *w, torch.zeros(rows, width), room)


WIDTHS = [(1024, 4096, 1024), (4096, 4096, 4096), (3136, 256, 2), (517, 1021, 129), (8, 8, 8), (40, 24, 8192), (8192, 64, 1000), (2048, 8192, 2048), (2000, 4000, 4000)]
ROWS = sorted({0, 1, 2, 63, 64, 65, 32768, 40000} | {32 * i + j for i in range(1, 200, 3) for j in (-1, 0, 1)} | {128 * i + j for i in range(1, 80) for j in (0, 1)})


@pytest.mark.parametrize("grads", ["same", "f32"])
@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=["f32", "bf16", "f16"])
@pytest.mark.parametrize("widths", WIDTHS, ids=lambda s: "x".join(map(str, s)))
def test_a_workspace_holds_any_smaller_number_of_rows(ctx, widths, dtype, grads):
    """workspace_bytes(rows) is for calls on up to `rows` rows: more rows never ask for less, and what is asked for holds what the split k axes
    take at this number of rows"""
    ff = training.GatedFF(ctx, *widths, dtype, "square", F32 if grads == "f32" else None)
    for name in ("emu_split_need", "emu_split_room"):
        getattr(ctx._L, name).restype = C.c_size_t
    for backward in (False, True):
        before = 0
        for rows in ROWS:
            n = ff.workspace_bytes(rows, backward=backward)
            assert n >= before, (rows, backward, n, before)
            before = n
            ff._s.rows = rows
            if rows:
                need, room = (f(ff._r, int(backward)) for f in (ctx._L.emu_split_need, ctx._L.emu_split_room))
                assert need <= room, (rows, backward, need, room)


def test_a_short_last_batch_trains_in_the_same_workspace(ctx):
    """a head made for 1537 rows (gate: 49 tiles, 7 parts) takes a step on 1536 (48 tiles, 8 parts, more memory) and on a few"""
    from paper_1911_11377_amd import head

    g = torch.Generator().manual_seed(3)
    weights = [ctx.guarded(torch.randn(s, generator=g) * s[1] ** -0.5) for s in ((2, 2048), (2, 2048), (2, 2))]
    h = head.GatedHead(ctx, 1537, weights, "square", F32, lambda shape, t: ctx.guarded(torch.zeros(shape, dtype=t)))
    for rows in (1536, 33, 0):
        x = ctx.guarded(torch.randn((rows, 2048), generator=g))
        h.step(x, lambda y, dy: dy.copy_(y * (1 / max(1, y.numel()))), 1e-3)
        assert all(bool(torch.isfinite(w).all()) for w in weights)
    assert ctx.errors() == 0


@pytest.mark.parametrize("dtype,rows", [(BF16, 3), (F32, 3), (BF16, 70)], ids=["bf16", "f32", "bf16-tiles"])
def test_relu_of_minus_infinity_is_zero(ctx, dtype, rows):
    """finite operands whose gate sums pass the type's range: max(g, 0) is 0 below it, infinite above, and a NaN stays one"""
    ff = training.GatedFF(ctx, 8, 8, 8, dtype, "relu")
    x = torch.full((rows, 8), 1.0, dtype=dtype)
    x[0], x[1], x[2, 3] = 3e38, -3e38, float("nan")
    wg, wu = torch.full((8, 8), -1.0, dtype=dtype), torch.zeros(8, 8, dtype=dtype)
    wu[:, 0] = 2.0**-120
    wd = torch.ones(8, 8, dtype=dtype)
    x, wg, wu, wd, dy = (ctx.guarded(t) for t in (x, wg, wu, wd, torch.ones(rows, 8, dtype=dtype)))
    y, dx, dw = ctx.guarded(torch.ones(rows, 8, dtype=dtype)), ctx.guarded(torch.ones(rows, 8, dtype=dtype)), [ctx.guarded(torch.ones(8, 8, dtype=dtype)) for _ in range(3)]
    saved, ws = (ctx.guarded(torch.full((max(16, n),), 255, dtype=torch.uint8)) for n in (ff.saved_bytes(rows), ff.workspace_bytes(rows, backward=True)))
    for keep in (saved, None):
        ff.forward(x, wg, wu, wd, y, ws, saved=keep)
        assert bool((y[0] == 0).all()) and bool((y[1] == -float("inf")).all()) and bool(torch.isnan(y[2]).all())
        assert bool((y[3:] == 0).all())
    ff.backward(x, wg, wu, wd, saved, dy, dx, *dw, ws)
    assert bool((dx[0] == 0).all())  # neither the gate's derivative nor its value is anything but 0 there


@pytest.mark.parametrize("dtype", [F16, BF16], ids=["f16", "bf16"])
@pytest.mark.parametrize("rows", [20, 70])
@pytest.mark.parametrize("scales", training_range.SCALES, ids=str)
def test_f32_gradients_of_16_bit_operands_have_the_range_of_f32(ctx, scales, rows, dtype):
    training_range.check(ctx, "cpu", ctx.guarded, rows, dtype, scales)
    assert ctx.errors() == 0


@pytest.mark.parametrize("dtype", [F16, BF16], ids=["f16", "bf16"])
def test_f32_gradients_of_infinite_products(ctx, dtype):
    """what overflows f32 itself is not finite in the gradients, and the rest is as it was"""
    rows = 20
    ff = training.GatedFF(ctx, 8, 8, 8, dtype, (0.0, 0.0, 0.0, 1e38), F32)
    x, dy = torch.zeros(rows, 8, dtype=dtype), torch.zeros(rows, 8, dtype=dtype)
    x[3], dy[3] = 4.0, 1.0
    x[4:, 0], dy[4:, 0] = 2.0**-10, 2.0**-10
    wg, wu = torch.zeros(8, 8, dtype=dtype), torch.ones(8, 8, dtype=dtype)
    wg[5] = 1.0
    x, dy, wg, wu, wd = (ctx.guarded(t) for t in (x, dy, wg, wu, torch.ones(8, 8, dtype=dtype)))
    y, dx, dw = ctx.guarded(torch.zeros(rows, 8, dtype=dtype)), ctx.guarded(torch.zeros(rows, 8, dtype=dtype)), [ctx.guarded(torch.zeros(8, 8)) for _ in range(3)]
    saved, ws = (ctx.guarded(torch.full((max(16, n),), 255, dtype=torch.uint8)) for n in (ff.saved_bytes(rows), ff.workspace_bytes(rows, backward=True)))
    ff.forward(x, wg, wu, wd, y, ws, saved=saved)
    ff.backward(x, wg, wu, wd, saved, dy, dx, *dw, ws)
    # unit 5 alone has a gate that is not zero: its row of dWg, dWu and its column of dWd
    for d in (dw[0], dw[1], dw[2].t()):
        assert not bool(torch.isfinite(d[5]).any()), d[5]
        assert bool(torch.isfinite(d[[i for i in range(8) if i != 5]]).all())
    if dtype == BF16:  # one value a factor: infinities stay infinities
        assert bool(torch.isinf(dw[1][5]).all())


class Interrupted(Calls):
    """a context in the midst of whose calls another thread uses the same plan"""

    def __init__(self, meanwhile):
        super().__init__()
        self.meanwhile, self.depth, self.seen = meanwhile, 0, []

    def _call(self, name, *args):
        own = [a._obj for a in args if hasattr(a, "_obj") and isinstance(a._obj, C.Structure)]
        before = [bytes(o) for o in own]
        self.depth += 1
        if self.depth == 1:
            self.meanwhile()
            self.seen.append((name, before == [bytes(o) for o in own]))
        self.depth -= 1


def test_calls_of_one_plan_do_not_share_what_they_are_given():
    x, y, w, room = torch.zeros(9, 8), torch.zeros(9, 8), [torch.zeros(8, 8)] * 3, torch.zeros(1 << 16, dtype=torch.uint8)
    dw = [torch.zeros(8, 8) for _ in range(3)]
    c = Interrupted(lambda: (ff.workspace_bytes(5), ff.saved_bytes(4), ff.forward(x[:3], *w, y[:3], room), ff.backward(x[:2], *w, room, y[:2], None, *dw, room)))
    ff = training.GatedFF(c, 8, 8, 8, F32, "square")
    ff.forward(x, *w, y, room, saved=room)
    ff.backward(x, *w, room, y, x, *dw, room)
    ff.workspace_bytes(9)
    c.meanwhile = lambda: opt.step(2e-3, (0.8, 0.9), 1e-7, 0.2, 9, seed=9)
    opt = training.AdamW(c, *([torch.zeros(7)] for _ in range(4)))
    opt.step(1e-3, (0.9, 0.99), 1e-8, 0.1, 4, seed=3)
    assert {"ckksmi_gated_ff_forward", "ckksmi_gated_ff_backward", "ckksmi_gated_ff_workspace_bytes", "ckksmi_adamw_step"} <= {n for n, _ in c.seen}
    assert all(same for _, same in c.seen), c.seen


@pytest.mark.parametrize("stream", [None, 4096])
def test_the_loss_of_a_step_is_on_the_stream_of_the_step(ctx, monkeypatch, stream):
    """forward, loss, backward and optimiser step of a stream's step are all on that stream, without one on the current one"""
    import contextlib

    from paper_1911_11377_amd import head

    current, used = ["current"], []

    @contextlib.contextmanager
    def on(s):
        current.append(s)
        yield
        current.pop()

    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle, **kw: handle)
    monkeypatch.setattr(torch.cuda, "stream", on)
    weights = [ctx.guarded(torch.ones(s)) for s in ((4, 8), (4, 8), (2, 4))]
    h = head.GatedHead(ctx, 6, weights, "square", F32, lambda shape, t: ctx.guarded(torch.zeros(shape, dtype=t)))
    monkeypatch.setattr(ctx, "_stream", lambda s: used.append(current[-1] if s is None else s))
    want = "current" if stream is None else stream

    def loss(y, dy):
        used.append(current[-1])
        dy.copy_(y)
        return 7

    assert h.step(ctx.guarded(torch.ones(5, 8)), loss, 1e-3, stream=stream) == 7
    assert used == [want] * 4, used
    assert current == ["current"]


@pytest.mark.parametrize("rows,widths,dtype,forward,backward", [
    (2**31 - 257, (8, 128, 8), BF16, True, True),       # 2^23 - 1 tiles of 256 x 256, 512 threads each
    (2**31 - 257, (8, 129, 8), BF16, False, False),     # two columns of tiles, the gate's
    (2**30, (8, 129, 8), BF16, False, False),           # 2^23 tiles: one too many
    (2**30 - 256, (8, 129, 8), BF16, True, True),
    (2**30, (300, 128, 8), BF16, True, False),          # dx alone has too many
    (2**31 - 257, (8, 64, 8), F32, True, True),         # 2^24 - 2 tiles of 128 x 128, 256 threads each
    (2**31 - 257, (8, 65, 8), F32, False, False),
    (64, (2**20, 2**20, 2**20), BF16, True, False),     # the weights' gradients alone
    (0, (2**20, 2**20, 2**20), F32, True, True),
], ids=str)
def test_launches_that_would_have_too_many_threads_are_refused_first(ctx, rows, widths, dtype, forward, backward):
    """a launch holds fewer than 2^32 threads along x: EUNSUPPORTED from every entry point of the pass, with nothing enqueued"""
    ff = training.GatedFF(ctx, *widths, dtype, "square")
    ff._s.rows = rows
    a = 1 << 56  # addresses that nothing is done with
    for which, fits in ((0, forward), (1, backward)):
        n = C.c_size_t(0)
        assert ctx._L.ckksmi_gated_ff_workspace_bytes(ctx._h, ff._r, which, C.byref(n)) == (ckksmi.OK if fits else ckksmi.EUNSUPPORTED)
    args = [a * i for i in range(1, 5)]
    if not forward:
        assert ctx._L.ckksmi_gated_ff_forward(ctx._h, ff._r, *args, 5 * a, None, 6 * a, 2**60, None) == ckksmi.EUNSUPPORTED
    if not backward:
        assert ctx._L.ckksmi_gated_ff_backward(ctx._h, ff._r, *args, 5 * a, 6 * a, 7 * a, 8 * a, 9 * a, 10 * a, 0, 11 * a, 2**60, None) == ckksmi.EUNSUPPORTED


def test_tensors_that_no_launch_holds_are_refused(ctx):
    z = [torch.zeros(4)]
    opt = training.AdamW(ctx, z, [z[0].clone()], [z[0].clone()], [z[0].clone()])
    opt._t[0].n = (2**24 - 1) * 4096 + 1  # 2^24 workgroups of 256 threads
    with pytest.raises(ckksmi.CkksmiError) as e:
        opt.step(1e-3, (0.9, 0.99), 1e-8, 0.0, 1)
    assert e.value.code == ckksmi.EINVAL
    out = (C.c_void_p * 1)(z[0].data_ptr())
    opt._t[0].m_unit = opt._t[0].v_unit = opt._t[0].m
    assert ctx._L.ckksmi_adamw_read_states(ctx._h, opt._t, 1, out, out, None) == ckksmi.EINVAL


@pytest.mark.parametrize("dtype,grads", [(BF16, None), (F16, F32)], ids=["bf16", "f16-f32"])
def test_copies_in_several_pieces_a_workgroup(ctx, dtype, grads):
    """operands off alignment, copied by fewer workgroups than they have pieces"""
    ff = training.GatedFF(ctx, 19, 21, 13, dtype, "square", grads)
    rows, g = 67, torch.Generator().manual_seed(2)
    x, wg, wu, wd, dy = (ctx.guarded(torch.randn(s, generator=g).to(dtype)) for s in ((rows, 19), (21, 19), (21, 19), (13, 21), (rows, 13)))
    y, dx = ctx.guarded(torch.zeros(rows, 13, dtype=dtype)), ctx.guarded(torch.zeros(rows, 19, dtype=dtype))
    dw = [ctx.guarded(torch.zeros(w.shape, dtype=grads or dtype)) for w in (wg, wu, wd)]
    saved, ws = (ctx.guarded(torch.full((max(16, n),), 255, dtype=torch.uint8)) for n in (ff.saved_bytes(rows), ff.workspace_bytes(rows, backward=True)))
    results = []
    for blocks in (1 << 23, 1, 2):
        ctx._L.emu_copy_blocks(blocks)
        try:
            ff.forward(x, wg, wu, wd, y, ws, saved=saved)
            ff.backward(x, wg, wu, wd, saved, dy, dx, *dw, ws)
        finally:
            ctx._L.emu_copy_blocks(1 << 23)
        results.append([t.clone() for t in (y, dx, *dw)])
        ws.fill_(255)
    assert all(torch.equal(a, b) for r in results[1:] for a, b in zip(r, results[0]))
    want = ref.block(x, wg, wu, wd, training.CUBICS["square"])["y"]
    assert bool(((y.double() - want[0]).abs() <= want[1]).all())


def test_tensors_that_overlap_are_refused():
    """a tied weight listed twice, a tensor inside another, states or copies that share memory: two workgroups would update the same bytes.
    Gradients are read only and may be one tensor; neighbours may touch"""
    flat = torch.zeros(6000)

    def plan(**kw):
        d = {k: [torch.zeros(700), torch.zeros(300), torch.zeros(0)] for k in ("params", "grads", "m", "v")}
        d.update(kw)
        return training.AdamW(Calls(), d["params"], d["grads"], d["m"], d["v"], copies=d.get("copies"))

    p = [torch.zeros(700), torch.zeros(300), torch.zeros(0)]
    plan()
    plan(params=[flat[:700], flat[700:1000], flat[:0]], m=[flat[1000:1700], flat[1700:2000], flat[:0]])
    plan(grads=[flat[:700], flat[400:700], flat[:0]])
    shared = torch.zeros(300)
    for bad in (dict(params=[flat[:700], flat[699:999], flat[:0]]), dict(params=[flat[:700], flat[200:500], flat[:0]]), dict(params=p, grads=p), dict(params=p, m=p),
                dict(m=[flat[:700], shared, flat[:0]], v=[torch.zeros(700), shared, flat[:0]]), dict(params=p, copies=[t.view(torch.bfloat16)[: t.numel()] for t in p]),
                dict(grads=[flat[:700], flat[:300], flat[:0]], v=[torch.zeros(700), flat[650:950], flat[:0]])):
        with pytest.raises(ValueError):
            plan(**bad)
    with pytest.raises(ValueError):
        training.AdamW(Calls(), [shared, shared], *([torch.zeros(300), torch.zeros(300)] for _ in range(3)))
    units = [torch.zeros(2)]
    with pytest.raises(ValueError):
        training.AdamW(Calls(), [torch.zeros(300)], [torch.zeros(300)], *([torch.zeros(300, dtype=torch.uint8)] for _ in range(2)), units, units)


def test_skip_is_one_int32():
    """the step reads four bytes: a truth value or an empty tensor has fewer, and the lower half of other numbers says something else"""
    c = Calls()
    opt = training.AdamW(c, *([torch.zeros(7)] for _ in range(4)))
    for bad in (torch.ones(1, dtype=torch.bool), torch.ones(1, dtype=torch.int64), torch.ones(1), torch.ones(0, dtype=torch.int32)):
        with pytest.raises(ValueError):
            opt.step(1e-3, (0.9, 0.99), 1e-8, 0.1, 4, skip=bad)
    assert not c.made
    opt.step(1e-3, (0.9, 0.99), 1e-8, 0.1, 4, skip=torch.zeros(1, dtype=torch.int32))
    opt.step(1e-3, (0.9, 0.99), 1e-8, 0.1, 4)
    assert c.made == ["ckksmi_adamw_step"] * 2


def test_one_kind_of_states_is_read_back(ctx):
    """m or v alone, as the library's call allows; both are what they are together.  Only float32 is written"""
    n = 700
    codes = ctx.guarded(torch.arange(n).to(torch.uint8)), ctx.guarded((torch.arange(n) * 3).to(torch.uint8))
    units = ctx.guarded(torch.tensor([1.0, 0.25, 3.0])), ctx.guarded(torch.tensor([2.0, 1e-3, 0.5]))
    opt = training.AdamW(ctx, [ctx.guarded(torch.zeros(n))], [ctx.guarded(torch.zeros(n))], [codes[0]], [codes[1]], [units[0]], [units[1]])
    both, one = [[[ctx.guarded(torch.zeros(n))] for _ in range(2)] for _ in range(2)]
    opt.read_states(*both)
    opt.read_states(m_out=one[0])
    opt.read_states(None, one[1])
    assert all(torch.equal(a[0], b[0]) and bool(a[0].any()) for a, b in zip(both, one))
    for bad in ([torch.zeros(n, dtype=torch.int32)], [torch.zeros(n - 1)], []):
        with pytest.raises(ValueError):
            opt.read_states(bad, None)
    with pytest.raises(ckksmi.CkksmiError):
        opt.read_states()


@pytest.mark.parametrize("grads", [None, F32], ids=["16", "fine"])
@pytest.mark.parametrize("rows,split", [(3, False), (70, False), (260, True)], ids=["few", "tiles", "parts"])
def test_infinities_are_not_joined_by_what_pads_a_row(ctx, rows, split, grads):
    """5 hidden units lie in rows of 8: an infinite x or dy (positive weights, all of the row's sums infinite) gives infinite answers and
    gradients, no NaN out of infinity times the zeros behind the weights' ends"""
    d_in = 600 if split else 9
    ff = training.GatedFF(ctx, d_in, 5, 600 if split else 7, BF16, "relu", grads)
    x, dy = torch.ones(rows, d_in, dtype=BF16), torch.ones(rows, ff.d_out, dtype=BF16)
    w = [torch.full(s, 0.5, dtype=BF16) for s in ((5, d_in), (5, d_in), (ff.d_out, 5))]
    x[1, 2], dy[0, 1] = float("inf"), float("inf")
    x, dy, wg, wu, wd = (ctx.guarded(t) for t in (x, dy, *w))
    y, dx = ctx.guarded(torch.zeros(rows, ff.d_out, dtype=BF16)), ctx.guarded(torch.zeros(rows, d_in, dtype=BF16))
    dw = [ctx.guarded(torch.zeros(t.shape, dtype=grads or BF16)) for t in w]
    saved, ws = (ctx.guarded(torch.full((max(16, n),), 255, dtype=torch.uint8)) for n in (ff.saved_bytes(rows), ff.workspace_bytes(rows, backward=True)))
    for keep in (saved, None):
        ff.forward(x, wg, wu, wd, y, ws, saved=keep)
        assert bool((y[1] == float("inf")).all()) and bool(torch.isfinite(y[torch.arange(rows) != 1]).all())
    ff.backward(x, wg, wu, wd, saved, dy, dx, *dw, ws)
    inf_rows = torch.arange(rows) < 2
    assert bool((dx[inf_rows] == float("inf")).all()) and bool(torch.isfinite(dx[~inf_rows]).all())
    # (f32 gradients take dg and du in parts, the later ones of an infinite value zeros: NaN where they meet the infinite x)
    keep = torch.arange(d_in) != 2
    assert all(bool((d[:, keep] == float("inf")).all()) and not bool(torch.isfinite(d).any()) for d in (dw[0], dw[1]))
