"""A gated head: trained in the clear, evaluated under encryption (call sequences over the library's operators).

The head behind a network's features is a gated feed-forward block, y = (act(x Wg^T) * (x Wu^T)) Wd^T.  `GatedHead` trains it on
plain features (training.py: one forward and one backward call and one optimiser step over its three matrices); `plan` and
`forward` evaluate the trained head on one ciphertext per feature (slot s = image s), the layout of cnn.py:
  fc      : Wg and Wu as one integer-weight layer of 2 d_hidden outputs, then a rescale      level l   -> l-1
  act     : linear, square, poly2 or poly3 (activation.py) on the gate's outputs             level l-1 -> l-1, l-2, l-3, l-3
  product : the other outputs dropped to that level, ciphertext x ciphertext, rescale        one level
  fc      : Wd, then a rescale                                                               one level

`ResidualHead` puts norms around such a block, r = a x + b gate * N_post(block(N_pre(x))): whoever encrypts the features norms them first
and takes the norm, the gate and the sum of what was decrypted, so the block under encryption stays the same.  `LowBitHead`
answers in the clear from the trained matrices in 4 bits.
"""
import contextlib
from dataclasses import dataclass

import numpy as np

from . import activation, ckksmi, lowbit, training


def _on_stream(stream, f, *args):
    """f(*args) with `stream` (an address; None: as it is) as torch's current one"""
    import torch

    with contextlib.nullcontext() if stream is None else torch.cuda.stream(torch.cuda.ExternalStream(stream)):
        return f(*args)


class GatedHead:
    """Training state of a head on up to `rows` rows a step.  weights: float32 device tensors [d_hidden][d_in] (twice) and
    [d_out][d_hidden], updated in place; dtype: the type the products run in (bfloat16 and float16: copies of the weights,
    renewed by each step); state_bits: 8 or 32.  optimizer: "adamw", or "muon" (steps along orthogonalised momentum, which is held in 32
    bits).  empty(shape, dtype) allocates zeros on the device.  The constructor waits for what it enqueues: answers and steps may
    use any stream.  Steps have to be ordered after each other, and answers after each other: each kind has buffers of its own and shares them with
    nothing else, so an answer on up to `rows` rows may be made within `loss` or beside a step; the weights that it reads move at the step's end."""

    def __init__(self, ctx, rows, weights, act, dtype, empty, state_bits=8, optimizer="adamw"):
        import torch

        if optimizer not in ("adamw", "muon"):
            raise ValueError("expected 'adamw' or 'muon', got %r" % (optimizer,))

        d_hidden, d_in = weights[0].shape
        self.weights, self.rows, self.steps = weights, rows, 0
        self.ff = training.GatedFF(ctx, d_in, d_hidden, weights[2].shape[0], dtype, act)
        copies = None
        if dtype != torch.float32:
            copies = [empty(tuple(w.shape), dtype) for w in weights]
            for c, w in zip(copies, weights):
                c.copy_(w)
        self.used = copies or weights
        self.grads = [empty(tuple(w.shape), dtype) for w in weights]
        self.opt_ws = None
        if optimizer == "muon":
            self.opt = training.Muon(ctx, weights, self.grads, [empty(tuple(w.shape), torch.float32) for w in weights], copies=copies)
            self.opt_ws = empty((max(16, self.opt.workspace_bytes()),), torch.uint8)
        else:
            state = torch.uint8 if state_bits == 8 else torch.float32
            m, v = [[empty(tuple(w.shape), state) for w in weights] for _ in range(2)]
            units = [[empty((-(-w.numel() // ckksmi.STATE_BLOCK),), torch.float32) for w in weights] for _ in range(2)] if state_bits == 8 else (None, None)
            self.opt = training.AdamW(ctx, weights, self.grads, m, v, *units, copies=copies)
        self.ws = empty((max(16, self.ff.workspace_bytes(rows, backward=True)),), torch.uint8)
        self.answer_ws = empty((max(16, self.ff.workspace_bytes(rows)),), torch.uint8)
        self.saved = empty((max(16, self.ff.saved_bytes(rows)),), torch.uint8)
        self.y, self.dy = [empty((rows, weights[2].shape[0]), dtype) for _ in range(2)]
        if weights[0].is_cuda:
            torch.cuda.current_stream(weights[0].device).synchronize()

    def answer(self, x, y, stream=None):
        # (more rows than a step's are answered in the steps' workspace, as far as that goes)
        self.ff.forward(x, *self.used, y, self.answer_ws if x.shape[0] <= self.rows else self.ws, stream=stream)

    def step(self, x, loss, lr, betas=(0.9, 0.99), eps=1e-8, weight_decay=0.0, stream=None):
        """One step on rows x.  loss(y, dy) writes the loss's gradient by the answers y into dy; what it returns is returned.  All of the step is
        enqueued on `stream`: loss is called with it as torch's current stream (x and what loss reads have to be ordered before it,
        and what loss returns is ready when it has come that far).  Muon: betas[0] is its momentum; eps is AdamW's alone."""
        rows = x.shape[0]
        y, dy = self.y[:rows], self.dy[:rows]
        self.ff.forward(x, *self.used, y, self.ws, saved=self.saved, stream=stream)
        out = _on_stream(stream, loss, y, dy)
        self.ff.backward(x, *self.used, self.saved, dy, None, *self.grads, self.ws, stream=stream)
        self._move(lr, betas, eps, weight_decay, stream)
        return out

    def _move(self, lr, betas, eps, weight_decay, stream):
        self.steps += 1
        if self.opt_ws is not None:
            self.opt.step(lr, betas[0], self.opt_ws, weight_decay=weight_decay, stream=stream)
        else:
            self.opt.step(lr, betas, eps, weight_decay, self.steps, seed=self.steps, stream=stream)


class ResidualHead:
    """A gated block between norms, answers of the features' width: r = residual_scale x + block_scale gate * N_post(block(N_pre(x))), with a learned
    gate for every channel.  `block` is the GatedHead inside (its weights, its optimizer); `vectors` are the norms' weights and the gate
    (float32, from ones; AdamW with 32-bit states).  Arguments, and which calls may run beside each other, as for GatedHead."""

    def __init__(self, ctx, rows, weights, act, dtype, empty, norm="rms", residual_scale=1.0, block_scale=1.0, eps=1e-5, optimizer="muon", state_bits=32):
        import torch

        d = weights[0].shape[1]
        if weights[2].shape[0] != d:
            raise ValueError("a residual block answers with as many values as it reads: %d and %d" % (weights[2].shape[0], d))
        self.block = GatedHead(ctx, rows, weights, act, dtype, empty, state_bits=state_bits, optimizer=optimizer)
        self.before = training.ResidualNorm(ctx, d, dtype, pre=norm, post=None, weight_dtype=torch.float32, eps=eps)
        self.after = training.ResidualNorm(ctx, d, dtype, pre=None, post=norm, gate="channel", weight_dtype=torch.float32, eps=eps, residual_scale=residual_scale,
                                           block_scale=block_scale)
        names = ["pre_weight", "post_weight", "gate"] + (["pre_bias", "post_bias"] if norm == "layer" else [])
        self.vectors = {k: empty((d,), torch.float32).fill_(0.0 if k.endswith("bias") else 1.0) for k in names}
        self.grads = {k: empty((d,), torch.float32) for k in names}
        states = [[empty((d,), torch.float32) for _ in names] for _ in range(2)]
        self.opt = training.AdamW(ctx, [self.vectors[k] for k in names], [self.grads[k] for k in names], *states)
        self.n, self.f, self.df, self.dn, self.r, self.dr, self.answer_n, self.answer_f = [empty((rows, d), dtype) for _ in range(8)]
        self.saved = [empty((max(16, p.saved_bytes(rows)),), torch.uint8) for p in (self.before, self.after)]
        self.ws = empty((max(16, self.before.workspace_bytes(rows), self.after.workspace_bytes(rows)),), torch.uint8)
        if weights[0].is_cuda:
            torch.cuda.current_stream(weights[0].device).synchronize()

    def _of(self, side, grads=False):
        at = self.grads if grads else self.vectors
        return {("d" if grads else "") + k: v for k, v in at.items() if k.startswith(side) or (side == "post" and k == "gate")}

    def normed(self, x, n, stream=None):
        """n = N_pre(x): what is encrypted"""
        self.before.forward(x, None, None, n, **self._of("pre"), stream=stream)

    def joined(self, x, f, r, stream=None):
        """r from x and the block's answers f (decrypted ones, say)"""
        self.after.forward(x, f, r, None, **self._of("post"), stream=stream)

    def answer(self, x, r, stream=None):
        n, f = (t[:x.shape[0]] for t in (self.answer_n, self.answer_f))
        self.normed(x, n, stream)
        self.block.answer(n, f, stream)
        self.joined(x, f, r, stream)

    def step(self, x, loss, lr, vector_lr=1e-3, betas=(0.9, 0.99), eps=1e-8, weight_decay=0.0, stream=None):
        """one step on rows x, like GatedHead.step; vector_lr: of the norms' weights and the gate"""
        rows, b = x.shape[0], self.block
        n, f, df, dn, r, dr = (t[:rows] for t in (self.n, self.f, self.df, self.dn, self.r, self.dr))
        self.before.forward(x, None, None, n, **self._of("pre"), saved=self.saved[0], stream=stream)
        b.ff.forward(n, *b.used, f, b.ws, saved=b.saved, stream=stream)
        self.after.forward(x, f, r, None, **self._of("post"), saved=self.saved[1], stream=stream)
        out = _on_stream(stream, loss, r, dr)
        self.after.backward(x, f, self.saved[1], dr, None, self.ws, df=df, **self._of("post", grads=True), **self._of("post"), stream=stream)
        b.ff.backward(n, *b.used, b.saved, df, dn, *b.grads, b.ws, stream=stream)
        self.before.backward(x, None, self.saved[0], None, dn, self.ws, **self._of("pre", grads=True), **self._of("pre"), stream=stream)
        b._move(lr, betas, eps, weight_decay, stream)
        self.opt.step(vector_lr, betas, eps, 0.0, b.steps, stream=stream)
        return out


class LowBitHead:
    """A trained head's answers in the clear from its matrices in 4 bits, up to `rows` rows a call.  weights: device tensors as for GatedHead (read once,
    here); empty(shape, dtype) allocates on the device.  The constructor waits for what it enqueues: answers may use any stream, but have to be
    ordered after each other, since they share a workspace; one that may run beside others takes its own, of workspace_bytes(rows)."""

    def __init__(self, ctx, rows, weights, act, dtype, empty, group=128):
        import torch

        d_hidden, d_in = weights[0].shape
        self.ff = lowbit.GatedFF4(ctx, d_in, d_hidden, weights[2].shape[0], dtype, act, group)
        self.matrices = []
        for w, plan in zip(weights, (self.ff.into, self.ff.into, self.ff.out)):
            pair = empty(plan.codes_shape, torch.uint8), empty(plan.scales_shape, dtype)
            plan.pack(w, *pair)
            self.matrices.append(pair)
        self.ws = empty((self.workspace_bytes(rows),), torch.uint8)
        if weights[0].is_cuda:
            torch.cuda.current_stream(weights[0].device).synchronize()

    def workspace_bytes(self, rows):
        return max(16, self.ff.workspace_bytes(rows))

    def answer(self, x, y, stream=None, ws=None):
        self.ff.forward(x, *self.matrices, y, self.ws if ws is None else ws, stream=stream)


@dataclass
class HeadPlan:
    act: str
    d_in: int
    d_hidden: int
    d_out: int
    level: int         # of the features
    level_act: int     # of the activated gate
    level_out: int
    scale_out: float
    w_in: np.ndarray   # [2 d_hidden][d_in] int64: the gate's rows, then the others
    w_out: np.ndarray  # [d_out][d_hidden] int64
    consts: object     # of the activation


def plan(w_gate, w_up, w_down, act, q, level, scale):
    """w_*: float arrays; q: ciphertext primes; level, scale: of the features"""
    down = {"linear": 0, "square": 1, "poly2": 2, "poly3": 2}
    if act not in down:
        raise ValueError("%r has no schedule under encryption" % (act,))
    level_in, level_act = level - 1, level - 1 - down[act]
    if level_act < 3:
        raise ValueError("not enough levels for the head")
    consts, s_act = None, scale
    if act == "square":
        s_act = scale * scale / float(q[level_in - 1])
    elif act == "poly2":
        consts = activation.poly2_constants(q, level_in, scale)
        s_act = consts.out_scale
    elif act == "poly3":
        consts = activation.poly3_constants(q, level_in, scale)
        s_act = consts.out_scale

    def whole(w, l):  # at the scale of the prime that the rescale drops: the layer keeps the scale
        return np.rint(np.asarray(w, dtype=np.float64) * float(q[l - 1])).astype(np.int64)

    w_in = whole(np.concatenate([np.asarray(w_gate), np.asarray(w_up)]), level)
    return HeadPlan(act, w_in.shape[1], w_in.shape[0] // 2, np.shape(w_down)[0], level, level_act, level_act - 2, s_act * scale / float(q[level_act - 1]), w_in,
                    whole(w_down, level_act - 1), consts)


def workspace_bytes(ctx, p, max_items=64):
    items = min(p.d_hidden, max_items)
    need = [ctx.conv2d_workspace_bytes(p.d_in, 2 * p.d_hidden, 1, 1, p.level), ctx.conv2d_workspace_bytes(p.d_hidden, p.d_out, 1, 1, p.level_act - 1),
            ctx.workspace_bytes(ckksmi.OP_RESCALE, p.level, min(2 * p.d_hidden, max_items)),
            ctx.workspace_bytes(ckksmi.OP_RESCALE, p.level_act - 1, min(p.d_out, max_items)),
            ctx.workspace_bytes(ckksmi.OP_HMUL_RELIN_RESCALE, p.level_act, items)]
    if p.act == "square":
        need.append(ctx.workspace_bytes(ckksmi.OP_HMUL_RELIN_RESCALE, p.level - 1, items))
    elif p.act != "linear":
        need.append(activation.workspace_bytes(ctx, p.level - 1, items))
    return max(need)


def forward(ctx, p, x, evk, empty, to_dev, ws, stream=None, max_items=64):
    """x: device array of d_in ciphertexts at p.level; empty(*shape) allocates 64-bit words, to_dev(int64 ndarray) uploads; ws as sized
    by workspace_bytes(ctx, p, max_items).  Returns d_out ciphertexts at p.level_out, scale p.scale_out."""
    N, H, l1, la = ctx.N, p.d_hidden, p.level - 1, p.level_act
    mac = empty(2 * H, 2, p.level, N)
    both = empty(2 * H, 2, l1, N)
    ctx.fc_mac(x, to_dev(p.w_in), p.d_in, 2 * H, mac, p.level, ws, stream=stream)
    ctx.rescale(mac, both, p.level, 2 * H, ws, stream=stream)
    words = 2 * l1 * N
    flat = both.reshape(-1)
    gate, up = flat[:H * words], flat[H * words:]
    if p.act == "linear":
        a = gate
    else:
        a = empty(H, 2, la, N)
        if p.act == "square":
            ctx.hmul_relin_rescale(gate, gate, evk, a, l1, H, ws, stream=stream)
        else:
            schedule, af, wa = getattr(activation, p.act), a.reshape(-1), 2 * la * N
            for i in range(0, H, max_items):
                n = min(max_items, H - i)
                schedule(ctx, gate[i * words:(i + n) * words], evk, af[i * wa:(i + n) * wa], l1, n, p.consts, ws, stream=stream)
    if la < l1:
        dropped = empty(H, 2, la, N)
        ctx.mod_drop(up, l1, la, dropped, H, stream=stream)
        up = dropped
    h = empty(H, 2, la - 1, N)
    ctx.hmul_relin_rescale(a, up, evk, h, la, H, ws, stream=stream)
    mac = empty(p.d_out, 2, la - 1, N)
    y = empty(p.d_out, 2, p.level_out, N)
    ctx.fc_mac(h, to_dev(p.w_out), H, p.d_out, mac, la - 1, ws, stream=stream)
    ctx.rescale(mac, y, la - 1, p.d_out, ws, stream=stream)
    return y
