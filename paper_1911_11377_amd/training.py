"""Training in the clear of weights that are evaluated under encryption (argument marshalling only).

The paper trains its network on plain data with the polynomials that replace the activations (sections 2.2, 3.2).  Two
operators, plans over the entry points of include/ckksmi_train.h:
  GatedFF : y = (act(x Wg^T) * (x Wu^T)) Wd^T, forward and backward; act a cubic of the encrypted schedules or what they replace
  AdamW   : one optimiser step over many tensors, states in 32 or 8 bits
Device buffers are torch tensors on the context's GPU and stay the caller's; calls enqueue on torch's current stream unless
told otherwise and allocate nothing.
"""
import ctypes as C

from . import activation, ckksmi

# the activations of activation.py as cubics c0 + c1 g + c2 g^2 + c3 g^3
CUBICS = {
    "linear": (0.0, 1.0, 0.0, 0.0),
    "square": (0.0, 0.0, 1.0, 0.0),
    "poly2": (0.0, activation.PAPER_POLY2[1], activation.PAPER_POLY2[0], 0.0),
    "poly3": (0.5, 0.25, 0.0, -0.02),
}
_OTHERS = {"relu": ckksmi.ACT_RELU, "silu": ckksmi.ACT_SILU, "gelu": ckksmi.ACT_GELU}


def _dtype_code(dtype):
    import torch

    codes = {torch.float32: ckksmi.F32, torch.bfloat16: ckksmi.BF16, torch.float16: ckksmi.F16}
    if dtype not in codes:
        raise ValueError("expected float32, bfloat16 or float16, got %r" % (dtype,))
    return codes[dtype]


class GatedFF:
    """Plan of a gated feed-forward block of fixed widths and types; any number of rows.

    activation: a name of CUBICS, "relu" | "silu" | "gelu", or four coefficients of a cubic."""

    def __init__(self, ctx, d_in, d_hidden, d_out, dtype, activation, grad_dtype=None):
        self.ctx, self.d_in, self.d_hidden, self.d_out = ctx, d_in, d_hidden, d_out
        self.dtype, self.grad_dtype = dtype, grad_dtype or dtype
        s = ckksmi.GatedFFShape()
        s.dtype, s.grad_dtype = _dtype_code(dtype), _dtype_code(self.grad_dtype)
        s.d_in, s.d_hidden, s.d_out = d_in, d_hidden, d_out
        if isinstance(activation, str) and activation in _OTHERS:
            s.act = _OTHERS[activation]
        else:
            cubic = CUBICS[activation] if isinstance(activation, str) else tuple(activation)
            if len(cubic) != 4:
                raise ValueError("a cubic has four coefficients")
            s.act, s.c = ckksmi.ACT_POLY, (C.c_float * 4)(*cubic)
        self._s, self._r = s, C.byref(s)  # what all calls have in common
        self._saved_of = (0, 0)  # rows of some call and what they save: replaced as a whole

    def _shape(self, rows, ld_x=0, ld_y=0, ld_dy=0, ld_dx=0):
        """a call's own sizes: calls from several threads do not meet in one structure"""
        s = ckksmi.GatedFFShape.from_buffer_copy(self._s)
        s.rows, s.ld_x, s.ld_y = rows, ld_x, ld_y
        if ld_dy:
            s.ld_dy, s.ld_dx = ld_dy, ld_dx
        return C.byref(s)

    def _bytes(self, name, rows, *args):
        n = C.c_size_t(0)
        self.ctx._call(name, self.ctx._h, self._shape(rows), *args, C.byref(n))
        return n.value

    def workspace_bytes(self, rows, backward=False):
        """for forward calls on up to `rows` rows; backward: for either pass"""
        return self._bytes("ckksmi_gated_ff_workspace_bytes", rows, 1 if backward else 0)

    def saved_bytes(self, rows):
        return self._bytes("ckksmi_gated_ff_saved_bytes", rows)

    def _rows_of(self, x, width, dtype, rows=None):
        """a [rows][width] tensor whose rows are contiguous: address and distance of its rows"""
        if x.dim() != 2 or x.shape[1] != width or (rows is not None and x.shape[0] != rows) or x.dtype != dtype:
            raise ValueError("expected [%s][%d] of %s, got %s of %s" % ("rows" if rows is None else rows, width, dtype, tuple(x.shape), x.dtype))
        if x.stride(1) != 1 and width > 1:
            raise ValueError("rows must be contiguous")
        if x.shape[0] > 1 and x.stride(0) < width:  # (0, a row repeated by expand(), would be taken for dense rows)
            raise ValueError("rows must not overlap: %d elements apart, %d wide" % (x.stride(0), width))
        return x.data_ptr(), x.stride(0) if x.shape[0] > 1 else width

    def _matrix(self, w, d0, d1, dtype):
        if tuple(w.shape) != (d0, d1) or w.dtype != dtype:
            raise ValueError("expected [%d][%d] of %s, got %s of %s" % (d0, d1, dtype, tuple(w.shape), w.dtype))
        return ckksmi._ptr(w)

    def _weights(self, w_gate, w_up, w_down, dtype):
        return (self._matrix(w_gate, self.d_hidden, self.d_in, dtype), self._matrix(w_up, self.d_hidden, self.d_in, dtype),
                self._matrix(w_down, self.d_out, self.d_hidden, dtype))

    def _saved(self, saved, rows):
        of = self._saved_of
        if of[0] != rows:
            of = self._saved_of = (rows, self.saved_bytes(rows))
        if ckksmi._nbytes(saved) < of[1]:
            raise ValueError("the buffer for saved activations holds %d bytes of %d" % (ckksmi._nbytes(saved), of[1]))
        return ckksmi._ptr(saved)

    def forward(self, x, w_gate, w_up, w_down, y, ws, saved=None, stream=None):
        """y = (act(x Wg^T) * (x Wu^T)) Wd^T; saved: a buffer of saved_bytes(rows) for the backward pass, or None"""
        rows = x.shape[0]
        sp = self._saved(saved, rows) if saved is not None else None
        px, ld_x = self._rows_of(x, self.d_in, self.dtype)
        py, ld_y = self._rows_of(y, self.d_out, self.dtype, rows)
        self.ctx._call("ckksmi_gated_ff_forward", self.ctx._h, self._shape(rows, ld_x, ld_y), px, *self._weights(w_gate, w_up, w_down, self.dtype), py, sp, ckksmi._ptr(ws),
                       ckksmi._nbytes(ws), self.ctx._stream(stream))

    def backward(self, x, w_gate, w_up, w_down, saved, dy, dx, dw_gate, dw_up, dw_down, ws, accumulate=False, stream=None):
        """gradients of the weights (added to the buffers' contents if accumulate) and of x (dx may be None)"""
        rows = x.shape[0]
        sp = self._saved(saved, rows)
        px, ld_x = self._rows_of(x, self.d_in, self.dtype)
        pdy, ld_dy = self._rows_of(dy, self.d_out, self.dtype, rows)
        pdx, ld_dx = self._rows_of(dx, self.d_in, self.dtype, rows) if dx is not None else (None, 0)
        self.ctx._call("ckksmi_gated_ff_backward", self.ctx._h, self._shape(rows, ld_x, 0, ld_dy, ld_dx), px, *self._weights(w_gate, w_up, w_down, self.dtype), sp, pdy, pdx,
                       *self._weights(dw_gate, dw_up, dw_down, self.grad_dtype), 1 if accumulate else 0, ckksmi._ptr(ws), ckksmi._nbytes(ws), self.ctx._stream(stream))


def _refuse_overlaps(written, read):
    """raises ValueError where a tensor that is written shares a byte with any other one"""
    ranges = sorted((t.data_ptr(), t.data_ptr() + ckksmi._nbytes(t), w) for ts, w in ((written, True), (read, False)) for t in ts if t.numel())
    end = written_end = 0  # of those that begin before
    for a, b, w in ranges:
        if a < (end if w else written_end):
            raise ValueError("tensors overlap or are listed twice")
        end, written_end = max(end, b), max(written_end, b) if w else written_end


class AdamW:
    """Plan of an optimiser step over a list of tensors.

    params, grads: tensors of one type each; m, v: float32 tensors, or uint8 with m_units, v_units (float32, one value per
    STATE_BLOCK elements of a tensor): 8-bit states.  copies: bfloat16 or float16 copies of the
    parameters, renewed by the step.  The buffers are the caller's; the plan keeps them.  No tensor that a step writes may overlap another."""

    def __init__(self, ctx, params, grads, m, v, m_units=None, v_units=None, copies=None):
        import torch

        self.ctx, self.n = ctx, len(params)
        self._keep = (params, grads, m, v, m_units, v_units, copies)
        lists = [x for x in self._keep if x is not None]
        if any(len(x) != self.n for x in lists):
            raise ValueError("lists of different lengths")
        self.bits = 8 if m_units is not None else 32
        if (m_units is None) != (v_units is None):
            raise ValueError("8-bit states have units for both")
        state = torch.uint8 if self.bits == 8 else torch.float32
        kinds = [(x, {t.dtype for t in x}) for x in lists]
        if any(len(k) > 1 for _, k in kinds):
            raise ValueError("tensors of one list have one type")
        for x, want in ((m, state), (v, state), (m_units, torch.float32), (v_units, torch.float32)):
            if x is not None and any(t.dtype != want for t in x):
                raise ValueError("states are float32, or uint8 with float32 units")
        _refuse_overlaps([t for x in (params, m, v, m_units, v_units, copies) if x is not None for t in x], grads)
        o = ckksmi.AdamWParams()
        o.p_dtype = _dtype_code(params[0].dtype) if self.n else ckksmi.F32
        o.grad_dtype = _dtype_code(grads[0].dtype) if self.n else ckksmi.F32
        o.copy_dtype = _dtype_code(copies[0].dtype) if copies else ckksmi.BF16
        o.state_bits = self.bits
        o.step = 1
        self._o = o  # what all steps have in common
        self._t = (ckksmi.AdamWTensor * max(self.n, 1))()
        for i in range(self.n):
            t, n = self._t[i], params[i].numel()
            blocks = -(-n // ckksmi.STATE_BLOCK)
            for x, want in ((grads, n), (m, n), (v, n), (copies, n), (m_units, blocks), (v_units, blocks)):
                if x is not None and x[i].numel() != want:
                    raise ValueError("tensor %d: %d elements where %d belong" % (i, x[i].numel(), want))
            t.p, t.grad, t.m, t.v, t.n = ckksmi._ptr(params[i]), ckksmi._ptr(grads[i]), ckksmi._ptr(m[i]), ckksmi._ptr(v[i]), n
            if self.bits == 8:
                t.m_unit, t.v_unit = ckksmi._ptr(m_units[i]), ckksmi._ptr(v_units[i])
            if copies is not None:
                t.copy = ckksmi._ptr(copies[i])

    def step(self, lr, betas, eps, weight_decay, step, grad_scale=1.0, seed=0, skip=None, stream=None):
        """step: 1, 2, ..; seed: another one at every step (8-bit states); skip: None or a device int32 that, if not 0, makes the step do nothing"""
        if skip is not None and not isinstance(skip, int):
            import torch

            if skip.dtype != torch.int32 or skip.numel() < 1:  # four bytes are read there
                raise ValueError("skip is an int32 on the device, got %s of %s" % (tuple(skip.shape), skip.dtype))
        o = ckksmi.AdamWParams.from_buffer_copy(self._o)
        o.lr, o.beta1, o.beta2, o.eps, o.weight_decay, o.grad_scale, o.step = lr, betas[0], betas[1], eps, weight_decay, grad_scale, step
        o.seed, o.skip = seed & (2**64 - 1), ckksmi._ptr(skip)
        self.ctx._call("ckksmi_adamw_step", self.ctx._h, C.byref(o), self._t, self.n, self.ctx._stream(stream))

    def read_states(self, m_out=None, v_out=None, stream=None):
        """8-bit states as the float32 values they stand for, into lists of tensors (either may be left out)"""
        import torch

        if self.bits != 8:
            raise ValueError("32-bit states are their own values")
        arrays = []
        for x in (m_out, v_out):
            if x is None:
                arrays.append(None)
                continue
            if len(x) != self.n or any(t.numel() != self._t[i].n or t.dtype != torch.float32 for i, t in enumerate(x)):
                raise ValueError("expected float32 tensors of the parameters' sizes")
            arrays.append((C.c_void_p * max(self.n, 1))(*[ckksmi._ptr(t) for t in x]))
        self.ctx._call("ckksmi_adamw_read_states", self.ctx._h, self._t, self.n, *arrays, self.ctx._stream(stream))
