"""Answers in the clear from weights in 4 bits (argument marshalling only).

A trained head answers single requests at the speed its weights are read.  Plans over the entry points of include/ckksmi_train.h:
  Product4 : y = x W^T, W held as codes of 4 bits with a scale for every `group` of neighbouring elements of a row
  GatedFF4 : y = (act(x Wg^T) * (x Wu^T)) Wd^T from three such matrices
A matrix is a pair (codes, scales): codes uint8 [d_out][round_up(d_in, 32) / 2], two's complement, the even element of a pair in the lower
half; scales [d_out][ceil(d_in / group)] of the plan's type.  `pack` makes them from a matrix, with the nearest codes.
Device buffers are torch tensors on the context's GPU and stay the caller's; calls enqueue on torch's current stream unless
told otherwise and allocate nothing.  Meant for up to 64 rows; each further 64 read the codes again.
"""
import ctypes as C

from . import ckksmi
from .training import _dtype_code, _rows_or_dense, activation_code


class Product4:
    """Plan of products with a d_out x d_in matrix in 4 bits; any number of rows.  group: 32, 64, .. 1024; dtype: of x, y and the scales"""

    def __init__(self, ctx, d_in, d_out, dtype, group=128):
        import torch

        self.ctx, self.d_in, self.d_out, self.dtype, self.group, self._uint8 = ctx, d_in, d_out, dtype, group, torch.uint8
        self.codes_shape = (d_out, -(-d_in // 32) * 16)
        self.scales_shape = (d_out, -(-d_in // group) if group > 0 else 0)
        m = ckksmi.Matrix4()
        m.dtype, m.group, m.d_in, m.d_out = _dtype_code(dtype), group, d_in, d_out
        self._m, self._r = m, C.byref(m)

    def _weights(self, codes, scales):
        if (codes.shape != self.codes_shape or codes.dtype != self._uint8 or scales.shape != self.scales_shape or scales.dtype != self.dtype or not codes.is_contiguous()
                or not scales.is_contiguous()):
            raise ValueError("expected contiguous codes %s and scales %s of %s, got %s of %s and %s of %s" % (
                self.codes_shape, self.scales_shape, self.dtype, tuple(codes.shape), codes.dtype, tuple(scales.shape), scales.dtype))
        return codes.data_ptr(), scales.data_ptr()

    def _matrix(self, w):
        if tuple(w.shape) != (self.d_out, self.d_in):
            raise ValueError("expected [%d][%d], got %s" % (self.d_out, self.d_in, tuple(w.shape)))
        return _dtype_code(w.dtype), ckksmi._ptr(w)

    def pack(self, w, codes, scales, stream=None):
        """nearest codes and scales of w (float32, bfloat16 or float16): scale = largest magnitude of a group / 7"""
        code, p = self._matrix(w)
        self.ctx._call("ckksmi_pack4", self.ctx._h, self._r, code, p, *self._weights(codes, scales), self.ctx._stream(stream))

    def unpack(self, codes, scales, w, stream=None):
        """w = scale * code, rounded to w's type"""
        code, p = self._matrix(w)
        self.ctx._call("ckksmi_unpack4", self.ctx._h, self._r, code, *self._weights(codes, scales), p, self.ctx._stream(stream))

    def forward(self, x, codes, scales, y, stream=None):
        """y = x W^T"""
        rows, ctx = x.shape[0], self.ctx
        px, ld_x = _rows_or_dense(x, rows, self.d_in, self.dtype)
        py, ld_y = _rows_or_dense(y, rows, self.d_out, self.dtype)
        ctx._call("ckksmi_product4", ctx._h, self._r, rows, px, ld_x, *self._weights(codes, scales), py, ld_y, ctx._stream(stream))


class GatedFF4:
    """Plan of a gated feed-forward block whose matrices are in 4 bits.  activation as for training.GatedFF; `into` and `out` are the
    plans of its matrices (for pack): d_hidden x d_in (twice) and d_out x d_hidden"""

    def __init__(self, ctx, d_in, d_hidden, d_out, dtype, activation, group=128):
        self.ctx = ctx
        self.into, self.out = Product4(ctx, d_in, d_hidden, dtype, group), Product4(ctx, d_hidden, d_out, dtype, group)
        s = ckksmi.GatedFF4Shape()
        s.dtype, s.group, s.d_in, s.d_hidden, s.d_out = _dtype_code(dtype), group, d_in, d_hidden, d_out
        s.act, s.c = activation_code(activation)
        self._s = s  # what all calls have in common

    def _shape(self, rows, ld_x=0, ld_y=0):
        s = ckksmi.GatedFF4Shape.from_buffer_copy(self._s)
        s.rows = rows
        if ld_x or ld_y:
            s.ld_x, s.ld_y = ld_x, ld_y
        return C.byref(s)

    def workspace_bytes(self, rows):
        """for calls on up to `rows` rows"""
        n = C.c_size_t(0)
        self.ctx._call("ckksmi_gated_ff4_workspace_bytes", self.ctx._h, self._shape(rows), C.byref(n))
        return n.value

    def forward(self, x, gate, up, down, y, ws, stream=None):
        """gate, up, down: pairs (codes, scales)"""
        rows, ctx, into, out = x.shape[0], self.ctx, self.into, self.out
        px, ld_x = _rows_or_dense(x, rows, into.d_in, into.dtype)
        py, ld_y = _rows_or_dense(y, rows, out.d_out, out.dtype)
        ctx._call("ckksmi_gated_ff4_forward", ctx._h, self._shape(rows, ld_x, ld_y), px, *into._weights(*gate), *into._weights(*up), *out._weights(*down), py, ckksmi._ptr(ws),
                  ckksmi._nbytes(ws), ctx._stream(stream))
