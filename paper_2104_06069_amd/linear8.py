"""A linear layer in 8 bits on the device (include/ob_layer.h): y = x W^T and both gradients from numbers of 8 bits with a scale for
each block of 128, argument checks and buffers around the calls.

    layer = Linear8(k, n, dtype=torch.bfloat16)
    w8 = layer.quantize_weight(w)                      # w [n, k], once for weights that stay, once a step for weights that are trained
    y = layer.forward(x, w8)                           # x in 16 or 32 bits, or a Matrix8 (RMSNorm.forward8 makes such)
    dx, dw = layer.backward(x, dy, w8, dw=flat_grad[a:b].view(n, k))

or, with torch's autograd, y = layer(x, w).
"""
from typing import NamedTuple

import torch
from torch.autograd.function import once_differentiable

from . import binding as ob
from .matrix8 import FORMATS, Matrix8, adjacent, format_of, rows_of
from .step import _OB_DTYPE, _current_stream

_TYPES = tuple(_OB_DTYPE)
_E4M3 = torch.float8_e4m3fn
_NO_MATRIX = (None, 0, None, 0)


class Weight8(NamedTuple):
    """W [n, k] in 8 bits and its transpose [k, n], with one scale for each 128 x 128 of it."""
    w: Matrix8
    transposed: Matrix8


class Linear8:
    def __init__(self, k, n, dtype=torch.bfloat16, grad_format=_E4M3, max_rows=1 << 22, device="cuda:0"):
        """dtype: of results, unless a call says otherwise; grad_format: of dy in 8 bits.  Products of few tiles share the object's
        workspace: calls on one object, those of autograd among them, must not overlap in time; on several streams, each has to wait for
        the one before.  The object holds no weights, only 32 MB of workspace: layers of one shape may share it."""
        self.device = torch.device(device)
        torch.cuda.set_device(self.device)
        self.ctx = None
        self.k, self.n, self.dtype, self.grad_format, self.max_rows = int(k), int(n), dtype, grad_format, int(max_rows)
        format_of(grad_format)
        if dtype not in _OB_DTYPE:
            raise ValueError("dtype is torch.float32, torch.float16 or torch.bfloat16")
        L = ob.lib()
        self._calls = L.ob_linear8_quantize, L.ob_linear8_forward, L.ob_linear8_input_grad, L.ob_linear8_weight_grad, L.ob_linear8_forward_few
        self._index = torch.cuda.current_device()
        self.ctx = ob.ob_linear8_create(self.k, self.n, max_rows)
        # rows whose numbers the product itself makes 8 bits (one launch): few, or short ones, up to 512 blocks of 128 in all, 127 in a row
        blocks = (self.k + 127) // 128
        self._few_rows = min(ob.OB_LINEAR8_FEW_ROWS, 512 // blocks) if blocks < 128 else 0

    def close(self):
        if self.ctx is not None:
            torch.cuda.synchronize(self.device)
            ob.ob_linear8_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # (A small layer's calls take 5 to 10 us on the device each: the common cases are looked at as a whole, anything else piece by piece, and
    # the library is called without a stop in between.)
    def _check(self, status, where):
        if status:
            raise ob.ObLambError(status, where, ob.lib().ob_linear8_last_hip_error(self.ctx).decode())

    def _rows(self, t, width, what):
        """The distance between t's rows"""
        if t.dim() == 2 and t.shape[1] == width and t.dtype in _OB_DTYPE and t.is_contiguous() and t.get_device() == self._index:
            return width
        return rows_of(t, width, _TYPES, self.device, what)

    def _quantize(self, t, what, width, rows_format=None, cols_format=None, square=False):
        """-> (t, t transposed) in the given formats, None where that is None"""
        if not isinstance(t, torch.Tensor):
            raise ValueError(f"{what}: a tensor, not {type(t).__name__}")
        ld, (rows, cols) = self._rows(t, width, what), t.shape
        m = None if rows_format is None else Matrix8(rows, cols, rows_format, self.device, square)
        mt = None if cols_format is None else Matrix8(cols, rows, cols_format, self.device, square)
        self._check(self._calls[0](self.ctx, t.data_ptr(), _OB_DTYPE[t.dtype], ld, rows, cols, ob.OB_BLOCK_SQUARE if square else ob.OB_BLOCK_ROWS,
                                   0 if m is None else FORMATS[rows_format], 0 if mt is None else FORMATS[cols_format],
                                   *(_NO_MATRIX if m is None else m.address()), *(_NO_MATRIX if mt is None else mt.address()), _current_stream(self.device)),
                    "ob_linear8_quantize")
        return m, mt

    def quantize(self, t, format=_E4M3):
        """t [rows, any width] in 8 bits, a scale for each 128 columns of a row."""
        format_of(format)
        if not isinstance(t, torch.Tensor) or t.dim() != 2:
            raise ValueError("t: a [rows, width] tensor")
        return self._quantize(t, "t", t.shape[1], rows_format=format)[0]

    def quantize_weight(self, w):
        """w [n, k] of torch.float32, torch.float16 or torch.bfloat16 -> Weight8."""
        if w.dim() != 2 or w.shape[0] != self.n:
            raise ValueError(f"w: a [{self.n}, {self.k}] tensor, not {tuple(w.shape)}")
        return Weight8(*self._quantize(w, "w", self.k, _E4M3, _E4M3, square=True))

    def _matrix(self, t, width, format, what):
        if isinstance(t, Matrix8):
            if t.cols != width or t.square or t.device != self.device:
                raise ValueError(f"{what}: [rows, {width}] with scales of rows, on {self.device}")
            return t
        return self._quantize(t, what, width, rows_format=format)[0]

    def _out(self, out, rows, width, dtype, dtypes, what="out"):
        if out is None:
            if dtype not in dtypes:
                raise ValueError(f"{what}: {' or '.join(map(str, dtypes))}, not {dtype}")
            return torch.empty((rows, width), device=self.device, dtype=dtype), width
        ld = rows_of(out, width, dtypes, self.device, what)
        if out.shape[0] != rows:
            raise ValueError(f"{what}: {rows} rows")
        return out, ld

    def _weight(self, w8):
        if isinstance(w8, Weight8):
            w, t = w8
            if w.rows == t.cols == self.n and w.cols == t.rows == self.k and w.square and t.square and w.dtype is t.dtype is _E4M3 and w.device == t.device == self.device:
                return
        raise ValueError(f"w8: the Weight8 of a [{self.n}, {self.k}] tensor on {self.device}")

    def forward(self, x, w8, out=None, out_dtype=None):
        """y = x W^T; x is quantised to e4m3 unless it is a Matrix8."""
        self._weight(w8)
        if not isinstance(x, Matrix8) and x.dim() == 2 and x.shape[0] <= self._few_rows:
            rows, ldx = x.shape[0], self._rows(x, self.k, "x")
            out, ldo = self._out(out, rows, self.n, out_dtype or self.dtype, _TYPES)
            self._check(self._calls[4](self.ctx, x.data_ptr(), _OB_DTYPE[x.dtype], ldx, ob.OB_E4M3, *w8.w.address(), rows, out.data_ptr(), ldo,
                                       _OB_DTYPE[out.dtype], _current_stream(self.device)), "ob_linear8_forward_few")
            return out
        m = self._matrix(x, self.k, _E4M3, "x")
        out, ldo = self._out(out, m.rows, self.n, out_dtype or self.dtype, _TYPES)
        self._check(self._calls[1](self.ctx, *m.address(), FORMATS[m.dtype], *w8.w.address(), m.rows, out.data_ptr(), ldo, _OB_DTYPE[out.dtype],
                                   _current_stream(self.device)), "ob_linear8_forward")
        return out

    def input_grad(self, dy, w8, out=None, out_dtype=None):
        """dx = dy W; dy is quantised to grad_format unless it is a Matrix8."""
        self._weight(w8)
        m = self._matrix(dy, self.n, self.grad_format, "dy")
        out, ldo = self._out(out, m.rows, self.k, out_dtype or self.dtype, _TYPES)
        self._check(self._calls[2](self.ctx, *m.address(), FORMATS[m.dtype], *w8.transposed.address(), m.rows, out.data_ptr(), ldo, _OB_DTYPE[out.dtype],
                                   _current_stream(self.device)), "ob_linear8_input_grad")
        return out

    def weight_grad(self, x, dy, out=None, out_dtype=torch.float32, accumulate=False):
        """dW = dy^T x, or with accumulate (a float32 `out`) dW += dy^T x.  x and dy are tensors: their blocks run along the rows here."""
        return self._weight_grad(x, dy, self._quantize(dy, "dy", self.n, cols_format=self.grad_format)[1], out, out_dtype, accumulate)

    def _weight_grad(self, x, dy, dy_t, out, out_dtype, accumulate):
        if not isinstance(x, torch.Tensor) or x.shape[:1] != dy.shape[:1]:
            raise ValueError("x and dy: tensors of one row each")
        x_t = self._quantize(x, "x", self.k, cols_format=_E4M3)[1]
        if accumulate and out is None:
            raise ValueError("accumulate needs an out to add to")
        out, ldo = self._out(out, self.n, self.k, out_dtype, (torch.float32,) if accumulate else _TYPES)
        self._check(self._calls[3](self.ctx, *dy_t.address(), FORMATS[dy_t.dtype], *x_t.address(), x.shape[0], out.data_ptr(), ldo, _OB_DTYPE[out.dtype],
                                   bool(accumulate), _current_stream(self.device)), "ob_linear8_weight_grad")
        return out

    def backward(self, x, dy, w8, dw=None, dw_dtype=torch.float32, accumulate=False):
        """-> (dx, dW), with one pass over dy for both of its forms in 8 bits."""
        self._weight(w8)
        m, mt = self._quantize(dy, "dy", self.n, self.grad_format, self.grad_format)
        return self.input_grad(m, w8), self._weight_grad(x, dy, mt, dw, dw_dtype, accumulate)

    def __call__(self, x, w):
        return _Apply.apply(x, w, self)


class _Apply(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w, layer):
        w8 = layer.quantize_weight(w)
        ctx.layer, ctx.w8, ctx.w_dtype = layer, w8, w.dtype
        ctx.save_for_backward(x)
        return layer.forward(x, w8)

    @staticmethod
    @once_differentiable      # (what the calls write has no graph: a derivative of it raises)
    def backward(ctx, dy):
        x, = ctx.saved_tensors
        dy = dy if adjacent(dy) else dy.contiguous()      # (a sum's gradient is one element, seen as all of them)
        dx, dw = None, None
        if all(ctx.needs_input_grad[:2]):
            dx, dw = ctx.layer.backward(x, dy, ctx.w8, dw_dtype=ctx.w_dtype)
        elif ctx.needs_input_grad[0]:
            dx = ctx.layer.input_grad(dy, ctx.w8)
        elif ctx.needs_input_grad[1]:
            dw = ctx.layer.weight_grad(x, dy, out_dtype=ctx.w_dtype)
        return None if dx is None else dx.to(x.dtype), dw, None
