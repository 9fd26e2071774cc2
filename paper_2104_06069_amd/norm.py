"""Root-mean-square norm of rows with the residual's addition on the device (include/ob_layer.h): argument checks and output
buffers around the calls.

    norm = RMSNorm(width, dtype=torch.bfloat16)
    y, h, rstd = norm.forward(x, weight, residual)            # h = x + residual, y = h rstd weight
    y8, h, rstd = norm.forward8(x, weight, residual)          # y in 8 bits, for Linear8.forward
    dh, dweight = norm.backward(dy, h, rstd, weight, dres)    # dres: the gradient that comes down the residual

or, with torch's autograd, y, h = norm(x, weight, residual), or y = norm(x, weight).
"""
import torch
from torch.autograd.function import once_differentiable

from . import binding as ob
from .matrix8 import Matrix8, adjacent, format_of, rows_of
from .step import _OB_DTYPE, _current_stream


class RMSNorm:
    def __init__(self, n, dtype=torch.bfloat16, residual_dtype=None, weight_dtype=torch.float32, eps=1e-6, device="cuda:0"):
        """n: 1 to 16384.  dtype: of x, y and dy; residual_dtype: of residual, h and their gradients, dtype or torch.float32 (default: dtype).
        Weight gradients share the object's workspace: calls of backward on one object must not overlap in time; on several streams,
        each has to wait for the one before.  The object holds no weights, only that workspace: layers of one width may share it."""
        self.device = torch.device(device)
        torch.cuda.set_device(self.device)
        self.n, self.dtype, self.residual_dtype, self.weight_dtype = int(n), dtype, residual_dtype or dtype, weight_dtype
        self.ctx = None
        if dtype not in _OB_DTYPE or self.residual_dtype not in (dtype, torch.float32) or weight_dtype not in _OB_DTYPE:
            raise ValueError("types are torch.float32, torch.float16 and torch.bfloat16; the residual's is dtype or torch.float32")
        self._index, self._call, self._backward = torch.cuda.current_device(), ob.lib().ob_norm_forward, ob.lib().ob_norm_backward
        self.ctx = ob.ob_norm_create(self.n, _OB_DTYPE[dtype], _OB_DTYPE[self.residual_dtype], _OB_DTYPE[weight_dtype], eps)

    def close(self):
        if self.ctx is not None:
            torch.cuda.synchronize(self.device)
            ob.ob_norm_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _like(self, t, rows, dtype, what):
        """(t, the distance between its rows), a new one where t is None"""
        if t is None:
            return torch.empty((rows, self.n), device=self.device, dtype=dtype), self.n
        ld = rows_of(t, self.n, (dtype,), self.device, what)
        if t.shape[0] != rows:
            raise ValueError(f"{what}: {rows} rows")
        return t, ld

    def _weight(self, t):
        if t is not None and (t.dtype is not self.weight_dtype or t.shape != (self.n,) or not t.is_contiguous() or t.get_device() != self._index):
            raise ValueError(f"weight: {self.n} adjacent {self.weight_dtype} on {self.device}")

    def _forward(self, x, weight, residual, h, y, want_y, format):
        # (a token's norm takes 3 us on the device: the common case is looked at as a whole, anything else piece by piece)
        n, rows = self.n, x.shape[0]
        dense, ldr, ldh, ldy = (rows, n), n, n, n
        whole = x.dtype is self.dtype and x.shape == dense and x.is_contiguous() and x.get_device() == self._index
        ldx = n if whole else rows_of(x, n, (self.dtype,), self.device, "x")
        self._weight(weight)
        if residual is None:
            if h is not None:
                raise ValueError("h is x where there is no residual")
        else:
            if residual.dtype is self.residual_dtype and residual.shape == dense and residual.is_contiguous() and residual.get_device() == self._index:
                if h is None:
                    h = torch.empty_like(residual)
            else:
                residual, ldr = self._like(residual, rows, self.residual_dtype, "residual")
            if h is None or h.shape != dense or h.dtype is not self.residual_dtype or not h.is_contiguous() or h.get_device() != self._index:
                h, ldh = self._like(h, rows, self.residual_dtype, "h")
        if want_y:
            if y is None and whole:
                y = torch.empty_like(x)
            else:
                y, ldy = self._like(y, rows, self.dtype, "out")
        m8, data, ld, scales, ld_scales, code = None, None, 0, None, 0, 0
        if format is not None:
            code = format_of(format)
            m8 = Matrix8(rows, n, format, self.device)
            data, ld, scales, ld_scales = m8.address()
        rstd = torch.empty(rows, device=self.device, dtype=torch.float32)
        status = self._call(self.ctx, x.data_ptr(), ldx, None if residual is None else residual.data_ptr(), ldr, None if weight is None else weight.data_ptr(), rows,
                            None if h is None else h.data_ptr(), ldh, y.data_ptr() if want_y else None, ldy, data, ld, scales, ld_scales, code, rstd.data_ptr(),
                            _current_stream(self.device))
        if status:
            raise ob.ObLambError(status, "ob_norm_forward", ob.lib().ob_norm_last_hip_error(self.ctx).decode())
        return y, m8, (x if residual is None else h), rstd

    def forward(self, x, weight=None, residual=None, h=None, out=None):
        """-> (y, h, rstd).  h: where x + residual goes (default: a new tensor); it may be residual itself, or x if their types are
        one.  Without a residual, h is x."""
        y, _, h, rstd = self._forward(x, weight, residual, h, out, True, None)
        return y, h, rstd

    def forward8(self, x, weight=None, residual=None, h=None, out=None, format=torch.float8_e4m3fn):
        """-> (y as a Matrix8, h, rstd).  out: where y goes in x's type too, for a weight gradient that reads it later."""
        _, m8, h, rstd = self._forward(x, weight, residual, h, out, out is not None, format)
        return m8, h, rstd

    def backward(self, dy, h, rstd, weight=None, dres=None, dweight=None, accumulate=False, out=None):
        """-> (dh, dweight): the gradient of h, so of x and of the residual alike, and of the weight in float32 (into `dweight` if
        given; with accumulate, added to what it holds).  dres: the gradient that h has from elsewhere."""
        n, rows, index = self.n, dy.shape[0], self._index
        dense, lddy, ldh, lddres, lddh = (rows, n), n, n, n, n
        if not (dy.dtype is self.dtype and dy.shape == dense and dy.is_contiguous() and dy.get_device() == index):
            lddy = rows_of(dy, n, (self.dtype,), self.device, "dy")
        whole = h.dtype is self.residual_dtype and h.shape == dense and h.is_contiguous() and h.get_device() == index
        if not whole:
            h, ldh = self._like(h, rows, self.residual_dtype, "h")
        self._weight(weight)
        if rstd.dtype is not torch.float32 or rstd.shape != (rows,) or not rstd.is_contiguous() or rstd.get_device() != index:
            raise ValueError(f"rstd: {rows} adjacent torch.float32 on {self.device}")
        if dres is not None and not (dres.dtype is self.residual_dtype and dres.shape == dense and dres.is_contiguous() and dres.get_device() == index):
            dres, lddres = self._like(dres, rows, self.residual_dtype, "dres")
        if out is None and whole:
            dh = torch.empty_like(h)
        else:
            dh, lddh = self._like(out, rows, self.residual_dtype, "out")
        if dweight is None:
            if accumulate:
                raise ValueError("accumulate needs a dweight to add to")
            dweight = torch.empty(n, device=self.device, dtype=torch.float32)
        elif dweight.dtype is not torch.float32 or dweight.shape != (n,) or not dweight.is_contiguous() or dweight.get_device() != index:
            raise ValueError(f"dweight: {n} adjacent torch.float32 on {self.device}")
        status = self._backward(self.ctx, dy.data_ptr(), lddy, h.data_ptr(), ldh, rstd.data_ptr(), None if weight is None else weight.data_ptr(),
                                None if dres is None else dres.data_ptr(), lddres, rows, dh.data_ptr(), lddh, dweight.data_ptr(), bool(accumulate),
                                _current_stream(self.device))
        if status:
            raise ob.ObLambError(status, "ob_norm_backward", ob.lib().ob_norm_last_hip_error(self.ctx).decode())
        return dh, dweight

    def __call__(self, x, weight=None, residual=None):
        """-> y, or with a residual (y, h)"""
        if self.residual_dtype != self.dtype and residual is None:
            raise ValueError("without a residual, h is x: a norm whose residual has x's type")
        y, h = _Apply.apply(x, weight, residual, self)
        return y if residual is None else (y, h)


class _Apply(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, residual, norm):
        y, h, rstd = norm.forward(x, weight, residual)
        ctx.norm, ctx.has_residual, ctx.weight_dtype = norm, residual is not None, None if weight is None else weight.dtype
        ctx.save_for_backward(h, rstd, weight)
        return y, h if residual is not None else None

    @staticmethod
    @once_differentiable      # (what the calls write has no graph: a derivative of it raises)
    def backward(ctx, dy, dres):
        h, rstd, weight = ctx.saved_tensors
        dy = dy if adjacent(dy) else dy.contiguous()      # (a sum's gradient is one element, seen as all of them)
        if dres is not None:
            dres = dres if adjacent(dres) else dres.contiguous()
        dh, dw = ctx.norm.backward(dy, h, rstd, weight, dres)
        return dh.to(dy.dtype), None if weight is None else dw.to(ctx.weight_dtype), dh if ctx.has_residual else None, None
