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
        each has to wait for the one before."""
        self.device = torch.device(device)
        torch.cuda.set_device(self.device)
        self.n, self.dtype, self.residual_dtype, self.weight_dtype = int(n), dtype, residual_dtype or dtype, weight_dtype
        self.ctx = None
        if dtype not in _OB_DTYPE or self.residual_dtype not in (dtype, torch.float32) or weight_dtype not in _OB_DTYPE:
            raise ValueError("types are torch.float32, torch.float16 and torch.bfloat16; the residual's is dtype or torch.float32")
        self._index, self._call = torch.cuda.current_device(), ob.lib().ob_norm_forward
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
        if t is not None and (t.dtype != self.weight_dtype or tuple(t.shape) != (self.n,) or not t.is_contiguous() or t.device != self.device):
            raise ValueError(f"weight: {self.n} adjacent {self.weight_dtype} on {self.device}")

    def _forward(self, x, weight, residual, h, y, want_y, format):
        # (a token's norm takes 3 us on the device: the common case is looked at as a whole, anything else piece by piece)
        n, rows = self.n, x.shape[0]
        dense, ldr, ldh, ldy = (rows, n), n, n, n
        whole = x.dtype is self.dtype and x.shape == dense and x.is_contiguous() and x.get_device() == self._index
        ldx = n if whole else rows_of(x, n, (self.dtype,), self.device, "x")
        if weight is not None and not (weight.dtype is self.weight_dtype and weight.shape == (n,) and weight.is_contiguous() and weight.get_device() == self._index):
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
        lddy, rows = rows_of(dy, self.n, (self.dtype,), self.device, "dy"), dy.shape[0]
        h, ldh = self._like(h, rows, self.residual_dtype, "h")
        self._weight(weight)
        if rstd.dtype != torch.float32 or tuple(rstd.shape) != (rows,) or not rstd.is_contiguous() or rstd.device != self.device:
            raise ValueError(f"rstd: {rows} adjacent torch.float32 on {self.device}")
        lddres = self.n
        if dres is not None:
            dres, lddres = self._like(dres, rows, self.residual_dtype, "dres")
        dh, lddh = self._like(out, rows, self.residual_dtype, "out")
        if dweight is None:
            if accumulate:
                raise ValueError("accumulate needs a dweight to add to")
            dweight = torch.empty(self.n, device=self.device, dtype=torch.float32)
        elif dweight.dtype != torch.float32 or tuple(dweight.shape) != (self.n,) or not dweight.is_contiguous() or dweight.device != self.device:
            raise ValueError(f"dweight: {self.n} adjacent torch.float32 on {self.device}")
        ob.ob_norm_backward(self.ctx, dy, lddy, h, ldh, rstd, weight, dres, lddres, rows, dh, lddh, dweight, accumulate, _current_stream(self.device))
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
