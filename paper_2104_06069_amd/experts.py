"""The products of an expert layer on the device (include/ob_matrix.h): argument checks and output buffers around the calls.

Rows are sorted by expert; `offsets` (int32, on the device, num_groups + 1 entries) says where each expert's begin, and the
host does not read it.  Weights may be a view of the flat 16-bit parameters that DeviceStep or MuonStep keeps (its x_lp), and
weight gradients can go straight into a view of the flat gradient that those read:

    layer = ExpertLinear(groups, k, n, dtype=torch.bfloat16, max_rows=rows)
    y = layer.forward(x, w, offsets)
    dx, dw = layer.backward(x, dy, w, offsets, dw=flat_grad[a:b].view(groups, k, n))

or, with torch's autograd, y = layer(x, w, offsets), where rows that belong to no expert are zeros and get none of a gradient.
"""
import torch
from torch.autograd.function import once_differentiable

from . import binding as ob
from .step import _OB_DTYPE, _current_stream

_LAYOUTS = {"kn": ob.OB_EXPERTS_KN, "nk": ob.OB_EXPERTS_NK}


def _adjacent(t):
    """Whether each row's elements follow each other and no row overlaps the next.  Of a single row only the distance to the next one
    is free."""
    rows, width = t.shape
    return rows == 0 or ((width < 2 or t.stride(1) == 1) and (rows < 2 or t.stride(0) >= width))


class ExpertLinear:
    def __init__(self, num_groups, k, n, dtype=torch.bfloat16, max_rows=1 << 20, layout="kn", w_stride=0, device="cuda:0"):
        """layout: "kn", W is [num_groups, k, n], or "nk", [num_groups, n, k].  w_stride: elements from one expert's weights
        to the next one's (0: they follow each other).  Weight gradients share the object's workspace: calls on one object, those of
        autograd among them, must not overlap in time; on several streams, each has to wait for the one before."""
        self.device = torch.device(device)
        torch.cuda.set_device(self.device)
        self.groups, self.k, self.n, self.dtype, self.layout = int(num_groups), int(k), int(n), dtype, layout
        if layout not in _LAYOUTS or dtype not in (torch.float16, torch.bfloat16):
            raise ValueError("layout is 'kn' or 'nk', dtype torch.float16 or torch.bfloat16")
        self.w_shape = (self.groups, self.k, self.n) if layout == "kn" else (self.groups, self.n, self.k)
        self.w_stride = int(w_stride) or self.k * self.n
        self._w_dense, self._offsets_shape = (self.w_stride, self.w_shape[2], 1), (self.groups + 1,)
        self._index = torch.cuda.current_device()
        self._forward, self._input_grad = ob.lib().ob_experts_forward, ob.lib().ob_experts_input_grad
        self.ctx = ob.ob_experts_create(self.groups, self.k, self.n, _OB_DTYPE[dtype], _LAYOUTS[layout], max_rows, w_stride)

    def close(self):
        if self.ctx is not None:
            torch.cuda.synchronize(self.device)
            ob.ob_experts_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _rows(self, t, width, dtypes, what):
        if t.dim() != 2 or t.shape[1] != width or t.dtype not in dtypes or t.device != self.device:
            raise ValueError(f"{what}: a [rows, {width}] tensor of {' or '.join(map(str, dtypes))} on {self.device}, not "
                             f"{tuple(t.shape)} of {t.dtype} on {t.device}")
        if not _adjacent(t):
            raise ValueError(f"{what}: rows of adjacent elements that do not overlap")
        return t.stride(0) if t.shape[0] > 1 else width

    def _weights(self, t, dtypes, what):
        inner = self.w_shape[2]
        if tuple(t.shape) != self.w_shape or t.dtype not in dtypes or t.device != self.device:
            raise ValueError(f"{what}: a {self.w_shape} tensor of {' or '.join(map(str, dtypes))} on {self.device}")
        for size, stride, want in zip(t.shape, t.stride(), (self.w_stride, inner, 1)):
            if size > 1 and stride != want:
                raise ValueError(f"{what}: strides ({self.w_stride}, {inner}, 1), not {t.stride()}")

    def _offsets(self, t):
        if t.dtype != torch.int32 or t.dim() != 1 or t.numel() != self.groups + 1 or not t.is_contiguous() or t.device != self.device:
            raise ValueError(f"offsets: {self.groups + 1} adjacent int32 on {self.device}")

    def _product(self, call, where, a, depth, width, w, offsets, out, out_dtype, names):
        # (a token's product takes 5 us on the device: the common case is looked at as a whole, anything else piece by piece)
        rows, lda = a.shape[0], depth
        if not (a.dtype is self.dtype and w.dtype is self.dtype and offsets.dtype is torch.int32 and a.shape == (rows, depth)
                and a.stride() == (depth, 1) and w.shape == self.w_shape and w.stride() == self._w_dense and offsets.shape == self._offsets_shape
                and offsets.is_contiguous() and a.get_device() == w.get_device() == offsets.get_device() == self._index):
            lda = self._rows(a, depth, (self.dtype,), names[0])
            self._weights(w, (self.dtype,), "w")
            self._offsets(offsets)
        if out is None:
            out = torch.empty((rows, width), device=self.device, dtype=out_dtype or self.dtype)
            ldo = width
        else:
            ldo = self._rows(out, width, (self.dtype, torch.float32), names[1])
            if out.shape[0] != rows:
                raise ValueError(f"{names[1]}: {rows} rows")
        status = call(self.ctx, a.data_ptr(), lda, w.data_ptr(), offsets.data_ptr(), rows, out.data_ptr(), ldo, _OB_DTYPE[out.dtype],
                      _current_stream(self.device))
        if status:
            raise ob.ObLambError(status, where, ob.lib().ob_experts_last_hip_error(self.ctx).decode())
        return out

    def forward(self, x, w, offsets, out=None, out_dtype=None):
        """y[r] = x[r] W_g.  Rows that belong to no expert are not written."""
        return self._product(self._forward, "ob_experts_forward", x, self.k, self.n, w, offsets, out, out_dtype, ("x", "out"))

    def input_grad(self, dy, w, offsets, out=None, out_dtype=None):
        """dx[r] = dy[r] W_g^T.  Rows that belong to no expert are not written."""
        return self._product(self._input_grad, "ob_experts_input_grad", dy, self.n, self.k, w, offsets, out, out_dtype, ("dy", "out"))

    def weight_grad(self, x, dy, offsets, out=None, out_dtype=None, accumulate=False):
        """dW_g = x_g^T dy_g, or with accumulate (a float32 `out`) dW_g += x_g^T dy_g."""
        ldx, lddy = self._rows(x, self.k, (self.dtype,), "x"), self._rows(dy, self.n, (self.dtype,), "dy")
        self._offsets(offsets)
        if x.shape[0] != dy.shape[0]:
            raise ValueError("x and dy: one row each")
        if out is None:
            if accumulate:
                raise ValueError("accumulate needs an out to add to")
            out = torch.empty_strided(self.w_shape, self._w_dense, device=self.device, dtype=out_dtype or self.dtype)      # (gaps as between W's)
        self._weights(out, (torch.float32,) if accumulate else (self.dtype, torch.float32), "out")
        ob.ob_experts_weight_grad(self.ctx, x, ldx, dy, lddy, offsets, x.shape[0], out, _OB_DTYPE[out.dtype], accumulate,
                                  _current_stream(self.device))
        return out

    def backward(self, x, dy, w, offsets, dw=None, dw_dtype=None):
        """-> (dx, dW).  Rows of dx that belong to no expert are not written."""
        return self.input_grad(dy, w, offsets), self.weight_grad(x, dy, offsets, out=dw, out_dtype=dw_dtype)

    def __call__(self, x, w, offsets):
        return _Apply.apply(x, w, offsets, self)


class _Apply(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w, offsets, layer):
        ctx.save_for_backward(x, w, offsets)
        ctx.layer = layer
        # (rows of no expert are not written: they are zeros, and so are their gradients)
        return layer.forward(x, w, offsets, out=x.new_zeros(x.shape[0], layer.n))

    @staticmethod
    @once_differentiable      # (what the calls write has no graph: a derivative of it raises)
    def backward(ctx, dy):
        x, w, offsets = ctx.saved_tensors
        dy = dy if _adjacent(dy) else dy.contiguous()      # (a sum's gradient is one element, seen as all of them)
        dx = ctx.layer.input_grad(dy, w, offsets, out=torch.zeros_like(x, memory_format=torch.contiguous_format)) if ctx.needs_input_grad[0] else None
        dw = ctx.layer.weight_grad(x, dy, offsets) if ctx.needs_input_grad[1] else None
        return dx, dw, None, None
