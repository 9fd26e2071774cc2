"""The norm of a flat gradient and its clipping on the device (include/ob_layer.h), on the lists of tensors that DeviceStep and MuonStep
step on:

    clip = GradClip(layer_offsets)
    norm = clip.clip(grad_flat, 1.0)       # grad_flat scaled to a norm of at most 1, before the step; norm: what it was
    clip.layer_norms                       # of each tensor, as the last call found them

Over several ranks that hold parts of a gradient, norm() and apply() with what the program makes of the ranks' norms in between.  The host
reads nothing.
"""
import torch

from . import binding as ob
from .step import _OB_DTYPE, _current_stream

_TYPES = tuple(_OB_DTYPE)


class GradClip:
    def __init__(self, layer_offsets, eps=1e-6, grad_scale=1.0, device="cuda:0"):
        """eps is added to the norm that max_norm is divided by.  grad_scale: the inverse loss scale; norms are those of the scaled gradient, and
        apply() and clip() multiply by it too.  Calls on one object share its workspace and layer_norms and must not overlap in time: on
        several streams, each has to wait for the one before."""
        self.device = torch.device(device)
        torch.cuda.set_device(self.device)
        self.ctx = None
        self.N = int(layer_offsets[-1])
        self.ctx = ob.ob_clip_create(layer_offsets, eps, grad_scale)
        self.layer_norms = torch.zeros(len(layer_offsets) - 1, device=self.device)
        self._call, self._layer_norms = ob.lib().ob_clip_norm_apply, self.layer_norms.data_ptr()

    def close(self):
        if self.ctx is not None:
            torch.cuda.synchronize(self.device)
            ob.ob_clip_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _flat(self, t, what):
        if t.dtype not in _OB_DTYPE or t.device != self.device or t.numel() < self.N or not t.is_contiguous():
            raise ValueError(f"{what}: at least {self.N} adjacent elements of {' or '.join(map(str, _TYPES))} on {self.device}")
        return t

    def _one(self):
        return torch.empty(1, device=self.device)

    def norm(self, grad):
        """-> norm [1] of the scaled gradient; layer_norms follow."""
        self._flat(grad, "grad")
        norm = self._one()
        ob.ob_clip_norm(self.ctx, grad, _OB_DTYPE[grad.dtype], norm, self.layer_norms, _current_stream(self.device))
        return norm

    def apply(self, grad, norm, max_norm, out=None):
        """out (default: grad, in place) = grad grad_scale min(1, max_norm / (norm + eps)), norm [1] float32 on the device."""
        out = self._flat(grad, "grad") if out is None else self._flat(out, "out")
        if norm.dtype != torch.float32 or norm.numel() != 1 or norm.device != self.device:
            raise ValueError(f"norm: one torch.float32 on {self.device}")
        ob.ob_clip_apply(self.ctx, self._flat(grad, "grad"), _OB_DTYPE[grad.dtype], norm, max_norm, out, _OB_DTYPE[out.dtype], _current_stream(self.device))
        return out

    def clip(self, grad, max_norm, out=None):
        """norm() and apply() in one call; -> the norm [1] before."""
        self._flat(grad, "grad")
        out = grad if out is None else self._flat(out, "out")
        norm = self._one()
        status = self._call(self.ctx, grad.data_ptr(), _OB_DTYPE[grad.dtype], max_norm, norm.data_ptr(), self._layer_norms, out.data_ptr(), _OB_DTYPE[out.dtype],
                            _current_stream(self.device))
        if status:
            raise ob.ObLambError(status, "ob_clip_norm_apply", ob.lib().ob_clip_last_hip_error(self.ctx).decode())
        return norm
