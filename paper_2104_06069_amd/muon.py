"""Device-side plumbing of the orthogonalised update (include/ob_matrix.h): the flat buffers and the calls, as DeviceStep is
for the LAMB steps.  It steps the matrices of a flat list of tensors; the others (vectors, embeddings) are left to another
optimizer on the same buffers.

    opt = MuonStep(layer_offsets, layer_rows, momentum=0.95, weight_decay=0.01)      # layer_rows[l] = 0: not a matrix
    opt.load_state(dict(x=params_flat))
    opt.step(grad_flat, lr)

The momentum may come from the 1-bit compressed exchange instead: after DeviceStep.compress_local / server_reduce have left
the global momentum in its 1-bit form, ob_lamb_momentum_dense writes it to opt.t["m"], and opt.step(None, lr) takes it as it is.
"""
import torch

from . import binding as ob
from .step import _OB_DTYPE, _current_stream


class MuonStep:
    def __init__(self, layer_offsets, layer_rows, device="cuda:0", momentum=0.95, nesterov=True, weight_decay=0.0, steps=5,
                 coefficients=(3.4445, -4.7750, 2.0315), eps=1e-7, layer_scale=None, precision=torch.float32, grad_scale=1.0,
                 x_lp_dtype=None, own_state=True):
        """precision: torch.float32 (numbers of 22 bits, 1e-6 to 3e-6 of relative error over a matrix of normal numbers), or torch.float16
        (11 bits where that saves time, 0.6 to 1 of it; 1e-3 to 2e-3).  Calls on one object share its workspace and must not overlap in
        time: on several streams, each has to wait for the one before.  layer_scale: factor of each tensor's direction (default 0.2 sqrt(max(rows, columns))).  grad_scale: the inverse
        loss scale.  own_state: allocate x and m; a program that has them puts its own flat float32 tensors into self.t."""
        self.device = torch.device(device)
        torch.cuda.set_device(self.device)
        self.N, self.grad_scale = int(layer_offsets[-1]), float(grad_scale)
        self.ctx = None
        self.ctx = ob.ob_muon_create(layer_offsets, layer_rows, layer_scale, coefficients, steps, eps, momentum, weight_decay,
                                     nesterov, _OB_DTYPE[precision])
        self.t = {k: torch.zeros(self.N, device=self.device) if own_state else None for k in ("x", "m")}
        self.x_lp = None if x_lp_dtype is None else torch.zeros(self.N, device=self.device, dtype=x_lp_dtype)

    def close(self):
        if self.ctx is not None:
            torch.cuda.synchronize(self.device)
            ob.ob_muon_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def load_state(self, st):
        """st: dict with x and / or m, as tensors or arrays; the 16-bit copy follows x."""
        for k in ("x", "m"):
            if st.get(k) is not None:
                self.t[k].copy_(torch.as_tensor(st[k]))
        if self.x_lp is not None and st.get("x") is not None:
            self.x_lp.copy_(self.t["x"])

    def _flat(self, t, dtypes, what):
        if t is None or t.dtype not in dtypes or t.device != self.device or t.numel() < self.N or not t.is_contiguous():
            raise ValueError(f"{what}: at least {self.N} adjacent elements of {' or '.join(map(str, dtypes))} on {self.device}")
        return t

    def orthogonalize(self, src, out=None, out_dtype=None):
        """out: the matrices of `src` with their singular values taken towards 1; the tensors left out are not written (zeros in
        an `out` made here)."""
        self._flat(src, tuple(_OB_DTYPE), "src")
        if out is None:
            out = torch.zeros(self.N, device=self.device, dtype=out_dtype or src.dtype)
        self._flat(out, tuple(_OB_DTYPE), "out")
        ob.ob_muon_orthogonalize(self.ctx, src, _OB_DTYPE[src.dtype], out, _OB_DTYPE[out.dtype], _current_stream(self.device))
        return out

    def step(self, grad, lr):
        """One step in place on t["x"] and t["m"] (and x_lp).  grad None: t["m"] is the direction, formed elsewhere."""
        x, m = (self._flat(self.t[k], (torch.float32,), k) for k in ("x", "m"))
        if grad is not None:
            self._flat(grad, tuple(_OB_DTYPE), "grad")
        ob.ob_muon_step(self.ctx, x, m, grad, ob.OB_F32 if grad is None else _OB_DTYPE[grad.dtype], self.grad_scale, lr,
                        self.x_lp, ob.OB_F32 if self.x_lp is None else _OB_DTYPE[self.x_lp.dtype], _current_stream(self.device))
