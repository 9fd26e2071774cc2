"""A layer of a residual stream trained in 8 bits with the operators next to the optimizer steps: out = h + relu(n W1^T) W2^T, n = rmsnorm(h) gain,
h = x + residual.

The norm writes the 8-bit rows that the first product reads, the weight gradients go straight into the flat gradient that
MuonStep reads, and the gradient is clipped by its norm over both lists of tensors, the matrices and the vector (the gain, under
uncompressed LAMB steps), before either is stepped on.

    python examples/layer8.py [--steps 30]
"""
import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2104_06069_amd.clip import GradClip  # noqa: E402
from paper_2104_06069_amd.linear8 import Linear8  # noqa: E402
from paper_2104_06069_amd.muon import MuonStep  # noqa: E402
from paper_2104_06069_amd.norm import RMSNorm  # noqa: E402
from paper_2104_06069_amd.step import DeviceStep  # noqa: E402


class Layer8:
    def __init__(self, width, hidden, seed=0, max_norm=1.0):
        self.width, self.hidden, self.max_norm = width, hidden, max_norm
        one = width * hidden
        offsets = np.array([0, one, 2 * one], dtype=np.int64)      # W1 [hidden, width], W2 [width, hidden]
        gen = torch.Generator().manual_seed(seed)
        start = torch.cat([torch.randn(one, generator=gen) * width ** -0.5, torch.randn(one, generator=gen) * hidden ** -0.5])
        self.matrices = MuonStep(offsets, [hidden, width], momentum=0.9, weight_decay=0.01, x_lp_dtype=torch.bfloat16)
        self.matrices.load_state(dict(x=start))
        self.vector = DeviceStep(np.array([0, width]), 1, 0, beta1=0.9, beta2=0.999, beta3=0.9, eta=1e-6, c_min=0.01, c_max=0.3, r_min=0.5, r_max=4.0,
                                 r_threshold=0.1, weight_decay=0.0)
        gain = torch.zeros(self.vector.n_pad)
        gain[:width] = 1.0
        self.vector.load_state(dict(x=gain))
        self.grad = torch.zeros(2 * one, device="cuda")
        self.grad_vector = torch.zeros(self.vector.n_pad, device="cuda")
        self.norm = RMSNorm(width)
        self.up, self.down = Linear8(width, hidden), Linear8(hidden, width)
        self.clips = GradClip(offsets), GradClip([0, width])

    def _both(self, flat):
        half = flat.numel() // 2
        return flat[:half].view(self.hidden, self.width), flat[half:].view(self.width, self.hidden)

    @property
    def gain(self):
        return self.vector.t["x"][:self.width]

    def gradients(self, x, residual, target):
        """Fills the flat gradients; -> the mean squared error"""
        w1, w2 = (op.quantize_weight(w) for op, w in zip((self.up, self.down), self._both(self.matrices.x_lp)))
        d1, d2 = self._both(self.grad)
        n = torch.empty_like(x)
        n8, h, rstd = self.norm.forward8(x, self.gain, residual, out=n)
        z = self.up.forward(n8, w1)
        a = torch.relu(z)
        err = h.float() + self.down.forward(a, w2, out_dtype=torch.float32) - target
        dout = (err * (2.0 / err.numel())).to(torch.bfloat16)
        da, _ = self.down.backward(a, dout, w2, dw=d2)
        dn, _ = self.up.backward(n, da * (z > 0), w1, dw=d1)
        self.norm.backward(dn, h, rstd, self.gain, dout, dweight=self.grad_vector[:self.width])
        return err.square().mean()

    def train(self, x, residual, target, lr):
        loss = self.gradients(x, residual, target)
        norm = (self.clips[0].norm(self.grad).square() + self.clips[1].norm(self.grad_vector).square()).sqrt()
        self.clips[0].apply(self.grad, norm, self.max_norm)
        self.clips[1].apply(self.grad_vector, norm, self.max_norm)
        self.matrices.step(self.grad, lr)
        self.vector.warmup_step(self.grad_vector, 10 * lr)
        return loss


def data(width, hidden, rows, seed=1):
    """Rows, their residual, and what a layer with other weights makes of them."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    x, residual = normal(rows, width).to(torch.bfloat16), normal(rows, width).to(torch.bfloat16)
    w1, w2 = normal(hidden, width) * width ** -0.5, normal(width, hidden) * hidden ** -0.5
    h = x.float() + residual.float()
    n = h * torch.rsqrt(h.square().mean(1, keepdim=True) + 1e-6)
    return x, residual, h + torch.relu(n @ w1.t()) @ w2.t()


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=30)
    ap.add_argument("--width", type=int, default=512)
    ap.add_argument("--hidden", type=int, default=2048)
    ap.add_argument("--rows", type=int, default=8192)
    a = ap.parse_args()
    batch = data(a.width, a.hidden, a.rows)
    layer = Layer8(a.width, a.hidden)
    for t in range(a.steps):
        loss = layer.train(*batch, 2e-2 * (1 - t / a.steps))
        if t % 5 == 0 or t == a.steps - 1:
            print(f"step {t}: mean squared error {loss.item():.5f}", flush=True)


if __name__ == "__main__":
    main()
