"""An expert layer trained with the matrix operators next to the LAMB steps: y = gain * (relu(x W1_g) W2_g) + bias.

The experts' matrices lie in one flat list of tensors that MuonStep steps on; its 16-bit copy of the parameters is what the
grouped products read, and their weight gradients go straight into the flat gradient that the step reads.  The vectors (gain
and bias) are a list of their own, under uncompressed LAMB steps (DeviceStep.warmup_step).

    python examples/expert_layer.py [--steps 30]
"""
import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2104_06069_amd.experts import ExpertLinear  # noqa: E402
from paper_2104_06069_amd.muon import MuonStep  # noqa: E402
from paper_2104_06069_amd.step import DeviceStep  # noqa: E402


class ExpertLayer:
    def __init__(self, groups, width, hidden, max_rows, seed=0):
        self.groups, self.width, self.hidden = groups, width, hidden
        one = width * hidden
        self.offsets = np.arange(2 * groups + 1, dtype=np.int64) * one        # W1 of each expert, then W2 of each
        rows = [width] * groups + [hidden] * groups
        gen = torch.Generator().manual_seed(seed)
        start = torch.cat([torch.randn(groups * one, generator=gen) * width ** -0.5, torch.randn(groups * one, generator=gen) * hidden ** -0.5])
        self.matrices = MuonStep(self.offsets, rows, momentum=0.9, weight_decay=0.01, x_lp_dtype=torch.bfloat16)
        self.matrices.load_state(dict(x=start))
        self.vectors = DeviceStep(np.array([0, width, 2 * width]), 1, 0, beta1=0.9, beta2=0.999, beta3=0.9, eta=1e-6, c_min=0.01, c_max=0.3,
                                  r_min=0.5, r_max=4.0, r_threshold=0.1, weight_decay=0.0)
        v = torch.zeros(self.vectors.n_pad)
        v[:width] = 1.0
        self.vectors.load_state(dict(x=v))
        self.grad = torch.zeros(2 * groups * one, device="cuda")
        self.grad_vectors = torch.zeros(self.vectors.n_pad, device="cuda")
        self.up = ExpertLinear(groups, width, hidden, max_rows=max_rows)
        self.down = ExpertLinear(groups, hidden, width, max_rows=max_rows)

    def _both(self, flat):
        half = flat.numel() // 2
        return flat[:half].view(self.up.w_shape), flat[half:].view(self.down.w_shape)

    def train(self, x, target, offsets, lr):
        """One step on rows that are sorted by expert; -> the mean squared error before it."""
        w1, w2 = self._both(self.matrices.x_lp)
        d1, d2 = self._both(self.grad)
        gain, bias = self.vectors.t["x"][:self.width], self.vectors.t["x"][self.width:2 * self.width]
        h = self.up.forward(x, w1, offsets)
        a = torch.relu(h)
        z = self.down.forward(a, w2, offsets, out_dtype=torch.float32)
        err = gain * z + bias - target
        dy = err * (2.0 / err.numel())
        self.grad_vectors[:self.width] = (dy * z).sum(0)
        self.grad_vectors[self.width:2 * self.width] = dy.sum(0)
        dz = (dy * gain).to(torch.bfloat16)
        da, _ = self.down.backward(a, dz, w2, offsets, dw=d2)
        self.up.weight_grad(x, da * (h > 0), offsets, out=d1)
        self.matrices.step(self.grad, lr)
        self.vectors.warmup_step(self.grad_vectors, 10 * lr)
        return err.square().mean()


def data(groups, width, hidden, rows, seed=1):
    """Rows that an uneven router dealt out, and what experts with other weights make of them."""
    rng, gen = np.random.default_rng(seed), torch.Generator(device="cuda").manual_seed(seed)
    p = np.exp(0.5 * rng.standard_normal(groups))
    counts = rng.multinomial(rows, p / p.sum())
    offsets = torch.tensor(np.concatenate([[0], np.cumsum(counts)]), dtype=torch.int32, device="cuda")
    normal = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    x = normal(rows, width).to(torch.bfloat16)
    up, down = ExpertLinear(groups, width, hidden, max_rows=rows), ExpertLinear(groups, hidden, width, max_rows=rows)
    w1, w2 = (normal(groups, a, b).mul_(a ** -0.5).to(torch.bfloat16) for a, b in ((width, hidden), (hidden, width)))
    return x, down.forward(torch.relu(up.forward(x, w1, offsets)), w2, offsets, out_dtype=torch.float32), offsets


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=30)
    ap.add_argument("--groups", type=int, default=8)
    ap.add_argument("--width", type=int, default=512)
    ap.add_argument("--hidden", type=int, default=2048)
    ap.add_argument("--rows", type=int, default=8192)
    a = ap.parse_args()
    x, target, offsets = data(a.groups, a.width, a.hidden, a.rows)
    layer = ExpertLayer(a.groups, a.width, a.hidden, a.rows)
    for t in range(a.steps):
        loss = layer.train(x, target, offsets, 2e-2 * (1 - t / a.steps))
        if t % 5 == 0 or t == a.steps - 1:
            print(f"step {t}: mean squared error {loss.item():.5f}", flush=True)


if __name__ == "__main__":
    main()
