"""The operators run together, as examples/expert_layer.py does."""
import os
import sys

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def test_the_layer_learns():
    from expert_layer import ExpertLayer, data
    x, target, offsets = data(4, 128, 256, 1500)
    layer = ExpertLayer(4, 128, 256, 1500)
    loss = [layer.train(x, target, offsets, 2e-2 * (1 - t / 40)).item() for t in range(40)]
    assert loss[-1] < 0.35 * loss[0], loss


def test_gradients_of_the_layer():
    """What goes into the flat gradients against torch's autograd in 64 bits on the same 16-bit weights.  The products' 16-bit
    results (h, dz, da) are each rounded to 2^-8: in the 2-norm a few times 2^-9."""
    from expert_layer import ExpertLayer, data
    groups, width, hidden = 3, 96, 160
    x, target, offsets = data(groups, width, hidden, 400)
    layer = ExpertLayer(groups, width, hidden, 400)
    w1, w2 = (w.double().clone().requires_grad_() for w in layer._both(layer.matrices.x_lp))
    v = layer.vectors.t["x"][:2 * width].double().clone().requires_grad_()
    layer.train(x, target, offsets, 0.0)
    ends = offsets.tolist()
    y = torch.cat([torch.relu(x[a:b].double() @ w1[g]) @ w2[g] for g, (a, b) in enumerate(zip(ends[:-1], ends[1:]))])
    (v[:width] * y + v[width:] - target.double()).square().mean().backward()
    for got, want in zip(layer._both(layer.grad), (w1.grad, w2.grad)):
        assert (got.double() - want).norm() <= 2e-2 * want.norm()
    assert (layer.grad_vectors[:2 * width].double() - v.grad).norm() <= 2e-2 * v.grad.norm()


def test_the_example_runs():
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, os.path.join(root, "examples", "expert_layer.py"), "--steps", "6", "--width", "128", "--hidden", "256",
                        "--rows", "1000"], capture_output=True, text=True, timeout=100)
    assert r.returncode == 0 and r.stdout.count("mean squared error") == 2, (r.stdout, r.stderr[-2000:])
