"""The operators run together: the norm's 8 bits into the product, gradients into the flat gradient, clipped, stepped on."""
import os
import subprocess
import sys

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))
BF = torch.bfloat16


@pytest.mark.parametrize("rows,width", [(1, 64), (5, 300), (200, 1000), (3, 2048), (40, 5000)])
def test_the_norm_writes_what_the_quantiser_would(rows, width):
    """With binary32 rows, so that y is what its 8 bits are made of."""
    from paper_2104_06069_amd.linear8 import Linear8
    from paper_2104_06069_amd.norm import RMSNorm
    gen = torch.Generator().manual_seed(0)
    x, r = (torch.randn(rows, width, generator=gen).cuda() for _ in range(2))
    w, matrix = (1 + 0.2 * torch.randn(width, generator=gen)).cuda(), torch.randn(96, width, generator=gen).cuda()
    norm, layer = RMSNorm(width, dtype=torch.float32), Linear8(width, 96)
    for fmt in (torch.float8_e4m3fn, torch.float8_e5m2):
        y = torch.empty_like(x)
        m, _, _ = norm.forward8(x, w, r, out=y, format=fmt)
        q = layer.quantize(y, fmt)
        assert torch.equal(m.data.view(torch.uint8), q.data.view(torch.uint8)) and torch.equal(m.scales.view(torch.uint8), q.scales.view(torch.uint8))
        w8 = layer.quantize_weight(matrix)
        assert torch.equal(layer.forward(m, w8), layer.forward(q, w8))


def test_gradients_of_the_layer():
    """Against autograd in 64 bits.  A number's rounding to 8 bits is off by up to 2^-4, 0.036 in the mean of squares; up to six operands
    between the loss and a gradient are rounded: 0.09; and the 4 % of z that lie within their error of zero may take the other side of the relu, half
    of them: 0.14.  In quadrature 0.17."""
    from layer8 import Layer8, data
    width, hidden, rows = 160, 300, 700
    layer = Layer8(width, hidden)
    x, residual, target = data(width, hidden, rows)
    w1, w2 = (w.double().clone().requires_grad_() for w in layer._both(layer.matrices.x_lp))
    gain = layer.gain.double().clone().requires_grad_()
    loss = layer.gradients(x, residual, target)
    h = (x.float() + residual.float()).to(BF).double()
    n = h / (h.square().mean(1, keepdim=True) + 1e-6).sqrt() * gain
    want = (h + torch.relu(n @ w1.T) @ w2.T - target.double()).square().mean()
    want.backward()
    assert abs(loss.item() / want.item() - 1) < 0.17
    d1, d2 = layer._both(layer.grad)
    for got, ref in ((d1, w1.grad), (d2, w2.grad), (layer.grad_vector[:width], gain.grad)):
        assert (got.double() - ref).norm() <= 0.17 * ref.norm()


def test_the_gradient_is_clipped_before_the_step():
    from layer8 import Layer8, data
    layer = Layer8(128, 256, max_norm=1e-3)
    batch = data(128, 256, 500)
    layer.gradients(*batch)
    whole = torch.cat([layer.grad, layer.grad_vector]).double().norm().item()
    first, vector = layer.grad.clone(), layer.grad_vector.clone()
    assert whole > 2e-3
    layer.train(*batch, 0.0)
    f = 1e-3 / (whole + 1e-6)
    for got, before in ((layer.grad, first), (layer.grad_vector, vector)):
        assert ((got.double() - before.double() * f).abs() <= 2.0 ** -20 * (before.double() * f).abs()).all()
    assert layer.train(*batch, 1e-2).isfinite()


def test_a_layer_of_autograd_calls():
    """norm, product and product again under torch's autograd, against the same calls made one by one."""
    from paper_2104_06069_amd.linear8 import Linear8
    from paper_2104_06069_amd.norm import RMSNorm
    gen = torch.Generator().manual_seed(0)
    rows, width, hidden = 60, 200, 136
    x, r = (torch.randn(rows, width, generator=gen).to(BF).cuda() for _ in range(2))
    g = torch.ones(width, device="cuda")
    w1, w2 = torch.randn(hidden, width, generator=gen).cuda(), torch.randn(width, hidden, generator=gen).cuda()
    norm, up, down = RMSNorm(width), Linear8(width, hidden), Linear8(hidden, width)
    leaves = [t.clone().requires_grad_() for t in (x, r, g, w1, w2)]
    n, h = norm(leaves[0], leaves[2], leaves[1])
    out = down(torch.relu(up(n, leaves[3])), leaves[4]) + h
    c = torch.randn(rows, width, generator=gen).to(BF).cuda()
    out.backward(c)
    n, h, rstd = norm.forward(x, g, r)
    q1, q2 = up.quantize_weight(w1), down.quantize_weight(w2)
    z = up.forward(n, q1)
    a = torch.relu(z)
    assert torch.equal(out, down.forward(a, q2) + h)
    da, d2 = down.backward(a, c, q2)
    dn, d1 = up.backward(n, da * (z > 0), q1)
    dh, dg = norm.backward(dn, h, rstd, g, c)
    for leaf, want in zip(leaves, (dh, dh, dg, d1, d2)):
        assert torch.equal(leaf.grad, want)


def test_the_example_runs():
    r = subprocess.run([sys.executable, os.path.join(ROOT, "examples", "layer8.py"), "--steps", "6", "--width", "128", "--hidden", "256", "--rows", "1000"],
                       capture_output=True, text=True, timeout=100)
    assert r.returncode == 0 and r.stdout.count("mean squared error") == 2, (r.stdout, r.stderr[-2000:])
