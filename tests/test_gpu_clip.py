"""The gradient's norm and its clipping against the definition in 64 bits.

Bounds: squares are exact in binary64 and their sum of m is off by m 2^-53; the norm is rounded once, 2^-24.  The factor has two
roundings, the sum and the quotient, beside the norm's, and its product with the scale a fourth: 4 2^-24, and the result one of its own."""
import itertools

import numpy as np
import pytest

torch = pytest.importorskip("torch")
from tests.layer8 import HALF, LOWEST, within  # noqa: E402

pytestmark = pytest.mark.gpu
BF, F16, F32 = torch.bfloat16, torch.float16, torch.float32


def op(*args, **kw):
    from paper_2104_06069_amd.clip import GradClip
    return GradClip(*args, **kw)


def offsets_of(sizes):
    return np.concatenate([[0], np.cumsum(sizes)]).astype(np.int64)


LISTS = [[1], [7], [0, 5, 0, 0, 3], [1] * 300, [2048, 2049, 1, 0, 4095], [100_003, 17], [5_000, 300_000, 1, 70_000, 0], [2_000] * 1500, [9_000_001, 3, 500_000],
         [1] * 5000]


def gradient(n, dtype, sigma=1.0, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(n, generator=gen, device="cuda") * sigma).to(dtype)


def check(sizes, dtype, max_norm, out_dtype=None, grad_scale=1.0, sigma=1.0, extra=0):
    offsets = offsets_of(sizes)
    n = int(offsets[-1])
    g = gradient(n + extra, dtype, sigma)
    c = op(offsets, grad_scale=grad_scale)
    grad_scale = float(np.float32(grad_scale))      # (what the call is handed: 0.3 is no binary32 number)
    d = g[:n].double().cpu()
    squares = torch.stack([d[a:b].square().sum() for a, b in zip(offsets[:-1].tolist(), offsets[1:].tolist())])
    want = grad_scale * squares.sum().sqrt()
    most = want.item() + 1e-6
    f = grad_scale * min(1.0, max_norm / most)
    norm = c.norm(g)
    layers = c.layer_norms.clone()
    within(norm[0], want, 2.0 ** -24 * (1 + 1e-6) * want, "norm")
    within(layers, grad_scale * squares.sqrt(), 2.0 ** -24 * (1 + 1e-6) * grad_scale * squares.sqrt(), "norms of the tensors")
    before = g.clone()
    out = None if out_dtype is None else torch.full((n + 3,), 9.0, device="cuda", dtype=out_dtype)
    again = c.clip(g, max_norm, out)
    assert torch.equal(again, norm) and torch.equal(c.layer_norms, layers)
    got = g if out is None else out
    within(got[:n], d * f, (4 * 2.0 ** -24 + HALF[got.dtype]) * (d * f).abs() + LOWEST[got.dtype], "clipped")
    if out is None:
        assert torch.equal(g[n:], before[n:])
    else:
        assert torch.equal(g, before) and (out[n:] == 9).all()
    other = before.clone()
    alone = c.apply(other, norm, max_norm, None if out is None else torch.empty_like(out))
    assert torch.equal(alone[:n], got[:n])
    c.close()


@pytest.mark.parametrize("sizes", LISTS, ids=lambda s: f"{len(s)}_of_{max(s)}")
@pytest.mark.parametrize("dtype", (F32, F16, BF))
def test_in_place(sizes, dtype):
    check(sizes, dtype, 0.5)


@pytest.mark.parametrize("dtype,out_dtype", itertools.product((F32, F16, BF), (F32, F16, BF)))
def test_into_another_buffer(dtype, out_dtype):
    check([1000, 3, 70_001], dtype, 2.0, out_dtype)
    check([1000, 3, 70_001], dtype, 1e9, out_dtype)


@pytest.mark.parametrize("scale", (1 / 1024, 8.0, 0.3))
def test_loss_scale(scale):
    check([1000, 3, 3_000_001], F16, 0.25, F32, grad_scale=scale)
    check([1000, 3, 301], BF, 0.25, grad_scale=scale)


def test_buffers_longer_than_the_list():
    check([100, 50], F32, 0.1, extra=9)


@pytest.mark.parametrize("sizes", ([300, 5], [9_000_000, 5]))
def test_below_the_limit_nothing_changes(sizes):
    n = sum(sizes)
    g = gradient(n, F32)
    c = op(offsets_of(sizes))
    before = g.clone()
    for limit in (1e9, float("inf"), c.norm(g).item() + 1.0):
        c.clip(g, limit)
        assert torch.equal(g, before)


@pytest.mark.parametrize("sizes", ([300, 5], [9_000_000, 5]))
def test_hard_values(sizes):
    n = sum(sizes)
    c = op(offsets_of(sizes))
    z = torch.zeros(n, device="cuda")
    assert c.clip(z, 1.0).item() == 0 and (z == 0).all() and c.clip(z, 0.0).item() == 0 and (z == 0).all()
    big = torch.full((n,), 1e30, device="cuda")
    want = 1e30 * n ** 0.5
    assert abs(c.clip(big, 1.0).item() / want - 1) < 1e-6 and abs(big[7].item() * n ** 0.5 - 1) < 1e-6
    tiny = torch.full((n,), 1e-30, device="cuda")
    assert abs(c.norm(tiny).item() / (1e-30 * n ** 0.5) - 1) < 1e-6
    g = gradient(n, F32)
    g[n - 2] = float("inf")
    assert c.clip(g, 1.0).item() == float("inf") and (g[:n - 2] == 0).all() and g[n - 2].isnan() and (c.layer_norms[0].isfinite() and c.layer_norms[1].isinf())
    g = gradient(n, F32)
    g[1] = float("nan")
    assert c.clip(g, 1.0).isnan().item() and g.isnan().all()
    g = gradient(n, F32)
    c.clip(g, 0.0)
    assert (g == 0).all()


def test_empty_list():
    c = op([0, 0])
    g = torch.empty(0, device="cuda")
    assert c.clip(g, 1.0).item() == 0 and c.layer_norms.item() == 0 and c.norm(g).item() == 0


def test_norm_from_elsewhere():
    """Two ranks' parts of a gradient, one after the other on one device."""
    a, b = op([0, 1000]), op([0, 500])
    g, h = gradient(1000, F32), gradient(500, F32, seed=1)
    whole = (a.norm(g).square() + b.norm(h).square()).sqrt()
    gd, hd = g.double().cpu(), h.double().cpu()
    f = 0.5 / ((gd.square().sum() + hd.square().sum()).sqrt() + 1e-6)
    a.apply(g, whole, 0.5)
    b.apply(h, whole, 0.5)
    for got, d in ((g, gd), (h, hd)):      # (four more roundings in the norm of both)
        within(got, d * f, 9 * 2.0 ** -24 * (d * f).abs(), "clipped")


@pytest.mark.parametrize("sizes", ([300, 5, 1000], [9_000_000, 5, 100_000]))
def test_another_stream_and_a_graph(sizes):
    n = sum(sizes)
    c = op(offsets_of(sizes))
    g = gradient(n, F32)
    want = g.clone()
    norm = c.clip(want, 0.5)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = g.clone()
        norm2 = c.clip(got, 0.5)
    s.synchronize()
    assert torch.equal(got, want) and torch.equal(norm, norm2)
    src, buf = g.clone(), torch.empty_like(g)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        buf.copy_(src)
        norm3 = c.clip(buf, 0.5)
        norm4 = c.norm(buf)
    for k in range(4):
        src.copy_(gradient(n, F32, sigma=10.0 ** (k - 2), seed=k))
        graph.replay()
        want = src.clone()
        norm = c.clip(want, 0.5)
        after = c.norm(want)
        torch.cuda.synchronize()
        assert torch.equal(buf, want) and torch.equal(norm3, norm) and torch.equal(norm4, after)


def test_long_lists():
    """Elements beyond 2^32 of one buffer: whole numbers, so that the sums are exact."""
    n = (1 << 32) + 70_001
    g = torch.zeros(n, device="cuda", dtype=BF)
    g[-70_000:] = 2.0
    g[5] = 3.0
    c = op([0, 1000, 1 << 32, n])
    norm = c.clip(g, 1.0)
    assert norm.item() == np.float32(np.sqrt(280_009.0)) and c.layer_norms.tolist() == [3.0, 0.0, np.float32(np.sqrt(280_000.0)).item()]
    f = np.float32(1.0) / (np.float32(np.sqrt(280_009.0)) + np.float32(1e-6))
    assert (g[-70_000:] == torch.tensor(np.float32(2.0) * f).to(BF).item()).all() and g[5].item() == torch.tensor(np.float32(3.0) * f).to(BF).item()
    assert (g[6:1 << 20] == 0).all()


def test_refusals():
    c = op([0, 10, 30])
    g = torch.zeros(30, device="cuda")
    for call in (lambda: c.norm(g[:29]), lambda: c.norm(g.cpu()), lambda: c.norm(g.double()), lambda: c.norm(torch.zeros(60, device="cuda")[::2]),
                 lambda: c.clip(g, 1.0, out=g[:29]), lambda: c.apply(g, torch.zeros(2, device="cuda"), 1.0), lambda: c.apply(g, torch.zeros(1), 1.0)):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: c.clip(g, -1.0), lambda: c.clip(g, float("nan")), lambda: op([0, 5, 3]), lambda: op([1, 5]), lambda: op([0, 5], eps=-1.0),
                 lambda: op([0, 5], grad_scale=0.0), lambda: op([0, 5], grad_scale=float("inf"))):
        with pytest.raises(RuntimeError):
            call()
