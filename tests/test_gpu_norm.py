"""The root-mean-square norm against the definition in 64 bits, element by element.

Bounds: a sum of squares is off by 2^-24 of it for each of its additions that a number goes through (up to 32 in a lane, then up to 9
between lanes and wavefronts) and for its square, rstd by half of that and its own four roundings, and two products follow: 30 2^-24
in all, taken as 2^-19; then the result's rounding.  In the backward pass the mean is off by as much of the mean of magnitudes."""
import itertools

import pytest

torch = pytest.importorskip("torch")
from tests.layer8 import E4M3, E5M2, HALF, LOWEST, blocks_of, padding_is_zero, scales_of, spread, values, within  # noqa: E402

pytestmark = pytest.mark.gpu
BF, F16, F32 = torch.bfloat16, torch.float16, torch.float32
TYPES = [(BF, BF), (F16, F16), (F32, F32), (BF, F32), (F16, F32)]


def op(*args, **kw):
    from paper_2104_06069_amd.norm import RMSNorm
    return RMSNorm(*args, **kw)


def normal(*shape, seed=0, dtype=F32, pitch=0, sigma=1.0):
    """pitch: elements between rows beyond their width"""
    gen = torch.Generator().manual_seed(seed)
    t = (torch.randn(shape[0], shape[1] + pitch, generator=gen) * sigma).to(dtype).cuda()
    return t[:, :shape[1]] if pitch else t


def want_forward(h, weight, eps):
    h = h.double().cpu()
    rstd = 1.0 / (h.square().mean(1, keepdim=True) + eps).sqrt()
    return h * rstd * (1.0 if weight is None else weight.double().cpu()), rstd


def check_forward(rows, n, x_type, h_type, residual=True, weight=True, pitch=0, eps=1e-6, weight_dtype=F32, seed=0):
    x, r = normal(rows, n, seed=seed, dtype=x_type, pitch=pitch), normal(rows, n, seed=seed + 1, dtype=h_type, pitch=2 * pitch) if residual else None
    w = (1.0 + normal(1, n, seed=seed + 2, sigma=0.2)[0]).to(weight_dtype) if weight else None
    norm = op(n, dtype=x_type, residual_dtype=h_type, eps=eps, weight_dtype=weight_dtype)
    y, h, rstd = norm.forward(x, w, r)
    if residual:
        assert torch.equal(h, (x.float() + r.float()).to(h_type))
    else:
        assert h is x
    want, want_rstd = want_forward(h, w, eps)
    within(rstd, want_rstd[:, 0], 2.0 ** -20 * want_rstd[:, 0], "rstd")
    within(y, want, (2.0 ** -19 + HALF[x_type]) * want.abs() + LOWEST[x_type], "y")
    for fmt, half, lowest in ((E4M3, 2.0 ** -4, 2.0 ** -10), (E5M2, 2.0 ** -3, 2.0 ** -17)):
        out = torch.empty_like(y)
        y8, h8, rstd8 = norm.forward8(x, w, r, out=out, format=fmt)
        assert torch.equal(h8, h) and torch.equal(rstd8, rstd) and torch.equal(out, y) and padding_is_zero(y8)
        most = blocks_of(want)
        lo, hi = scales_of(most * (1 - 2.0 ** -18), fmt), scales_of(most * (1 + 2.0 ** -18), fmt)
        got = y8.scales.cpu().double()
        assert ((got == lo) | (got == hi)).all()
        within(values(y8), want, (2.0 ** -19 + half) * want.abs() + spread(got, want.shape) * lowest, "y in 8 bits")
    norm.close()


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("rows,n", [(1, 1), (3, 7), (2, 8), (5, 127), (4, 128), (1, 129), (9, 512), (7, 513), (130, 1000), (2, 1024), (6, 1111), (3, 2048),
                                    (5, 2049), (4, 4096), (3, 5000), (2, 8192), (3, 8193), (2, 16384), (2, 12001)])
def test_forward(rows, n, types):
    check_forward(rows, n, *types)


@pytest.mark.parametrize("residual,weight", [(False, True), (True, False), (False, False)])
def test_forward_without(residual, weight):
    for rows, n in ((5, 200), (3, 3000)):
        check_forward(rows, n, BF, BF, residual, weight)


@pytest.mark.parametrize("weight_dtype", (BF, F16))
def test_weights_of_16_bits(weight_dtype):
    check_forward(5, 333, BF, F32, weight_dtype=weight_dtype)


@pytest.mark.parametrize("pitch", (1, 3, 8))
@pytest.mark.parametrize("types", [(BF, BF), (F16, F32), (F32, F32)])
def test_strided_rows(types, pitch):
    check_forward(6, 300, *types, pitch=pitch)
    check_backward(6, 300, *types, pitch=pitch)


def check_backward(rows, n, x_type, h_type, dres=True, weight=True, pitch=0, seed=10):
    dy, h = normal(rows, n, seed=seed, dtype=x_type, pitch=pitch), normal(rows, n, seed=seed + 1, dtype=h_type, pitch=pitch)
    r = normal(rows, n, seed=seed + 2, dtype=h_type, pitch=pitch) if dres else None
    w = 1.0 + normal(1, n, seed=seed + 3, sigma=0.2)[0] if weight else None
    rstd = (h.double().square().mean(1) + 1e-6).rsqrt().float()
    norm = op(n, dtype=x_type, residual_dtype=h_type)
    dh, dw = norm.backward(dy, h, rstd, w, r)
    s, hd, dyd = rstd.double().cpu()[:, None], h.double().cpu(), dy.double().cpu()
    xhat = hd * s
    g = dyd * w.double().cpu() if weight else dyd
    want = s * (g - xhat * (g * xhat).mean(1, keepdim=True)) + (r.double().cpu() if dres else 0.0)
    size = s * (g.abs() + xhat.abs() * (g * xhat).abs().mean(1, keepdim=True)) + (r.double().cpu().abs() if dres else 0.0)
    within(dh, want, 2.0 ** -18 * size + HALF[h_type] * want.abs() + LOWEST[h_type], "dh")
    # (a sum of m numbers in any order: (m - 1) 2^-24 of their magnitudes; xhat and the products are rounded once each)
    within(dw, (dyd * xhat).sum(0), (rows + 8) * 2.0 ** -24 * (dyd * xhat).abs().sum(0), "dweight")
    again, dw2 = norm.backward(dy, h, rstd, w, r, dweight=dw.clone(), accumulate=True)
    assert torch.equal(again, dh) and torch.equal(dw2, dw + dw)
    norm.close()


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("rows,n", [(1, 1), (3, 7), (8, 128), (9, 129), (70, 512), (33, 513), (300, 1000), (5000, 64), (6, 1111), (17, 2048), (5, 2049), (4, 4096),
                                    (3, 5000), (9, 8192), (3, 8193), (700, 2048), (260, 16384)])
def test_backward(rows, n, types):
    check_backward(rows, n, *types)


@pytest.mark.parametrize("dres,weight", [(False, True), (True, False), (False, False)])
def test_backward_without(dres, weight):
    check_backward(20, 200, BF, BF, dres, weight)


def test_no_rows():
    norm = op(100)
    x = torch.empty(0, 100, device="cuda", dtype=BF)
    w = torch.ones(100, device="cuda")
    y, h, rstd = norm.forward(x, w, x)
    assert y.shape == h.shape == (0, 100) and rstd.shape == (0,)
    assert norm.forward8(x, w)[0].data.shape == (0, 100)
    dh, dw = norm.backward(x, x, rstd, w, dweight=torch.full((100,), 3.0, device="cuda"))
    assert dh.shape == (0, 100) and (dw == 0).all()
    assert (norm.backward(x, x, rstd, w, dweight=torch.full((100,), 3.0, device="cuda"), accumulate=True)[1] == 3).all()


@pytest.mark.parametrize("n", (40, 700, 3000, 9000))
def test_results_in_the_place_of_operands(n):
    norm = op(n, dtype=BF)
    x, r, w = normal(9, n, seed=1, dtype=BF), normal(9, n, seed=2, dtype=BF), torch.ones(n, device="cuda")
    y, h, rstd = norm.forward(x, w, r)
    for into in (0, 1):
        a, b = x.clone(), r.clone()
        y2, h2, _ = norm.forward(a, w, b, h=(a, b)[into])
        assert h2 is (a, b)[into] and torch.equal(h2, h) and torch.equal(y2, y)
    dy = normal(9, n, seed=3, dtype=BF)
    dh, dw = norm.backward(dy, h, rstd, w, r)
    for into in (0, 1):
        a, b = dy.clone(), r.clone()
        dh2, dw2 = norm.backward(a, h, rstd, w, b, out=(a, b)[into])
        assert torch.equal(dh2, dh) and torch.equal(dw2, dw)


def test_rows_that_are_not_finite_stay_alone():
    n = 300
    norm = op(n, dtype=BF)
    x = normal(6, n, seed=4, dtype=BF)
    w = torch.ones(n, device="cuda")
    y, _, _ = norm.forward(x, w)
    y8, _, _ = norm.forward8(x, w)
    x[2, 7], x[4, 299], x[5] = float("inf"), float("nan"), 0.0
    z, _, rstd = norm.forward(x, w)
    assert torch.equal(z[[0, 1, 3]], y[[0, 1, 3]])
    assert rstd[2] == 0 and z[2, 7].isnan() and (z[2, 8:] == 0).all()      # 1 / infinity; infinity times 0
    assert z[4].isnan().all() and (z[5] == 0).all()
    z8, _, _ = norm.forward8(x, w)
    v = values(z8)
    assert torch.equal(z8.data.view(torch.uint8)[[0, 1, 3]], y8.data.view(torch.uint8)[[0, 1, 3]]) and padding_is_zero(z8)
    assert v[2, :128].isnan().all() and (v[2, 128:] == 0).all() and v[4].isnan().all() and (v[5] == 0).all()


def test_zeros_without_eps_and_large_numbers():
    norm = op(64, dtype=F32, eps=0.0)
    x = torch.zeros(2, 64, device="cuda")
    x[1] = 1e18
    y, _, rstd = norm.forward(x)
    assert rstd[0].isinf() and y[0].isnan().all()      # 0 times infinity
    within(y[1], torch.ones(64, dtype=torch.float64), torch.tensor(2.0 ** -19), "y")


@pytest.mark.parametrize("types", [(F32, F32), (BF, BF), (F16, F32)])
@pytest.mark.parametrize("n", (1, 300, 700, 1500, 3000, 5000, 16384))
def test_rows_beyond_the_squares_of_binary32(n, types):
    """Rows whose squares over- or underflow in binary32, each next to an ordinary one, whose result is the one it has alone.  rstd is off by a
    rounding where it is below the normal numbers, 2^-150; what test_forward allows holds y."""
    x_type, h_type = types
    gen = torch.Generator().manual_seed(n)
    sizes = torch.tensor([1e18, 1.0, 1e20, 1.0, 1e30, 3e38, 1.0, 1e-22, 1.0, 1e-30, 1e-37])[:, None]
    r = ((0.1 + 0.9 * torch.rand(11, n, generator=gen)) * torch.randint(0, 2, (11, n), generator=gen).mul(2).sub(1) * sizes).to(h_type).cuda()
    x, w = torch.zeros(11, n, device="cuda", dtype=x_type), (1.0 + normal(1, n, seed=3, sigma=0.2)[0])
    for eps in (0.0, 1e-38, 1e-6):
        norm = op(n, dtype=x_type, residual_dtype=h_type, eps=eps)
        eps = torch.tensor(eps).double().item()      # (what the call is handed)
        y, h, rstd = norm.forward(x, w, r)
        assert torch.equal(h, r)
        want, want_rstd = want_forward(h, w, eps)
        within(rstd, want_rstd[:, 0], 2.0 ** -20 * want_rstd[:, 0] + 2.0 ** -150, "rstd")
        # (below bfloat16's normal numbers, where eps is far above a row's squares, its step is 2^-133)
        within(y, want, (2.0 ** -19 + HALF[x_type]) * want.abs() + max(LOWEST[x_type], 2.0 ** -133), "y")
        y8, _, rstd8 = norm.forward8(x, w, r)
        assert torch.equal(rstd8, rstd)
        within(values(y8), want, (2.0 ** -19 + 2.0 ** -4) * want.abs() + spread(y8.scales.cpu().double(), want.shape) * 2.0 ** -10, "y in 8 bits")
        rest = [1, 3, 6, 8]
        alone, _, rstd1 = norm.forward(x[rest].contiguous(), w, r[rest].contiguous())
        assert torch.equal(alone, y[rest]) and torch.equal(rstd1, rstd[rest])
        norm.close()


@pytest.mark.parametrize("n", (300, 700, 3000, 16384))
def test_gradients_of_rows_beyond_the_squares_of_binary32(n):
    """Against autograd in 64 bits: 2^-18 of the magnitudes that a gradient is the difference of, which are at most about twice its own here; a
    gradient of the largest rows and their rstd are below the normal numbers, 2^-21 off more."""
    gen = torch.Generator().manual_seed(n)
    sizes = torch.tensor([1e18, 1e20, 1.0, 1e30, 3e38, 1e-22, 1e-30])[:, None]
    x = ((0.1 + 0.9 * torch.rand(7, n, generator=gen)) * torch.randint(0, 2, (7, n), generator=gen).mul(2).sub(1) * sizes).cuda().requires_grad_()
    w, dy = (1.0 + normal(1, n, seed=3, sigma=0.2)[0]).requires_grad_(), normal(7, n, seed=4)
    op(n, dtype=F32, eps=0.0)(x, w).backward(dy)
    xd, wd = x.detach().double().requires_grad_(), w.detach().double().requires_grad_()
    (xd / xd.square().mean(1, keepdim=True).sqrt() * wd).backward(dy.double())
    assert ((x.grad.double() - xd.grad).norm(dim=1) <= 2.0 ** -16.5 * xd.grad.norm(dim=1)).all()
    assert (w.grad.double() - wd.grad).norm() <= 2.0 ** -18 * wd.grad.norm()


def test_gradients_against_differences():
    """Autograd's backward against central differences of the definition in 64 bits: the third derivative's share of them at 1e-4 is
    below 1e-6 of the numbers met here, and binary32 results are off by 2^-18 of the magnitudes."""
    n = 24
    norm = op(n, dtype=F32)
    x, r, w = (normal(5, n, seed=s) for s in (1, 2, 3))
    w = w[0].clone()
    c, d = normal(5, n, seed=4).double().cpu(), normal(5, n, seed=5).double().cpu()
    leaves = [t.clone().requires_grad_() for t in (x, w, r)]
    y, h = norm(*leaves)
    ((y * c.float().cuda()).sum() + (h * d.float().cuda()).sum()).backward()

    def loss(x, w, r):
        h = x + r
        return ((h / (h.square().mean(1, keepdim=True) + 1e-6).sqrt() * w) * c).sum() + (h * d).sum()
    for k, leaf in enumerate(leaves):
        host = [t.double().cpu() for t in (x, w, r)]
        got, flat = leaf.grad.double().cpu().view(-1), host[k].view(-1)
        for i in range(0, flat.numel(), 7):
            at, step = flat[i].item(), 1e-4
            flat[i] = at + step
            up = loss(*host)
            flat[i] = at - step
            down = loss(*host)
            flat[i] = at
            assert abs((up - down).item() / (2 * step) - got[i].item()) < 2e-5


def test_autograd_types_and_missing_gradients():
    norm = op(100, dtype=BF, residual_dtype=F32, weight_dtype=BF)
    x, r, w = normal(4, 100, seed=1, dtype=BF).requires_grad_(), normal(4, 100, seed=2).requires_grad_(), torch.ones(100, device="cuda", dtype=BF).requires_grad_()
    y, h = norm(x, w, r)
    y.sum().backward()                       # (h has no gradient, y's is one element seen as all)
    assert x.grad.dtype == BF and r.grad.dtype == F32 and w.grad.dtype == BF
    assert torch.equal(x.grad, r.grad.to(BF))
    y, h = norm(x, w, r)
    g, = torch.autograd.grad(h.sum(), r, create_graph=True)
    within(g, torch.ones(4, 100, dtype=torch.float64), torch.tensor(0.0), "of h alone")
    plain = op(100, dtype=BF)
    y = plain(x.detach().requires_grad_(), w.detach().float())
    assert y.dtype == BF


def test_another_stream_and_a_graph():
    norm = op(1000, dtype=BF)
    x, r, w = normal(200, 1000, seed=1, dtype=BF), normal(200, 1000, seed=2, dtype=BF), torch.ones(1000, device="cuda")
    y, h, rstd = norm.forward(x, w, r)
    dh, dw = norm.backward(y, h, rstd, w, r)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        y2, h2, rstd2 = norm.forward(x, w, r)
        dh2, dw2 = norm.backward(y2, h2, rstd2, w, r)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in ((y, y2), (dh, dh2), (dw, dw2)))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y3, h3, rstd3 = norm.forward(x, w, r)
        dh3, dw3 = norm.backward(y3, h3, rstd3, w, r)
    for k in range(3):
        x.copy_(normal(200, 1000, seed=20 + k, dtype=BF))
        graph.replay()
        y4, h4, rstd4 = norm.forward(x, w, r)
        want = norm.backward(y4, h4, rstd4, w, r)
        torch.cuda.synchronize()
        assert torch.equal(y3, y4) and torch.equal(dh3, want[0]) and torch.equal(dw3, want[1])


def test_offsets_beyond_32_bits():
    """Rows whose elements lie beyond 2^31 from the first."""
    n, rows, pitch = 128, 3, 1 << 30
    buf = torch.empty(2 * pitch + n, device="cuda", dtype=BF)
    x = buf.as_strided((rows, n), (pitch, 1))
    x.copy_(normal(rows, n, seed=1, dtype=BF))
    y, _, rstd = op(n, dtype=BF).forward(x)
    want, _ = want_forward(x, None, 1e-6)
    within(y, want, (2.0 ** -19 + HALF[BF]) * want.abs(), "y")
    dh, _ = op(n, dtype=BF).backward(y, x, rstd)
    ref, _ = op(n, dtype=BF).backward(y, x.contiguous(), rstd)
    assert torch.equal(dh, ref)


def test_more_rows_than_a_grid_has_threads_for():
    """2^21 rows of 1024 threads are as many as a launch counts."""
    n, rows = 4100, (1 << 21) + 5
    x = torch.zeros(rows, n, device="cuda", dtype=BF)
    x[:3], x[-9:] = normal(3, n, seed=1, dtype=BF), normal(9, n, seed=2, dtype=BF)
    norm = op(n, dtype=BF)
    y, _, rstd = norm.forward(x)
    for part in (slice(0, 3), slice(rows - 9, rows)):
        want, want_rstd = want_forward(x[part], None, 1e-6)
        within(y[part], want, (2.0 ** -19 + HALF[BF]) * want.abs(), "y")
        within(rstd[part], want_rstd[:, 0], 2.0 ** -20 * want_rstd[:, 0], "rstd")
    assert (y[3:1000] == 0).all() and (y[rows - 1000:rows - 9] == 0).all()
    del y
    y8, _, _ = norm.forward8(x)
    at = torch.arange(rows - 9, rows, device="cuda")
    numbers = y8.buffer[(rows - 9) * y8.ld:rows * y8.ld].view(9, y8.ld)[:, :n].view(E4M3).cpu().double()
    scales = y8.scales[at].cpu().double()
    within(numbers * spread(scales, (9, n)), want, (2.0 ** -19 + 2.0 ** -4) * want.abs() + spread(scales, (9, n)) * 2.0 ** -10, "y in 8 bits")


def test_refusals():
    norm = op(64, dtype=BF)
    x, w = torch.zeros(3, 64, device="cuda", dtype=BF), torch.ones(64, device="cuda")
    good = norm.forward(x, w)
    bad = [lambda: norm.forward(x[:, :63], w), lambda: norm.forward(x.float(), w), lambda: norm.forward(x.cpu(), w), lambda: norm.forward(x, w.to(BF)),
           lambda: norm.forward(x, w[:63]), lambda: norm.forward(x, w, x.float()), lambda: norm.forward(x, w, x[:2]), lambda: norm.forward(x, w, h=x),
           lambda: norm.forward(x[:1].expand(3, 64), w), lambda: norm.forward(torch.zeros(64, 3, device="cuda", dtype=BF).t(), w),
           lambda: norm.forward(x, w, out=torch.zeros(2, 64, device="cuda", dtype=BF)), lambda: norm.forward8(x, w, format=BF),
           lambda: norm.backward(x, x, good[2][:2], w), lambda: norm.backward(x, x[:2], good[2], w), lambda: norm.backward(x, x, good[2], w, accumulate=True),
           lambda: norm.backward(x, x, good[2], w, dweight=torch.zeros(64, device="cuda", dtype=BF))]
    for k, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail(str(k))
    for args in ((0,), (16385,), (64, F32, BF), (64, torch.float64)):
        with pytest.raises((ValueError, RuntimeError)):
            op(*args)
    with pytest.raises(RuntimeError):
        op(64, eps=-1.0)
    with pytest.raises(ValueError):
        op(64, dtype=BF, residual_dtype=F32)(x)
