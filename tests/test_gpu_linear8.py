"""The linear layer in 8 bits: what is quantised bit by bit against the definition, and the products against 64 bits, element by element.

Bounds: operands and their products are exact; they are summed in binary32 in some order, each addition off by at most 2^-23 of
what has been summed so far (twice a rounding, for a matrix core that truncates): depth 2^-23 |a| |b|; then one rounding of the result.
For results of 16 bits the matrix cores cut each of eight adjacent products off 13 bits below the largest power of two among them: less
than 8 2^-13 of that one for the eight, and 2^-10 |a| |b| for all (of normal numbers 1.5e-5 in the 2-norm, taken as 1e-4 there)."""
import itertools

import pytest

torch = pytest.importorskip("torch")
from tests.layer8 import E4M3, E5M2, HALF, LOWEST, padding_is_zero, quantized, spread, values, within  # noqa: E402

pytestmark = pytest.mark.gpu
BF, F16, F32 = torch.bfloat16, torch.float16, torch.float32


def op(*args, **kw):
    from paper_2104_06069_amd.linear8 import Linear8
    return Linear8(*args, **kw)


def numbers(rows, width, dtype, seed=0, pitch=0):
    """Normal numbers whose columns and rows differ in size, with a few blocks of zeros"""
    gen = torch.Generator().manual_seed(seed)
    t = torch.randn(rows, width + pitch, generator=gen) * torch.exp(torch.randn(width + pitch, generator=gen)) * torch.exp(torch.randn(rows, 1, generator=gen))
    if rows > 3:
        t[3] = 0
    if width > 200:
        t[:, 128:190] = 0
    t = t.to(dtype).cuda()
    return t[:, :width] if pitch else t


def same8(m, want, what):
    q, scales = want
    got, got_scales = m.data.cpu().double(), m.scales.cpu().double()
    assert torch.equal(got_scales.nan_to_num(-1), scales.nan_to_num(-1)), f"{what}: scales"
    assert torch.equal(got.nan_to_num(1e9), q.nan_to_num(1e9)), f"{what}: numbers"
    assert padding_is_zero(m), f"{what}: bytes behind the rows"


@pytest.mark.parametrize("dtype,fmt", itertools.product((BF, F16, F32), (E4M3, E5M2)))
@pytest.mark.parametrize("rows,width,pitch", [(1, 1, 0), (1, 1024, 0), (3, 7, 1), (8, 128, 0), (130, 129, 0), (128, 256, 8), (257, 500, 3), (1000, 64, 0)])
def test_quantize(rows, width, pitch, dtype, fmt):
    t = numbers(rows, width, dtype, pitch=pitch)
    layer = op(width, 64)
    same8(layer.quantize(t, fmt), quantized(t.cpu(), fmt), "rows")
    m, mt = layer._quantize(t, "t", width, fmt, E4M3)
    same8(m, quantized(t.cpu(), fmt), "rows, of both")
    same8(mt, quantized(t.cpu().t().contiguous(), E4M3), "columns, of both")
    same8(layer._quantize(t, "t", width, None, fmt)[1], quantized(t.cpu().t().contiguous(), fmt), "columns")
    w8 = op(width, rows).quantize_weight(t)
    same8(w8.w, quantized(t.cpu(), E4M3, square=True), "squares")
    q, scales = quantized(t.cpu(), E4M3, square=True)
    same8(w8.transposed, (q.t(), scales.t()), "squares, transposed")


@pytest.mark.parametrize("rows,width,dtype", [(40001, 1701, BF), (70000, 960, F16), (19000, 1900, F32)])
def test_quantize_past_the_caches(rows, width, dtype):
    """More numbers than the rule for that asks for (128 MB): the same as a few thousand rows at a time."""
    gen = torch.Generator("cuda").manual_seed(1)
    t = (torch.randn(rows, width, generator=gen, device="cuda") * torch.exp(torch.randn(rows, 1, generator=gen, device="cuda"))).to(dtype)
    assert t.numel() * t.element_size() > 128 << 20
    t[77, 5], t[rows - 1, width - 1] = float("inf"), float("nan")
    layer = op(width, 64)
    alone, (m, mt), turned = layer.quantize(t, E5M2), layer._quantize(t, "t", width, E4M3, E5M2), layer._quantize(t, "t", width, None, E4M3)[1]
    for i in range(0, rows, 4096):
        part = t[i:i + 4096]
        k, j = part.shape[0], i // 128
        want, (w, wt), wturned = layer.quantize(part, E5M2), layer._quantize(part, "t", width, E4M3, E5M2), layer._quantize(part, "t", width, None, E4M3)[1]
        for got, of in ((alone, want), (m, w)):
            assert torch.equal(got.buffer[:rows * got.ld].view(rows, -1)[i:i + k], of.buffer[:k * of.ld].view(k, -1))
            assert torch.equal(got.scales.view(torch.uint8)[i:i + k], of.scales.view(torch.uint8))
        for got, of in ((mt, wt), (turned, wturned)):
            assert torch.equal(got.buffer[:width * got.ld].view(width, -1)[:, i:i + of.ld], of.buffer[:width * of.ld].view(width, -1))
            assert torch.equal(got.scales.view(torch.uint8)[:, j:j + (k + 127) // 128], of.scales.view(torch.uint8))


@pytest.mark.parametrize("fmt,largest", [(E4M3, 448.0), (E5M2, 57344.0)])
def test_quantize_at_the_borders(fmt, largest):
    """Largest magnitudes at the border between two scales and a bit beside it, ties, numbers below the format's and binary32's smallest, and what
    is not finite."""
    t = torch.zeros(16, 130)
    up, down = torch.nextafter(torch.tensor(largest), torch.tensor(1e9)).item(), torch.nextafter(torch.tensor(largest), torch.tensor(0.0)).item()
    for row, v in enumerate((largest, up, down, largest * 2.0 ** -100, 3.4e38, 1e-38, 1e-45, 2.0 ** -126 * largest, 1.0)):
        t[row, 5] = v
    t[0, 6:12] = torch.tensor([17.0, 18.0, 19.0, -17.0, 2.0 ** -10, 1.5 * 2.0 ** -9])
    t[8, 6:70] = torch.arange(64) / 64.0
    t[9, 3], t[10, 127], t[11, 129], t[12, 128] = float("inf"), float("nan"), -float("inf"), float("nan")
    t[9:13, 40] = 1.0
    layer = op(130, 64)
    same8(layer.quantize(t.cuda(), fmt), quantized(t, fmt), "rows")
    same8(layer._quantize(t.cuda(), "t", 130, None, fmt)[1], quantized(t.t().contiguous(), fmt), "columns")


def product_near(got, a, b, depth, what):
    """got = a b^T"""
    want, size = a @ b.T, a.abs() @ b.abs().T
    short = 0.0 if got.dtype == F32 else 2.0 ** -10
    bound = (depth * 2.0 ** -23 + short) * size + HALF[got.dtype] * want.abs() + LOWEST[got.dtype]
    if got.dtype == F16:      # an infinity where the result, as far off as it may be, is beyond the largest number and half a step, 65520
        beyond = got.double().cpu().isinf()
        assert (want.abs() + bound >= 65520)[beyond].all() and (want.sign() * bound.sign() == got.double().cpu().sign())[beyond].all(), what
        got, want = torch.where(beyond.to(got.device), torch.zeros_like(got), got), torch.where(beyond, torch.zeros_like(want), want)
    within(got, want, bound, what)
    if got.dtype != F32 and want.numel() > 100:
        off = (got.double().cpu() - want).norm() / want.norm()
        assert off <= 1e-4 + HALF[got.dtype], what


SIZES = [(1, 1, 1), (2, 64, 64), (5, 128, 16), (16, 200, 130), (17, 1024, 33), (63, 77, 520), (64, 256, 64), (65, 130, 65), (129, 500, 257), (300, 64, 300),
         (33, 2000, 64), (1, 3000, 500), (513, 384, 270), (700, 1100, 140)]


@pytest.mark.parametrize("rows,k,n", SIZES)
@pytest.mark.parametrize("dtype,grad", [(BF, E4M3), (F16, E5M2)])
def test_products(rows, k, n, dtype, grad):
    layer = op(k, n, dtype=dtype, grad_format=grad)
    x, dy, w = numbers(rows, k, dtype, 1), numbers(rows, n, dtype, 2), numbers(n, k, dtype, 3)
    w8 = layer.quantize_weight(w)
    wv = values(w8.w)
    y = layer.forward(x, w8)
    xv = values(layer.quantize(x))
    product_near(y, xv, wv, k, "y")
    dx, dw = layer.backward(x, dy, w8)
    product_near(dx, values(layer.quantize(dy, grad)), wv.T, n, "dx")
    dyt = values(layer._quantize(dy, "dy", n, None, grad)[1])
    xt = values(layer._quantize(x, "x", k, None, E4M3)[1])
    product_near(dw, dyt, xt, rows, "dw")
    assert torch.equal(layer.input_grad(dy, w8), dx) and torch.equal(layer.weight_grad(x, dy), dw)
    assert torch.equal(layer.forward(layer.quantize(x), w8), y)
    y5 = layer.forward(layer.quantize(x, E5M2), w8, out_dtype=F32)
    product_near(y5, values(layer.quantize(x, E5M2)), wv, k, "y from e5m2")
    layer.close()


@pytest.mark.parametrize("rows,k,n", [(64, 130, 65), (40, 100, 72), (2000, 60, 50), (300, 1000, 30)])
def test_types_strides_and_accumulation(rows, k, n):
    layer = op(k, n, dtype=BF)
    x, dy, w = numbers(rows, k, F32, 1, pitch=3), numbers(rows, n, BF, 2, pitch=5), numbers(n, k, F32, 3, pitch=1)
    w8 = layer.quantize_weight(w)
    for dtype in (F32, F16, BF):
        wide = torch.full((rows, n + 7), 5.0, device="cuda", dtype=dtype)
        y = layer.forward(x, w8, out=wide[:, 3:n + 3])
        assert torch.equal(y, layer.forward(x, w8, out_dtype=dtype)) and (wide[:, :3] == 5).all() and (wide[:, n + 3:] == 5).all()
    once = layer.weight_grad(x, dy)
    size = values(layer._quantize(dy, "dy", n, None, E4M3)[1]).abs() @ values(layer._quantize(x, "x", k, None, E4M3)[1]).abs().T
    start = torch.randn(n, k, device="cuda")
    flat = torch.zeros(n * k + 11, device="cuda")
    view = flat[5:5 + n * k].view(n, k)
    view.copy_(start)
    twice = layer.weight_grad(x, dy, out=view, accumulate=True)
    assert torch.equal(twice, start + once) and (flat[:5] == 0).all() and (flat[5 + n * k:] == 0).all()
    within(layer.weight_grad(x, dy, out_dtype=BF), once.double().cpu(), 2.0 ** -7 * once.double().cpu().abs() + 2.0 ** -9 * size, "dw in 16 bits")


def test_no_rows():
    layer = op(100, 72)
    x, dy = torch.empty(0, 100, device="cuda", dtype=BF), torch.empty(0, 72, device="cuda", dtype=BF)
    w8 = layer.quantize_weight(numbers(72, 100, BF))
    assert layer.forward(x, w8).shape == (0, 72)
    dx, dw = layer.backward(x, dy, w8, dw=torch.full((72, 100), 3.0, device="cuda"))
    assert dx.shape == (0, 100) and (dw == 0).all()
    assert (layer.weight_grad(x, dy, out=torch.full((72, 100), 3.0, device="cuda"), accumulate=True) == 3).all()


def test_values_that_are_not_finite_stay_in_their_rows():
    for rows in (5, 200):
        layer = op(300, 80)
        x, w = numbers(rows, 300, BF, 1), numbers(80, 300, BF, 2)
        w8 = layer.quantize_weight(w)
        y = layer.forward(x, w8)
        x[1, 299], x[4, 0] = float("inf"), float("nan")
        z = layer.forward(x, w8)
        rest = [r for r in range(rows) if r not in (1, 4)]
        assert torch.equal(z[rest], y[rest]) and z[1].isnan().all() and z[4].isnan().all()
        w[7, 3] = float("nan")      # a square of the weights: its 128 rows of W
        z = layer.forward(x, layer.quantize_weight(w))
        assert z.isnan().all()


def test_gradients_of_autograd():
    """Whole numbers up to 4 are exact in 8 bits, and so are these sums: the gradients are those of the plain product."""
    for dtype in (BF, F32):
        layer = op(96, 40, dtype=dtype)
        gen = torch.Generator().manual_seed(0)
        whole = lambda *s: torch.randint(-4, 5, s, generator=gen).to(dtype).cuda()  # noqa: E731
        x, w, c = whole(50, 96), whole(40, 96), whole(50, 40)
        xl, wl = x.clone().requires_grad_(), w.clone().requires_grad_()
        y = layer(xl, wl)
        y.backward(c)
        xd, wd, cd = x.double().cpu(), w.double().cpu(), c.double().cpu()
        zero = torch.zeros(())
        within(y, xd @ wd.T, HALF[dtype] * (xd @ wd.T).abs(), "y")
        within(xl.grad, cd @ wd, HALF[dtype] * (cd @ wd).abs(), "dx")
        within(wl.grad, cd.T @ xd, HALF[dtype] * (cd.T @ xd).abs() + zero, "dw")
        assert wl.grad.dtype == dtype and xl.grad.dtype == dtype
        only = x.clone().requires_grad_()
        layer(only, w).backward(c)
        assert torch.equal(only.grad, xl.grad)
        only = w.clone().requires_grad_()
        layer(x, only).sum().backward()
        assert only.grad is not None
        # differences: the product is linear, so that steps of a whole number are exact
        up, down = x.clone(), x.clone()
        up[3, 5] += 1
        down[3, 5] -= 1
        diff = ((layer(up, w).double() - layer(down, w).double()) * c.double()).sum() / 2
        if dtype == F32:
            assert diff.item() == xl.grad[3, 5].item()


def test_another_stream_and_a_graph():
    layer = op(600, 200)
    x, dy, w = numbers(500, 600, BF, 1), numbers(500, 200, BF, 2), numbers(200, 600, BF, 3)

    def step():
        w8 = layer.quantize_weight(w)
        return (layer.forward(x, w8), layer.forward(x[:3], w8)) + layer.backward(x, dy, w8)
    want = step()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = step()
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for k in range(3):
        x.copy_(numbers(500, 600, BF, 10 + k))
        graph.replay()
        want = step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_refusals():
    layer = op(64, 32)
    x, dy, w = (torch.zeros(5, 64, device="cuda", dtype=BF), torch.zeros(5, 32, device="cuda", dtype=BF), torch.zeros(32, 64, device="cuda"))
    w8 = layer.quantize_weight(w)
    x8 = layer.quantize(x)
    bad = [lambda: layer.forward(x[:, :63], w8), lambda: layer.forward(x.cpu(), w8), lambda: layer.forward(x.double(), w8), lambda: layer.forward(x8, w),
           lambda: layer.forward(dy, w8), lambda: layer.forward(w8.w, w8), lambda: layer.quantize_weight(w.t()), lambda: layer.quantize_weight(w[:31]),
           lambda: layer.quantize(x, BF), lambda: layer.forward(x[:1].expand(5, 64), w8), lambda: layer.forward(x, w8, out=torch.zeros(4, 32, device="cuda")),
           lambda: layer.weight_grad(x, dy[:4]), lambda: layer.weight_grad(x, dy, accumulate=True), lambda: layer.quantize(x[0]),
           lambda: layer.weight_grad(x, dy, out=torch.zeros(32, 64, device="cuda", dtype=BF), accumulate=True), lambda: op(64, 32, grad_format=BF),
           lambda: op(64, 32, dtype=torch.float64)]
    from paper_2104_06069_amd.linear8 import Weight8
    other = op(32, 64).quantize_weight(w.t().contiguous())
    bad += [lambda: layer.weight_grad(x8, dy), lambda: layer.weight_grad(x, layer.quantize(dy)), lambda: layer.quantize(x8), lambda: layer.backward(x8, dy, w8),
            lambda: layer.forward(x, Weight8(w8.w, w8.w)), lambda: layer.input_grad(dy, Weight8(w8.w, layer.quantize(w.t().contiguous()))),
            lambda: layer.forward(x, Weight8(layer.quantize(w), w8.transposed)), lambda: layer.forward(x, other)]
    for k, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail(str(k))
    for args in ((0, 4), (4, 0), (1 << 21, 4)):
        with pytest.raises(RuntimeError):
            op(*args)
    with pytest.raises(RuntimeError):
        op(64, 32, max_rows=4).forward(x, w8)


@pytest.mark.parametrize("rows,k,n", [(1, 1024, 4096), (1, 100, 72), (3, 9000, 40), (16, 2048, 9000), (7, 130, 8200), (16, 500, 300), (15, 3000, 16), (31, 2100, 8192),
                                      (32, 130, 20), (50, 2500, 33), (64, 700, 8200), (1, 17000, 200)])
@pytest.mark.parametrize("dtype", (BF, F16, F32))
def test_few_rows(rows, k, n, dtype):
    """One token and a few: from x itself and from its 8 bits, the same."""
    layer = op(k, n, dtype=dtype)
    x, w = numbers(rows, k, dtype, 1, pitch=5), numbers(n, k, BF, 3)
    w8 = layer.quantize_weight(w)
    x8 = layer.quantize(x)
    y = layer.forward(x, w8)
    product_near(y, values(x8), values(w8.w), k, "y")
    assert torch.equal(layer.forward(x8, w8), y)
    assert torch.equal(layer.forward(layer.quantize(x, E5M2), w8), layer.forward(layer.quantize(x, E5M2), w8))
    dy = numbers(rows, n, dtype, 4)
    product_near(layer.input_grad(dy, w8), values(layer.quantize(dy)), values(w8.w).T, n, "dx")
    if rows < 40:      # a weight gradient of few rows of W
        few = op(k, rows, dtype=dtype)
        xs, g = numbers(300, k, dtype, 5), numbers(300, rows, dtype, 6)
        product_near(few.weight_grad(xs, g), values(few._quantize(g, "dy", rows, None, E4M3)[1]), values(few._quantize(xs, "x", k, None, E4M3)[1]), 300, "dw")


@pytest.mark.parametrize("rows,k,n", [(4096, 512, 2048), (5000, 300, 4200), (4070, 1000, 4090), (4090, 2100, 4096), (8190, 2100, 4096), (20000, 400, 1032), (4097, 300, 4097), (2100, 1000, 3000), (600, 4100, 2056), (3000, 130, 3000), (70, 5000, 70), (70, 30000, 100), (100, 2000, 130), (1000, 1100, 990)])
@pytest.mark.parametrize("dtype", (BF, F16, F32))
def test_many_tiles(rows, k, n, dtype):
    """Sizes that take every kind of tile, several for a workgroup, and sums in parts; sums in 64 bits on the device."""
    layer = op(k, n, dtype=dtype)
    x, w = numbers(rows, k, BF, 1) / 64, numbers(n, k, BF, 3) / 64
    w8, x8 = layer.quantize_weight(w), layer.quantize(x)
    wide = torch.full((rows + 2, n + 8), 7.0, device="cuda", dtype=dtype)
    y = layer.forward(x8, w8, out=wide[1:rows + 1, :n])
    assert (wide[0] == 7).all() and (wide[rows + 1:] == 7).all() and (wide[:, n:] == 7).all()
    a, b = values(x8).cuda(), values(w8.w).cuda()
    want, size = a @ b.T, a.abs() @ b.abs().T
    bound = (k * 2.0 ** -23 + (0.0 if dtype == F32 else 2.0 ** -10)) * size + HALF[dtype] * want.abs() + LOWEST[dtype]
    got, beyond = y.double(), want.abs() + bound >= 65520 if dtype == F16 else torch.zeros_like(want, dtype=torch.bool)
    assert (((got - want).abs() <= bound) | beyond).all()
    assert (got[~beyond] - want[~beyond]).norm() / want[~beyond].norm() <= HALF[dtype] + (2e-6 if dtype == F32 else 1e-4)
    assert torch.equal(layer.forward(x8, w8), y)


@pytest.mark.parametrize("rows,k,n", [(2100, 4096, 4096), (2100, 4096, 8190), (2100, 4090, 4096), (1000, 200, 4096)])
def test_accumulating_into_many_tiles(rows, k, n):
    layer = op(k, n)
    x, dy = numbers(rows, k, BF, 1), numbers(rows, n, BF, 2)
    once = layer.weight_grad(x, dy)
    flat = torch.randn(n * k + 16, device="cuda")
    view, start = flat[8:8 + n * k].view(n, k), flat.clone()
    layer.weight_grad(x, dy, out=view, accumulate=True)
    assert torch.equal(view, start[8:8 + n * k].view(n, k) + once) and torch.equal(flat[:8], start[:8]) and torch.equal(flat[-8:], start[-8:])
    layer.weight_grad(x, dy, out=view)
    assert torch.equal(view, once)


@pytest.mark.parametrize("rows,k,n", [(1, 1024, 4096), (5, 100, 72), (16, 2048, 9000), (7, 130, 8200), (16, 9000, 40), (3, 17000, 64)])
@pytest.mark.parametrize("dtype", (BF, F16, F32))
def test_few_rows_made_e5m2_on_the_way(rows, k, n, dtype):
    """ob_linear8_forward_few with the other format, from rows some elements apart into rows some apart."""
    from paper_2104_06069_amd import binding as ob
    codes = {F32: ob.OB_F32, F16: ob.OB_F16, BF: ob.OB_BF16}
    layer = op(k, n)
    x, w8 = numbers(rows, k, dtype, 1, pitch=3), layer.quantize_weight(numbers(n, k, BF, 2))
    x8 = layer.quantize(x, E5M2)
    for out_dtype in (BF, F16, F32):
        wide = torch.full((rows, n + 5), 5.0, device="cuda", dtype=out_dtype)
        y = wide[:, 2:n + 2]
        ob.ob_linear8_forward_few(layer.ctx, x, codes[dtype], k + 3, ob.OB_E5M2, *w8.w.address(), rows, y, n + 5, codes[out_dtype],
                                  torch.cuda.current_stream().cuda_stream)
        product_near(y, values(x8), values(w8.w), k, "y")
        product_near(layer.forward(x8, w8, out_dtype=out_dtype), values(x8), values(w8.w), k, "y from 8 bits")
        assert (wide[:, :2] == 5).all() and (wide[:, n + 2:] == 5).all()
    with pytest.raises(RuntimeError):
        ob.ob_linear8_forward_few(layer.ctx, x, codes[dtype], k + 3, 2, *w8.w.address(), rows, y, n + 5, ob.OB_F32)
    with pytest.raises(RuntimeError):
        ob.ob_linear8_forward_few(layer.ctx, x, codes[dtype], k + 3, ob.OB_E5M2, *w8.w.address(), ob.OB_LINEAR8_FEW_ROWS + 1, y, n + 5, ob.OB_F32)


@pytest.mark.parametrize("fmt,largest,lowest", [(E4M3, 448.0, -124), (E5M2, 57344.0, -117)])
@pytest.mark.parametrize("rows", (5, 70, 8192))
def test_binary32_results_are_exact_down_to_these_scales(rows, fmt, largest, lowest):
    """Numbers down to 2^-133, bfloat16's smallest: multiples of it up to 200, times whole numbers up to 8 (times 2^90), 256 of them: sums below 2^19
    such units, exact in binary32."""
    k, n = 256, 2048
    layer = op(k, n, dtype=F32)
    gen = torch.Generator().manual_seed(rows)
    x = torch.randint(-200, 201, (rows, k), generator=gen).double() * 2.0 ** -133
    x[:, 0] = x[:, 128] = largest * 2.0 ** lowest
    w = torch.randint(-8, 9, (n, k), generator=gen).float() * 2.0 ** 90
    w[:, 0] = w[:, 128] = 0      # (beside numbers that set the scale)
    x8, w8 = layer.quantize(x.float().cuda(), fmt), layer.quantize_weight(w.cuda())
    assert (x8.scales.cpu().double() == 2.0 ** lowest).all()
    assert torch.equal(layer.forward(x8, w8).double(), values(x8).cuda() @ values(w8.w).cuda().T.contiguous())


def test_types_of_results_are_refused_like_others():
    layer = op(64, 32)
    x, dy = torch.zeros(20, 64, device="cuda", dtype=BF), torch.zeros(20, 32, device="cuda", dtype=BF)
    w8 = layer.quantize_weight(torch.zeros(32, 64, device="cuda"))
    for call in (lambda: layer.forward(x, w8, out_dtype=torch.float64), lambda: layer.forward(x[:1], w8, out_dtype=E4M3), lambda: layer.input_grad(dy, w8, out_dtype=torch.int32),
                 lambda: layer.weight_grad(x, dy, out_dtype=torch.float64), lambda: layer.backward(x, dy, w8, dw_dtype=E5M2)):
        with pytest.raises(ValueError):
            call()
