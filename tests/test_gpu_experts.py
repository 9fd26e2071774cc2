"""The products of an expert layer against the definition in 64 bits, element by element.

Bounds: operands are exact, n products are summed in binary32 in some order, each addition off by at most 2^-23 of what has
been summed so far (twice a rounding, for a matrix core that truncates): depth 2^-23 |x| |w|; then one rounding of the
result, 2^-8 (bfloat16), 2^-11 (binary16, or 2^-25 below its normal numbers) or 2^-24 of it."""
import itertools

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
ROUNDING = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}


def layer(*args, **kw):
    from paper_2104_06069_amd.experts import ExpertLinear
    return ExpertLinear(*args, **kw)


def inputs(counts, k, n, dtype, layout, seed=0, ld_extra=0, first=0, after=0):
    gen = torch.Generator().manual_seed(seed)
    rows, G = first + sum(counts) + after, len(counts)
    def made(*shape):
        t = torch.randn(*shape, generator=gen).to(dtype).cuda()
        return t[:, :shape[1] - ld_extra] if ld_extra else t
    x, dy = made(rows, k + ld_extra), made(rows, n + ld_extra)
    w = torch.randn(*((G, k, n) if layout == "kn" else (G, n, k)), generator=gen).to(dtype).cuda()
    offsets = torch.tensor([first] + (first + np.cumsum(counts)).tolist(), dtype=torch.int32).cuda()
    return x, dy, w, offsets


def near(got, want, size, depth, what):
    """size: the sum of the products' magnitudes."""
    err = (got.double().cpu() - want).abs()
    bound = depth * 2.0 ** -23 * size + ROUNDING[got.dtype] * want.abs() + (2.0 ** -25 if got.dtype == torch.float16 else 0.0)
    worst = (err - bound).max().item() if err.numel() else 0.0
    assert worst <= 0.0, f"{what}: {err.max().item():.3g} off, {worst:.3g} over its bound"


def check(counts, k, n, dtype, layout, out_dtype=None, dw_dtype=torch.float32, **kw):
    x, dy, w, offsets = inputs(counts, k, n, dtype, layout, **kw)
    out_dtype = out_dtype or dtype
    op = layer(len(counts), k, n, dtype=dtype, max_rows=x.shape[0], layout=layout)
    mark = 77.0
    y = torch.full((x.shape[0], n), mark, dtype=out_dtype, device="cuda")
    dx = torch.full((x.shape[0], k), mark, dtype=out_dtype, device="cuda")
    dw = torch.full(op.w_shape, mark, dtype=dw_dtype, device="cuda")
    op.forward(x, w, offsets, out=y)
    op.input_grad(dy, w, offsets, out=dx)
    op.weight_grad(x, dy, offsets, out=dw)
    torch.cuda.synchronize()
    ends = offsets.tolist()
    xd, dyd, wd = x.double().cpu(), dy.double().cpu(), w.double().cpu()
    wd = wd if layout == "kn" else wd.transpose(1, 2)
    dwc = dw.cpu() if layout == "kn" else dw.cpu().transpose(1, 2)
    for g, (a, b) in enumerate(zip(ends[:-1], ends[1:])):
        near(y[a:b], xd[a:b] @ wd[g], xd[a:b].abs() @ wd[g].abs(), k, f"y of group {g}")
        near(dx[a:b], dyd[a:b] @ wd[g].T, dyd[a:b].abs() @ wd[g].T.abs(), n, f"dx of group {g}")
        near(dwc[g], xd[a:b].T @ dyd[a:b], xd[a:b].T.abs() @ dyd[a:b].abs(), b - a, f"dw of group {g}")
    for t in (y, dx):
        assert (t[:ends[0]] == mark).all() and (t[ends[-1]:] == mark).all(), "rows that belong to no group"
    op.close()


@pytest.mark.parametrize("dtype,layout", itertools.product((torch.bfloat16, torch.float16), ("kn", "nk")))
@pytest.mark.parametrize("counts,k,n", [
    ([1], 8, 8), ([1, 0, 3], 64, 64), ([64, 64], 64, 128), ([5, 0, 0, 130, 63], 128, 192), ([65, 1, 257], 72, 200),
    ([0, 0, 0], 64, 64), ([300, 17], 257, 96), ([33, 2, 90], 100, 129), ([7, 40], 1, 1), ([9, 3], 3, 70), ([20, 11], 70, 5),
    ([260, 515], 320, 264), ([1] * 70 + [0] * 30 + [2] * 40, 96, 64), ([700, 0, 3], 520, 1000),
])
def test_against_64_bits(counts, k, n, dtype, layout):
    check(counts, k, n, dtype, layout)


@pytest.mark.parametrize("layout", ("kn", "nk"))
@pytest.mark.parametrize("counts,k,n", [([1, 1, 0, 0, 0, 0, 0, 0], 1024, 1024), ([2, 9, 0, 16, 17], 512, 320), ([3, 31], 2048, 72),
                                        ([1000, 20, 300], 512, 512), ([2500], 256, 512), ([3000, 10], 64, 64), ([1], 2500, 40)])
def test_longer_sums_and_more_tiles(counts, k, n, layout):
    check(counts, k, n, torch.bfloat16, layout)


@pytest.mark.parametrize("layout", ("kn", "nk"))
def test_strided_rows_and_rows_of_no_group(layout):
    check([40, 0, 77], 96, 136, torch.float16, layout, ld_extra=8, first=5, after=9)
    check([40, 0, 77], 96, 136, torch.bfloat16, layout, ld_extra=3, first=1, after=2)
    check([3, 2, 1], 96, 136, torch.bfloat16, layout, ld_extra=3, first=1, after=2)


@pytest.mark.parametrize("out_dtype,dw_dtype", [(torch.float32, torch.bfloat16), (torch.bfloat16, torch.bfloat16)])
def test_types_of_the_results(out_dtype, dw_dtype):
    check([40, 0, 77], 96, 136, torch.bfloat16, "kn", out_dtype=out_dtype, dw_dtype=dw_dtype)
    check([2, 0, 5], 200, 77, torch.bfloat16, "nk", out_dtype=out_dtype, dw_dtype=dw_dtype)


def test_no_rows_at_all():
    op = layer(3, 64, 32, max_rows=0)
    x, dy = torch.empty(0, 64, device="cuda", dtype=torch.bfloat16), torch.empty(0, 32, device="cuda", dtype=torch.bfloat16)
    w, offsets = torch.ones(3, 64, 32, device="cuda", dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int32, device="cuda")
    assert op.forward(x, w, offsets).shape == (0, 32)
    dw = op.weight_grad(x, dy, offsets, out=torch.full((3, 64, 32), 5.0, device="cuda"))
    assert (dw == 0).all()


@pytest.mark.parametrize("counts", ([30, 0, 50], [2, 0, 3]))
def test_accumulating_weight_gradient(counts):
    x, dy, _, offsets = inputs(counts, 72, 80, torch.bfloat16, "kn")
    op = layer(3, 72, 80, max_rows=x.shape[0])
    once = op.weight_grad(x, dy, offsets, out_dtype=torch.float32)
    start = torch.randn(3, 72, 80, device="cuda")
    twice = op.weight_grad(x, dy, offsets, out=start.clone(), accumulate=True)
    assert torch.equal(twice, start + once)


def test_weights_inside_a_flat_buffer():
    """Experts' weights with other tensors between them, at addresses that are no multiples of 16 bytes."""
    G, k, n, gap, first = 3, 48, 40, 7, 5
    gen = torch.Generator().manual_seed(3)
    flat = torch.randn(first + G * (k * n + gap), generator=gen).to(torch.bfloat16).cuda()
    grad = torch.full((flat.numel(),), 9.0, device="cuda")
    view = lambda t: t[first:].as_strided((G, k, n), (k * n + gap, n, 1))  # noqa: E731
    x, dy, _, offsets = inputs([20, 0, 33], k, n, torch.bfloat16, "kn")
    op = layer(G, k, n, max_rows=53, w_stride=k * n + gap)
    y = op.forward(x, view(flat), offsets, out_dtype=torch.float32)
    op.weight_grad(x, dy, offsets, out=view(grad))
    for g, (a, b) in enumerate([(0, 20), (20, 20), (20, 53)]):
        xd, wd, dd = x[a:b].double().cpu(), view(flat)[g].double().cpu(), dy[a:b].double().cpu()
        near(y[a:b], xd @ wd, xd.abs() @ wd.abs(), k, "y")
        near(view(grad)[g], xd.T @ dd, xd.T.abs() @ dd.abs(), b - a, "dw")
    rest = torch.ones_like(grad, dtype=torch.bool)
    view(rest)[:] = False
    assert (grad[rest] == 9.0).all()


def test_values_that_are_not_finite_stay_where_they_are():
    """An infinity or a NaN in a group's last row reaches that row's results and that group's weight gradient alone, also where
    the slab that holds it ends inside."""
    for counts, layout in itertools.product(([65, 3, 70], [2, 3, 1]), ("kn", "nk")):
        x, dy, w, offsets = inputs(counts, 100, 72, torch.float16, layout)
        ends = offsets.tolist()
        clean = layer(3, 100, 72, dtype=torch.float16, max_rows=200, layout=layout)
        y0, dw0 = clean.forward(x, w, offsets), clean.weight_grad(x, dy, offsets, out_dtype=torch.float32)
        x[ends[1] - 1, 99], x[ends[3] - 1, 0] = float("inf"), float("nan")
        y1, dw1 = clean.forward(x, w, offsets), clean.weight_grad(x, dy, offsets, out_dtype=torch.float32)
        for r in range(ends[3]):
            if r in (ends[1] - 1, ends[3] - 1):
                assert not torch.isfinite(y1[r]).any()
            else:
                assert torch.equal(y0[r], y1[r])
        assert torch.equal(dw0[1], dw1[1]) and not torch.isfinite(dw1[0]).all() and not torch.isfinite(dw1[2]).all()


def test_offsets_are_brought_into_range():
    """A table that is no table reads and writes nothing out of bounds."""
    x, dy, w, _ = inputs([10, 10, 10], 64, 64, torch.bfloat16, "kn")
    op = layer(3, 64, 64, max_rows=30)
    offsets = torch.tensor([-7, 12, 12, 1 << 30], dtype=torch.int32, device="cuda")
    y = op.forward(x, w, offsets)
    want = op.forward(x, w, torch.tensor([0, 12, 12, 30], dtype=torch.int32, device="cuda"))
    assert torch.equal(y, want)
    op.weight_grad(x, dy, torch.tensor([5, 2, -1, 3], dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()


@pytest.mark.parametrize("layout", ("kn", "nk"))
@pytest.mark.parametrize("counts", ([5, 0, 40, 12], [1, 0, 2, 1]))
def test_gradients_against_differences(counts, layout):
    """On small whole numbers every sum is exact: what y changes by along a direction is what the gradients say, to the last bit."""
    k, n, G, rows = 40, 24, 4, sum(counts)
    gen = torch.Generator().manual_seed(1)
    whole = lambda *s: torch.randint(-3, 4, s, generator=gen).to(torch.bfloat16).cuda()  # noqa: E731
    op = layer(G, k, n, max_rows=rows, layout=layout)
    x, dy, w, vx, vw = whole(rows, k), whole(rows, n), whole(*op.w_shape), whole(rows, k), whole(*op.w_shape)
    offsets = torch.tensor(np.concatenate([[0], np.cumsum(counts)]), dtype=torch.int32, device="cuda")
    f = lambda a, b: (op.forward(a, b, offsets, out_dtype=torch.float32).double() * dy.double()).sum().item()  # noqa: E731
    dx, dw = op.input_grad(dy, w, offsets, out_dtype=torch.float32), op.weight_grad(x, dy, offsets, out_dtype=torch.float32)
    assert f(x + vx, w) - f(x, w) == (dx.double() * vx.double()).sum().item()
    assert f(x, w + vw) - f(x, w) == (dw.double() * vw.double()).sum().item()
    xa, wa = x.clone().requires_grad_(), w.clone().requires_grad_()
    op(xa, wa, offsets).backward(dy)
    assert torch.equal(xa.grad, dx.to(torch.bfloat16)) and torch.equal(wa.grad, dw.to(torch.bfloat16))


def test_on_another_stream_and_twice_the_same():
    x, dy, w, offsets = inputs([100, 3, 250], 256, 192, torch.bfloat16, "kn")
    op = layer(3, 256, 192, max_rows=400)
    first = (op.forward(x, w, offsets), *op.backward(x, dy, w, offsets, dw_dtype=torch.float32))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        second = (op.forward(x, w, offsets), *op.backward(x, dy, w, offsets, dw_dtype=torch.float32))
    torch.cuda.current_stream().wait_stream(side)
    for a, b in zip(first, second):
        assert torch.equal(a, b)


def test_in_a_graph():
    for counts in ([100, 0, 250], [1, 0, 2]):
        x, dy, w, offsets = inputs(counts, 512, 192, torch.bfloat16, "nk")
        op = layer(3, 512, 192, max_rows=400, layout="nk")
        y, dx = torch.empty_like(dy), torch.empty_like(x)
        dw = torch.empty(op.w_shape, device="cuda")
        op.forward(x, w, offsets, out=y)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            op.forward(x, w, offsets, out=y)
            op.input_grad(dy, w, offsets, out=dx)
            op.weight_grad(x, dy, offsets, out=dw)
        for i in range(4):
            x.mul_(-0.5)
            y.zero_(), dx.zero_(), dw.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(y, op.forward(x, w, offsets)) and torch.equal(dx, op.input_grad(dy, w, offsets))
            assert torch.equal(dw, op.weight_grad(x, dy, offsets, out_dtype=torch.float32))


def test_refusals_of_the_python_class():
    op = layer(2, 64, 32, max_rows=16)
    x, dy, w, offsets = inputs([8, 8], 64, 32, torch.bfloat16, "kn")
    for bad in (lambda: op.forward(x.float(), w, offsets), lambda: op.forward(x[:, :32], w, offsets), lambda: op.forward(x, w[:1], offsets),
                lambda: op.forward(x.cpu(), w, offsets), lambda: op.forward(x.T.contiguous().T, w, offsets),
                lambda: op.forward(x, w, offsets.long()), lambda: op.forward(x, w, offsets[:2]), lambda: op.weight_grad(x, dy[:8], offsets),
                lambda: op.weight_grad(x, dy, offsets, accumulate=True), lambda: op.forward(x, w, offsets, out=dy[:8]),
                lambda: op.weight_grad(x, dy, offsets, out=w, accumulate=True), lambda: layer(2, 64, 32, dtype=torch.float32)):
        with pytest.raises(ValueError):
            bad()
    from paper_2104_06069_amd import ObLambError
    with pytest.raises(ObLambError):
        op.forward(torch.cat([x, x]), w, offsets)      # more rows than max_rows


@pytest.mark.parametrize("counts,k,n", [([3000, 10, 0, 2000], 64, 64), ([5000, 1], 128, 200), ([1, 4000, 700], 72, 70), ([2000], 33, 129)])
@pytest.mark.parametrize("layout", ("kn", "nk"))
def test_weight_gradients_of_few_tiles_and_many_rows(counts, k, n, layout):
    """Several workgroups share the rows of a tile."""
    x, dy, w, offsets = inputs(counts, k, n, torch.bfloat16, layout)
    op = layer(len(counts), k, n, max_rows=x.shape[0], layout=layout)
    mark = torch.full(op.w_shape, 77.0, device="cuda")
    dw = op.weight_grad(x, dy, offsets, out=mark)
    low = op.weight_grad(x, dy, offsets)
    start = torch.randn(op.w_shape, device="cuda")
    assert torch.equal(op.weight_grad(x, dy, offsets, out=start.clone(), accumulate=True), start + dw)
    assert torch.equal(low, dw.to(torch.bfloat16))
    assert torch.equal(op.weight_grad(x, dy, offsets, out_dtype=torch.float32), dw)
    ends, xd, dyd = offsets.tolist(), x.double().cpu(), dy.double().cpu()
    dwc = dw.cpu() if layout == "kn" else dw.cpu().transpose(1, 2)
    for g, (a, b) in enumerate(zip(ends[:-1], ends[1:])):
        near(dwc[g], xd[a:b].T @ dyd[a:b], xd[a:b].T.abs() @ dyd[a:b].abs(), b - a, f"dw of group {g}")


def test_tables_that_are_none_at_any_row_count():
    """Overlapping and reversed ranges in each kernel: nothing is read or written out of bounds (the results are not defined)."""
    for rows, k, n in ((24, 64, 64), (600, 128, 136), (9000, 256, 512)):
        x, dy, w, _ = inputs([rows], k, n, torch.bfloat16, "kn")
        w = w.expand(4, k, n).contiguous()
        op = layer(4, k, n, max_rows=rows)
        for table in ([0, rows, 0, rows, 0], [rows, 0, rows, 5, 1], [-9, -3, rows + 7, rows, 1 << 30], [0, rows, rows, rows, rows]):
            offsets = torch.tensor(table, dtype=torch.int32, device="cuda")
            op.forward(x, w, offsets)
            op.backward(x, dy, w, offsets)
    torch.cuda.synchronize()


@pytest.mark.parametrize("counts,k,n", [([16384 - 300, 300], 64, 1024), ([4000, 2000, 96, 4000], 96, 2048), ([20000], 40, 520)])
def test_last_round_of_large_tiles(counts, k, n):
    """More tiles than the card has CUs, so that those of the last round are split."""
    check(counts, k, n, torch.bfloat16, "kn")


@pytest.mark.parametrize("rows,k,ld", [(270_000, 8200, 8200), (700, 64, (1 << 22) - 8), (700, 64, (1 << 22) - 5)])
def test_rows_beyond_32_bits(rows, k, ld):
    """The last group's rows lie more than 2^31 elements behind the first ones."""
    n, last = 24, 40
    assert (rows - last) * ld > 2 ** 31
    gen = torch.Generator(device="cuda").manual_seed(3)
    def wide():
        return torch.empty(rows, ld, dtype=torch.bfloat16, device="cuda")[:, :k]
    x, dx = wide(), wide()
    x.normal_(generator=gen)
    dy = torch.randn(rows, n, generator=gen, device="cuda", dtype=torch.bfloat16)
    w = torch.randn(2, k, n, generator=gen, device="cuda", dtype=torch.bfloat16)
    offsets = torch.tensor([0, rows - last, rows], dtype=torch.int32, device="cuda")
    op = layer(2, k, n, max_rows=rows)
    y, dw = op.forward(x, w, offsets), op.weight_grad(x, dy, offsets)
    op.input_grad(dy, w, offsets, out=dx)
    for a, b, g in ((0, last, 0), (rows - 2 * last, rows - last, 0), (rows - last, rows, 1)):      # (first rows, last of group 0, group 1)
        xd, dyd, wd = x[a:b].double().cpu(), dy[a:b].double().cpu(), w[g].double().cpu()
        near(y[a:b], xd @ wd, xd.abs() @ wd.abs(), k, f"y from row {a}")
        near(dx[a:b], dyd @ wd.T, dyd.abs() @ wd.T.abs(), n, f"dx from row {a}")
    near(dw[1], xd.T @ dyd, xd.T.abs() @ dyd.abs(), last, "dw of the last group")
    op.close()
