"""Products in 8 bits on every kind of tile, of both formats, forward and both gradients, against sums in 64 bits on the device; the bounds are those
of tests/test_gpu_linear8.py."""
import pytest

torch = pytest.importorskip("torch")
from tests.layer8 import E4M3, E5M2, HALF, LOWEST, values  # noqa: E402

pytestmark = pytest.mark.gpu
BF, F16, F32 = torch.bfloat16, torch.float16, torch.float32

# Rows, depth and columns of a product (tests/test_linear8_plan.py holds them to every kind of tile): tiles of 256 that workgroups go through two
# and three or four slabs at a time, the same where results are not eights, tiles of 128 and of 64, and sums in parts
TILES = [(19999, 200, 4096), (12001, 390, 4096), (20000, 200, 523), (1001, 300, 4095), (520, 1000, 264), (511, 2000, 258), (70, 9000, 130)]


def numbers(rows, width, seed):
    """Normal numbers whose columns and rows differ in size, and a block of zeros"""
    gen = torch.Generator("cuda").manual_seed(seed)
    normal = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    t = normal(rows, width) * torch.exp(normal(width)) * torch.exp(normal(rows, 1)) / 256
    t[3:5] = 0
    return t.to(BF)


def near(results, a, b, depth):
    """results (of several types) = a b^T"""
    a, b = values(a).cuda(), values(b).cuda()
    want, size = a @ b.T.contiguous(), a.abs() @ b.abs().T.contiguous()
    for got in results:
        short, off = (0.0, 2e-6) if got.dtype == F32 else (2.0 ** -10, 1e-4)
        bound = (depth * 2.0 ** -23 + short) * size + HALF[got.dtype] * want.abs() + LOWEST[got.dtype]
        beyond = want.abs() + bound >= 65520 if got.dtype == F16 else torch.zeros_like(want, dtype=torch.bool)
        assert (((got.double() - want).abs() <= bound) | beyond).all(), got.dtype
        rest = ~beyond
        assert (got.double()[rest] - want[rest]).norm() <= (HALF[got.dtype] + off) * want[rest].norm(), got.dtype


def op(*args, **kw):
    from paper_2104_06069_amd.linear8 import Linear8
    return Linear8(*args, **kw)


@pytest.mark.parametrize("fmt", (E4M3, E5M2), ids=("e4m3", "e5m2"))
@pytest.mark.parametrize("rows,depth,cols", TILES)
def test_forward(rows, depth, cols, fmt):
    layer = op(depth, cols)
    x8, w8 = layer.quantize(numbers(rows, depth, 1), fmt), layer.quantize_weight(numbers(cols, depth, 2))
    near([layer.forward(x8, w8, out_dtype=t) for t in (BF, F16, F32)], x8, w8.w, depth)


@pytest.mark.parametrize("fmt", (E4M3, E5M2), ids=("e4m3", "e5m2"))
@pytest.mark.parametrize("rows,depth,cols", TILES)
def test_input_gradient(rows, depth, cols, fmt):
    layer = op(cols, depth, grad_format=fmt)
    dy, w8 = numbers(rows, depth, 3), layer.quantize_weight(numbers(depth, cols, 4))
    near([layer.input_grad(dy, w8, out_dtype=t) for t in (BF, F16, F32)], layer.quantize(dy, fmt), w8.transposed, depth)


@pytest.mark.parametrize("fmt", (E4M3, E5M2), ids=("e4m3", "e5m2"))
@pytest.mark.parametrize("rows,depth,cols", TILES)
def test_weight_gradient(rows, depth, cols, fmt):
    """`rows` of the weight, `depth` of x and dy: both operands have scales of rows."""
    layer = op(cols, rows, grad_format=fmt)
    x, dy = numbers(depth, cols, 5), numbers(depth, rows, 6)
    once = layer.weight_grad(x, dy)
    near([layer.weight_grad(x, dy, out_dtype=t) for t in (BF, F16)] + [once], layer._quantize(dy, "dy", rows, None, fmt)[1], layer._quantize(x, "x", cols, None, E4M3)[1],
         depth)
    start = torch.randn(rows, cols, generator=torch.Generator("cuda").manual_seed(7), device="cuda")
    assert torch.equal(layer.weight_grad(x, dy, out=start.clone(), accumulate=True), start + once)


@pytest.mark.parametrize("rows,depth,cols", [(5, 300, 80), (40, 3000, 72)] + TILES[1:6])
def test_rows_that_are_not_finite_stay_alone(rows, depth, cols):
    """An infinity or a NaN in a row of x, in its last block too, makes that row of the result NaNs and no other number different, in every type; and one in x of
    a weight gradient its column."""
    layer = op(depth, cols)
    x, w8 = numbers(rows, depth, 1), layer.quantize_weight(numbers(cols, depth, 2))
    bad = x.clone()
    at = [1, rows // 2, rows - 1]
    bad[at[0], 0], bad[at[1], depth - 1], bad[at[2], depth // 2] = float("inf"), float("nan"), -float("inf")
    rest = torch.ones(rows, dtype=torch.bool, device="cuda")
    rest[at] = False
    for t in (BF, F16, F32):
        y, z = layer.forward(x, w8, out_dtype=t), layer.forward(bad, w8, out_dtype=t)
        assert z[~rest].isnan().all() and torch.equal(z[rest], y[rest]), t
    grad = op(rows, cols)      # dw [cols, rows] from x [depth, rows]
    x, dy = numbers(depth, rows, 3), numbers(depth, cols, 4)
    bad = x.clone()
    bad[0, at[0]], bad[depth - 1, at[1]], bad[depth // 2, at[2]] = float("nan"), float("inf"), float("nan")
    for t in (BF, F32):
        y, z = grad.weight_grad(x, dy, out_dtype=t), grad.weight_grad(bad, dy, out_dtype=t)
        assert z[:, ~rest].isnan().all() and torch.equal(z[:, rest], y[:, rest]), t
