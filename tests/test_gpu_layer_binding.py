"""The binding's own calls of a layer's operators (include/ob_layer.h), for programs that keep their buffers themselves: bit by bit what the objects'
methods give, on the default stream and on another."""
import pytest

torch = pytest.importorskip("torch")
from paper_2104_06069_amd import binding as ob  # noqa: E402

pytestmark = pytest.mark.gpu
BF, E4M3, E5M2 = torch.bfloat16, torch.float8_e4m3fn, torch.float8_e5m2


def normal(*shape, seed, dtype=torch.float32):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()


@pytest.fixture(params=("default", "other"))
def stream(request):
    if request.param == "default":
        yield None
        return
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        yield s.cuda_stream
    s.synchronize()


def test_norm(stream):
    from paper_2104_06069_amd.matrix8 import Matrix8
    from paper_2104_06069_amd.norm import RMSNorm
    rows, n = 37, 1000
    norm = RMSNorm(n)
    x, r, dy, dres = (normal(rows, n, seed=s, dtype=BF) for s in range(4))
    w = normal(n, seed=4)
    ctx = ob.ob_norm_create(n, ob.OB_BF16, ob.OB_BF16, ob.OB_F32, 1e-6)
    h, y, rstd, m = torch.empty_like(r), torch.empty_like(x), torch.empty(rows, device="cuda"), Matrix8(rows, n, E5M2, x.device)
    ob.ob_norm_forward(ctx, x, n, r, n, w, rows, h, n, y, n, *m.address(), ob.OB_E5M2, rstd, stream)
    want = torch.empty_like(x)
    m8, h8, rstd8 = norm.forward8(x, w, r, out=want, format=E5M2)
    assert torch.equal(h, h8) and torch.equal(rstd, rstd8) and torch.equal(y, want)
    assert torch.equal(m.data.view(torch.uint8), m8.data.view(torch.uint8)) and torch.equal(m.scales.view(torch.uint8), m8.scales.view(torch.uint8))
    dh, dw = torch.empty_like(h), torch.ones(n, device="cuda")
    ob.ob_norm_backward(ctx, dy, n, h, n, rstd, w, dres, n, rows, dh, n, dw, True, stream)
    dh8, dw8 = norm.backward(dy, h, rstd, w, dres)
    assert torch.equal(dh, dh8) and torch.equal(dw, 1.0 + dw8)
    assert ob.ob_norm_workspace_bytes(ctx) == ob.ob_norm_workspace_bytes(norm.ctx) > 0
    torch.cuda.synchronize()
    ob.ob_norm_destroy(ctx)


def test_linear8(stream):
    from paper_2104_06069_amd.linear8 import Linear8
    from paper_2104_06069_amd.matrix8 import Matrix8
    rows, k, n = 70, 300, 200
    layer = Linear8(k, n, grad_format=E5M2)
    x, dy, w = normal(rows, k, seed=1, dtype=BF), normal(rows, n, seed=2, dtype=BF), normal(n, k, seed=3)
    ctx = ob.ob_linear8_create(k, n, rows)
    w8, wt8 = Matrix8(n, k, E4M3, x.device, square=True), Matrix8(k, n, E4M3, x.device, square=True)
    ob.ob_linear8_quantize(ctx, w, ob.OB_F32, k, n, k, ob.OB_BLOCK_SQUARE, ob.OB_E4M3, ob.OB_E4M3, *w8.address(), *wt8.address(), stream)
    want_w = layer.quantize_weight(w)
    for got, want in ((w8, want_w.w), (wt8, want_w.transposed)):
        assert torch.equal(got.data.view(torch.uint8), want.data.view(torch.uint8)) and torch.equal(got.scales.view(torch.uint8), want.scales.view(torch.uint8))
    x8, xt8, d8, dt8 = Matrix8(rows, k, E4M3, x.device), Matrix8(k, rows, E4M3, x.device), Matrix8(rows, n, E5M2, x.device), Matrix8(n, rows, E5M2, x.device)
    ob.ob_linear8_quantize(ctx, x, ob.OB_BF16, k, rows, k, ob.OB_BLOCK_ROWS, ob.OB_E4M3, ob.OB_E4M3, *x8.address(), *xt8.address(), stream)
    ob.ob_linear8_quantize(ctx, dy, ob.OB_BF16, n, rows, n, ob.OB_BLOCK_ROWS, ob.OB_E5M2, ob.OB_E5M2, *d8.address(), *dt8.address(), stream)
    y, dx, dw = torch.empty(rows, n, device="cuda", dtype=BF), torch.empty(rows, k, device="cuda", dtype=BF), torch.ones(n, k, device="cuda")
    ob.ob_linear8_forward(ctx, *x8.address(), ob.OB_E4M3, *w8.address(), rows, y, n, ob.OB_BF16, stream)
    ob.ob_linear8_input_grad(ctx, *d8.address(), ob.OB_E5M2, *wt8.address(), rows, dx, k, ob.OB_BF16, stream)
    ob.ob_linear8_weight_grad(ctx, *dt8.address(), ob.OB_E5M2, *xt8.address(), rows, dw, k, ob.OB_F32, True, stream)
    dx8, dw8 = layer.backward(x, dy, want_w)
    assert torch.equal(y, layer.forward(x, want_w)) and torch.equal(dx, dx8) and torch.equal(dw, 1.0 + dw8)
    assert ob.ob_linear8_workspace_bytes(ctx) == ob.ob_linear8_workspace_bytes(layer.ctx) > 0
    torch.cuda.synchronize()
    ob.ob_linear8_destroy(ctx)


@pytest.mark.parametrize("sizes", ([300, 5], [9_000_000, 5]))
def test_clip(stream, sizes):
    from paper_2104_06069_amd.clip import GradClip
    offsets = [0, sizes[0], sum(sizes)]
    g = normal(offsets[-1], seed=5)
    clip, ctx = GradClip(offsets), ob.ob_clip_create(offsets)
    norm, layers, out = torch.empty(1, device="cuda"), torch.empty(2, device="cuda"), torch.empty_like(g)
    ob.ob_clip_norm_apply(ctx, g, ob.OB_F32, 0.5, norm, layers, out, ob.OB_F32, stream)
    want = g.clone()
    assert torch.equal(clip.clip(want, 0.5), norm) and torch.equal(want, out) and torch.equal(clip.layer_norms, layers)
    norm2, layers2 = torch.empty_like(norm), torch.empty_like(layers)
    ob.ob_clip_norm(ctx, g, ob.OB_F32, norm2, layers2, stream)
    ob.ob_clip_apply(ctx, g, ob.OB_F32, norm2, 0.5, g, ob.OB_F32, stream)
    assert torch.equal(norm2, norm) and torch.equal(layers2, layers) and torch.equal(g, out)
    assert ob.ob_clip_workspace_bytes(ctx) == ob.ob_clip_workspace_bytes(clip.ctx) > 0
    torch.cuda.synchronize()
    ob.ob_clip_destroy(ctx)
