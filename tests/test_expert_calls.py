"""What ExpertLinear hands to the library's calls, without a device: the calls are stood in for by ones that read and write the same
addresses on the host."""
import ctypes

import pytest

torch = pytest.importorskip("torch")


def at(address, rows, width, ld, dtype):
    """[rows, width] elements from an address on, rows ld elements apart."""
    count = (rows - 1) * ld + width if rows and width else 0
    size = torch.empty(0, dtype=dtype).element_size()
    flat = torch.frombuffer((ctypes.c_char * max(count * size, 1)).from_address(address), dtype=dtype, count=count) if count else torch.empty(0, dtype=dtype)
    return flat.as_strided((rows, width), (ld, 1)) if count else flat.view(rows, width)


@pytest.fixture
def host_layer(monkeypatch):
    """-> a function that makes an ExpertLinear whose products run on the host."""
    from paper_2104_06069_amd import binding as ob
    from paper_2104_06069_amd import experts
    types = {v: k for k, v in experts._OB_DTYPE.items()}
    layers = {}

    def groups_of(layer, offsets, rows):
        ends = at(offsets, 1, layer.groups + 1, layer.groups + 1, torch.int32)[0].clamp(0, rows).tolist()
        return enumerate(zip(ends[:-1], ends[1:]))

    def weights(layer, address, dtype):
        _, r, c = layer.w_shape
        flat = at(address, 1, (layer.groups - 1) * layer.w_stride + r * c, 1, dtype)[0]
        return flat.as_strided(layer.w_shape, (layer.w_stride, c, 1))

    def rows_call(transposed):
        def call(ctx, a, lda, w, offsets, rows, out, ldo, out_dtype, stream):
            layer = layers[ctx]
            depth, width = (layer.n, layer.k) if transposed else (layer.k, layer.n)
            x, y, wv = at(a, rows, depth, lda, layer.dtype), at(out, rows, width, ldo, types[out_dtype]), weights(layer, w, layer.dtype)
            for g, (lo, hi) in groups_of(layer, offsets, rows):
                m = wv[g] if layer.layout == "kn" else wv[g].T
                y[lo:hi] = (x[lo:hi].double() @ (m.T if transposed else m).double()).to(y.dtype)
            return 0
        return call

    def weight_grad(ctx, x, ldx, dy, lddy, offsets, rows, dw, dw_dtype, accumulate=False, stream=None):
        layer = layers[ctx]
        xv, dv = at(x.data_ptr(), rows, layer.k, ldx, layer.dtype), at(dy.data_ptr(), rows, layer.n, lddy, layer.dtype)
        out = weights(layer, dw.data_ptr(), types[dw_dtype])
        for g, (lo, hi) in groups_of(layer, offsets.data_ptr(), rows):
            p = xv[lo:hi].double().T @ dv[lo:hi].double()
            p = p if layer.layout == "kn" else p.T
            out[g] = (out[g].double() + p if accumulate else p).to(out.dtype)

    class Lib:
        ob_experts_forward, ob_experts_input_grad = staticmethod(rows_call(False)), staticmethod(rows_call(True))

    def create(*args):
        return len(layers) + 1
    monkeypatch.setattr(ob, "lib", lambda: Lib)
    monkeypatch.setattr(ob, "ob_experts_create", create)
    monkeypatch.setattr(ob, "ob_experts_destroy", lambda ctx: None)
    monkeypatch.setattr(ob, "ob_experts_weight_grad", weight_grad)
    monkeypatch.setattr(experts, "_current_stream", lambda device: 0)
    monkeypatch.setattr(torch.cuda, "set_device", lambda device: None)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: -1)       # (a host tensor's get_device())
    monkeypatch.setattr(torch.cuda, "synchronize", lambda device=None: None)

    def make(groups, k, n, **kw):
        layer = experts.ExpertLinear(groups, k, n, device="cpu", **kw)
        layers[layer.ctx] = layer
        return layer
    return make


def whole(*shape, seed=0, dtype=torch.bfloat16):
    """Small whole numbers: every sum is exact."""
    return torch.randint(-3, 4, shape, generator=torch.Generator().manual_seed(seed)).to(dtype)


def table(*ends):
    return torch.tensor(ends, dtype=torch.int32)


def test_the_stand_in_computes_the_products(host_layer):
    for layout in ("kn", "nk"):
        op = host_layer(2, 8, 4, layout=layout)
        x, dy, w = whole(5, 8), whole(5, 4, seed=1), whole(*op.w_shape, seed=2)
        m = w if layout == "kn" else w.transpose(1, 2)
        y, (dx, dw) = op.forward(x, w, table(0, 2, 5)), op.backward(x, dy, w, table(0, 2, 5), dw_dtype=torch.float32)
        for g, (a, b) in enumerate(((0, 2), (2, 5))):
            assert torch.equal(y[a:b].float(), x[a:b].float() @ m[g].float()) and torch.equal(dx[a:b].float(), dy[a:b].float() @ m[g].float().T)
            p = x[a:b].float().T @ dy[a:b].float()
            assert torch.equal(dw[g], p if layout == "kn" else p.T)


def test_one_row_of_elements_that_are_not_adjacent_is_refused(host_layer):
    """Of one row only the distance to the next one is free, not the distance between its elements."""
    op = host_layer(1, 8, 4)
    x, dy, w, offsets = whole(1, 8), whole(1, 4, seed=1), whole(1, 8, 4, seed=2), table(0, 1)
    apart = {n: (whole(n, 3, seed=3).T[:1], whole(1, 2 * n, seed=4)[:, ::2], whole(1, 1, seed=5).expand(1, n)) for n in (8, 4)}
    for bad in apart[8]:
        for call in (lambda: op.forward(bad, w, offsets), lambda: op.weight_grad(bad, dy, offsets), lambda: op.input_grad(dy, w, offsets, out=bad)):
            with pytest.raises(ValueError):
                call()
    for bad in apart[4]:
        for call in (lambda: op.input_grad(bad, w, offsets), lambda: op.weight_grad(x, bad, offsets), lambda: op.forward(x, w, offsets, out=bad)):
            with pytest.raises(ValueError):
                call()
    # a row of a wider matrix is one of adjacent elements, and so is a single element
    wide = whole(3, 20, seed=6)[1:2, 5:13]
    assert torch.equal(op.forward(wide, w, offsets), op.forward(wide.clone(), w, offsets))
    one = host_layer(1, 1, 4)
    column = whole(3, 5, seed=7)[1:2, 2:3]
    assert torch.equal(one.forward(column, w[:, :1].contiguous(), offsets), (column.float() * w[0, :1].float()).to(torch.bfloat16))


@pytest.mark.parametrize("rows", (1, 2))
def test_a_gradient_that_is_one_number(host_layer, rows):
    """The gradient of a sum has one element in memory, whatever its shape."""
    op = host_layer(1, 8, 4)
    x, w = whole(rows, 8).requires_grad_(), whole(1, 8, 4, seed=2).requires_grad_()
    op(x, w, table(0, rows)).sum().backward()
    assert torch.equal(x.grad.float(), w[0].detach().float().sum(1).expand(rows, 8))
    assert torch.equal(w.grad[0].float(), x.detach().float().sum(0)[:, None].expand(8, 4))


@pytest.fixture
def marked_memory():
    """Memory that nobody has written yet holds NaNs."""
    torch.use_deterministic_algorithms(True)
    assert torch.utils.deterministic.fill_uninitialized_memory and torch.isnan(torch.empty(1)).all()
    yield
    torch.use_deterministic_algorithms(False)


def test_rows_of_no_expert_through_autograd(host_layer, marked_memory):
    """They have no product and no gradient: zeros, not what the allocator left."""
    op = host_layer(2, 8, 4)
    x, w = whole(9, 8).requires_grad_(), whole(2, 8, 4, seed=2).requires_grad_()
    y = op(x, w, table(2, 4, 6))
    inside = torch.zeros(9, dtype=torch.bool)
    inside[2:6] = True
    assert (y[~inside] == 0).all() and torch.isfinite(y).all()
    y.backward(whole(9, 4, seed=3))
    assert (x.grad[~inside] == 0).all() and torch.equal(x.grad[2:4].float(), whole(9, 4, seed=3)[2:4].float() @ w[0].detach().float().T)
    assert torch.equal(w.grad[1].float(), x.detach()[4:6].float().T @ whole(9, 4, seed=3)[4:6].float())


def test_second_derivatives_are_refused(host_layer):
    """The gradients are kernels' results that autograd knows nothing about: asking for theirs is an error, not a missing term."""
    op = host_layer(1, 8, 4)
    x, w = whole(3, 8).requires_grad_(), whole(1, 8, 4, seed=2).requires_grad_()
    loss = op(x, w, table(0, 3)).float().square().sum()
    dx, = torch.autograd.grad(loss, x, create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        (loss + dx.float().square().sum()).backward()


def test_autograd_with_other_tensors_between_the_weights(host_layer):
    """w_stride beyond k * n, as in a flat list where something lies between one expert's weights and the next one's."""
    op = host_layer(2, 8, 4, w_stride=40)
    flat = whole(80, seed=2).requires_grad_()
    view = flat.as_strided((2, 8, 4), (40, 4, 1), 5)
    x, dy = whole(5, 8).requires_grad_(), whole(5, 4, seed=3)
    op(x, view, table(0, 2, 5)).backward(dy)
    want = torch.zeros(80)
    for g, (a, b) in enumerate(((0, 2), (2, 5))):
        assert torch.equal(x.grad[a:b].float(), dy[a:b].float() @ view[g].detach().float().T)
        want[5 + 40 * g:5 + 40 * g + 32] = (x.detach()[a:b].float().T @ dy[a:b].float()).reshape(-1)
    assert torch.equal(flat.grad.float(), want)
