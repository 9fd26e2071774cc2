"""ExpertLinear's calls and their autograd form on the device, where tests/test_expert_calls.py has stand-ins for the kernels.  Operands are
small whole numbers, so that every sum is exact."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def layer(*args, **kw):
    from paper_2104_06069_amd.experts import ExpertLinear
    return ExpertLinear(*args, **kw)


def whole(*shape, seed=0, dtype=torch.bfloat16):
    return torch.randint(-3, 4, shape, generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()


def table(*ends):
    return torch.tensor(ends, dtype=torch.int32).cuda()


@pytest.mark.parametrize("rows", (1, 2))
@pytest.mark.parametrize("layout", ("kn", "nk"))
def test_a_gradient_that_is_one_number(layout, rows):
    """The gradient of a sum has one element in memory, whatever its shape."""
    op = layer(1, 72, 40, max_rows=rows, layout=layout)
    x, w = whole(rows, 72).requires_grad_(), whole(*op.w_shape, seed=2).requires_grad_()
    op(x, w, table(0, rows)).sum().backward()
    m = w[0].detach() if layout == "kn" else w[0].detach().T
    assert torch.equal(x.grad.float(), m.float().sum(1).expand(rows, 72))
    dw = x.detach().float().sum(0)[:, None].expand(72, 40)
    assert torch.equal(w.grad[0].float(), dw if layout == "kn" else dw.T)


def test_one_row_of_elements_that_are_not_adjacent_is_refused():
    op = layer(1, 72, 40, max_rows=1)
    x, w, offsets = whole(72, 3, seed=3), whole(1, 72, 40, seed=2), table(0, 1)
    with pytest.raises(ValueError):
        op.forward(x.T[:1], w, offsets)
    with pytest.raises(ValueError):
        op.forward(x.T[:1].contiguous(), w, offsets, out=whole(40, 3).T[:1])
    wide = whole(3, 100, seed=6)[1:2, 5:77]
    assert torch.equal(op.forward(wide, w, offsets), op.forward(wide.clone(), w, offsets))


@pytest.fixture
def marked_memory():
    """Memory that nobody has written yet holds NaNs."""
    torch.use_deterministic_algorithms(True)
    assert torch.utils.deterministic.fill_uninitialized_memory and torch.isnan(torch.empty(1, device="cuda")).all()
    yield
    torch.use_deterministic_algorithms(False)


@pytest.mark.parametrize("rows", (9, 300))
def test_rows_of_no_expert_through_autograd(marked_memory, rows):
    """They have no product and no gradient: zeros, not what the allocator left."""
    op = layer(2, 72, 40, max_rows=rows)
    x, w, dy = whole(rows, 72).requires_grad_(), whole(2, 72, 40, seed=2).requires_grad_(), whole(rows, 40, seed=3)
    y = op(x, w, table(2, 4, rows - 3))
    inside = torch.zeros(rows, dtype=torch.bool, device="cuda")
    inside[2:rows - 3] = True
    assert (y[~inside] == 0).all() and torch.isfinite(y).all()
    y.backward(dy)
    assert (x.grad[~inside] == 0).all() and torch.isfinite(x.grad).all()
    assert torch.equal(x.grad[2:4], (dy[2:4].float() @ w[0].detach().float().T).to(torch.bfloat16))
    assert torch.equal(w.grad[1], (x.detach()[4:rows - 3].float().T @ dy[4:rows - 3].float()).to(torch.bfloat16))


def test_autograd_with_other_tensors_between_the_weights():
    """w_stride beyond k * n, as in a flat list where something lies between one expert's weights and the next one's."""
    op = layer(2, 24, 40, max_rows=50, w_stride=1000)
    flat = whole(2000, seed=2).requires_grad_()
    view = flat.as_strided((2, 24, 40), (1000, 40, 1), 5)
    x, dy = whole(50, 24).requires_grad_(), whole(50, 40, seed=3)
    op(x, view, table(0, 20, 50)).backward(dy)
    want = torch.zeros(2000, device="cuda")
    for g, (a, b) in enumerate(((0, 20), (20, 50))):
        assert torch.equal(x.grad[a:b], (dy[a:b].float() @ view[g].detach().float().T).to(torch.bfloat16))
        want[5 + 1000 * g:965 + 1000 * g] = (x.detach()[a:b].float().T @ dy[a:b].float()).reshape(-1)
    assert torch.equal(flat.grad, want.to(torch.bfloat16))


def test_second_derivatives_are_refused():
    op = layer(1, 24, 40, max_rows=3)
    x, w = whole(3, 24).requires_grad_(), whole(1, 24, 40, seed=2).requires_grad_()
    loss = op(x, w, table(0, 3)).float().square().sum()
    dx, = torch.autograd.grad(loss, x, create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        (loss + dx.float().square().sum()).backward()
