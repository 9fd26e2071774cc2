"""The orthogonalised update against its definition in 64 bits.

Bounds, as the 2-norm of the difference over that of the result.  precision float32: each number of a working matrix is off
by at most 2^-22 of it; what that does to a singular value near zero grows with it, at most a^5 = 485 times: 485 * 2^-22 =
1.2e-4.  precision float16: the Gram matrix and the polynomial's matrix are rounded to 2^-11 at every step, and the
polynomial's terms (3.4, 4.8, 2.0) cancel to about 0.7 of the result, on rounding errors of about half the bound:
5 steps * 2 * 2^-11 = 5e-3.  A 16-bit output adds its rounding, in the 2-norm 2^-9 or 2^-12 and a little less."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
ROUNDING = {torch.bfloat16: 2.0 ** -9, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
BOUND = {torch.float32: 1.2e-4, torch.float16: 5e-3}
QUINTIC = (3.4445, -4.7750, 2.0315)


def muon(*args, **kw):
    from paper_2104_06069_amd.muon import MuonStep
    return MuonStep(*args, **kw)


def definition(G, steps=5, coefficients=QUINTIC, eps=1e-7):
    G = G.double().cpu()
    X = G.T if G.shape[0] > G.shape[1] else G
    X = X / (X.norm() + eps)
    for k in range(steps):
        a, b, c = coefficients[3 * min(k, len(coefficients) // 3 - 1):][:3]
        S = X @ X.T
        X = a * X + (b * S + c * S @ S) @ X
    return X.T if G.shape[0] > G.shape[1] else X


def layout(shapes):
    sizes = [max(r, 1) * c for r, c in shapes]
    return np.concatenate([[0], np.cumsum(sizes)]).astype(np.int64), [r for r, _ in shapes]


def matrix(kind, r, c, gen):
    if kind == "low_rank":
        k = max(1, min(r, c) // 16)
        return torch.randn(r, k, generator=gen) @ torch.randn(k, c, generator=gen) + 0.01 * torch.randn(r, c, generator=gen)
    g = torch.randn(r, c, generator=gen)
    if kind == "student_t3":
        g = g / torch.randn(3, r, c, generator=gen).square().mean(0).sqrt()
    return g


def flat_of(shapes, kind="normal", seed=0, scale=1.0):
    gen = torch.Generator().manual_seed(seed)
    return torch.cat([scale * matrix(kind, max(r, 1), c, gen).reshape(-1) for r, c in shapes])


def off(got, want):
    return ((got.double().cpu() - want).norm() / want.norm()).item()


LISTS = {
    "odd": [(65, 63), (0, 3), (200, 130), (0, 1), (1, 1), (1, 40), (40, 1), (0, 5), (7, 9), (64, 64), (130, 333)],
    "one_wide": [(96, 1000)],
    "one_tall": [(0, 1), (1000, 96)],
    "block": [(128, 128), (0, 128), (128, 128), (128, 512), (0, 512), (512, 128)],
}


@pytest.mark.parametrize("precision", (torch.float32, torch.float16))
@pytest.mark.parametrize("kind", ("normal", "student_t3", "low_rank"))
@pytest.mark.parametrize("name", LISTS)
def test_orthogonalize(name, kind, precision):
    shapes = LISTS[name]
    offsets, rows = layout(shapes)
    src = flat_of(shapes, kind, scale=1e-3)
    opt = muon(offsets, rows, precision=precision, own_state=False)
    out = opt.orthogonalize(src.cuda(), torch.full((len(src),), 7.0, device="cuda"))
    for (r, c), a, b in zip(shapes, offsets[:-1], offsets[1:]):
        if r:
            assert off(out[a:b].view(r, c), definition(src[a:b].view(r, c))) <= BOUND[precision], (r, c)
        else:
            assert (out[a:b] == 7.0).all()
    opt.close()


@pytest.mark.parametrize("shape", [(600, 600), (300, 1100), (1030, 520), (257, 255)])
@pytest.mark.parametrize("precision", (torch.float32, torch.float16))
def test_larger_matrices(shape, precision):
    offsets, rows = layout([shape, (0, 7), shape])
    src = flat_of([shape, (0, 7), shape], seed=2)
    out = muon(offsets, rows, precision=precision, own_state=False).orthogonalize(src.cuda())
    for a, b in ((offsets[0], offsets[1]), (offsets[2], offsets[3])):
        assert off(out[a:b].view(shape), definition(src[a:b].view(shape))) <= BOUND[precision]


@pytest.mark.parametrize("src_dtype", (torch.float32, torch.float16, torch.bfloat16))
@pytest.mark.parametrize("out_dtype", (torch.float32, torch.float16, torch.bfloat16))
def test_types(src_dtype, out_dtype):
    shapes = [(0, 3), (70, 90), (90, 71)]
    offsets, rows = layout(shapes)
    src = flat_of(shapes, seed=5).to(src_dtype)
    out = muon(offsets, rows, own_state=False).orthogonalize(src.cuda(), out_dtype=out_dtype)
    for (r, c), a, b in list(zip(shapes, offsets[:-1], offsets[1:]))[1:]:
        assert off(out[a:b].view(r, c), definition(src[a:b].view(r, c))) <= BOUND[torch.float32] + ROUNDING[out_dtype]


@pytest.mark.parametrize("steps,coefficients", [(1, QUINTIC), (3, (3.4445, -4.7750, 2.0315, 2.0, -1.5, 0.5)), (10, (1.5, -0.5, 0.0)),
                                                (4, (1.5, -0.5, 0.0) + QUINTIC), (6, (1.875, -1.25, 0.375))])
@pytest.mark.parametrize("precision", (torch.float32, torch.float16))
def test_coefficients(steps, coefficients, precision):
    shapes = [(100, 130), (90, 64)]
    offsets, rows = layout(shapes)
    src = flat_of(shapes, seed=8)
    out = muon(offsets, rows, precision=precision, steps=steps, coefficients=coefficients, own_state=False).orthogonalize(src.cuda())
    for (r, c), a, b in zip(shapes, offsets[:-1], offsets[1:]):
        assert off(out[a:b].view(r, c), definition(src[a:b].view(r, c), steps, coefficients)) <= BOUND[precision] * max(1, steps / 5)


@pytest.mark.parametrize("coefficients", [(1.5, -0.5, 1e-6), (1.4, -0.45, 0.05), (0.5, 0.3, 0.2), (1.2, 0.1, -0.3)])
@pytest.mark.parametrize("shapes", ([(60, 64), (64, 30)], [(100, 130), (90, 64)], [(300, 1100), (257, 255)]))
@pytest.mark.parametrize("precision", (torch.float32, torch.float16))
def test_vertex_of_the_polynomial_anywhere(precision, shapes, coefficients):
    """-b / 2c far beyond the singular values' squares, close behind them, and below zero.  The bounds as above: with a shift
    within [0, 2] every rounded term stays below 1.5."""
    offsets, rows = layout(shapes)
    src = flat_of(shapes, seed=9)
    out = muon(offsets, rows, precision=precision, coefficients=coefficients, own_state=False).orthogonalize(src.cuda())
    for (r, c), a, b in zip(shapes, offsets[:-1], offsets[1:]):
        assert off(out[a:b].view(r, c), definition(src[a:b].view(r, c), 5, coefficients)) <= BOUND[precision], (r, c)


def test_singular_values_and_vectors():
    """On a diagonal matrix every singular value becomes what the scalar polynomial makes of it, small ones as well."""
    s = 10.0 ** -np.linspace(0.0, 3.0, 50)
    G = torch.zeros(50, 80)
    G[torch.arange(50), torch.arange(50)] = torch.from_numpy(s).float()
    out = muon([0, 4000], [50], own_state=False).orthogonalize(G.reshape(-1).cuda()).view(50, 80).cpu().double()
    v = G.double().diagonal() / (G.double().norm() + 1e-7)
    for _ in range(5):
        v = 3.4445 * v - 4.7750 * v ** 3 + 2.0315 * v ** 5
    assert ((out.diagonal() - v).abs() <= 1.2e-4 * v.abs() + 1e-6).all()
    out[torch.arange(50), torch.arange(50)] = 0
    assert out.abs().max() <= 1e-6


@pytest.mark.parametrize("scale", (1e-30, 1e-9, 1e12, 1e30))
def test_range_of_the_input(scale):
    offsets, rows = layout([(40, 60)])
    src = flat_of([(40, 60)], scale=scale)
    out = muon(offsets, rows, eps=0.0, own_state=False).orthogonalize(src.cuda())
    assert off(out.view(40, 60), definition(src.view(40, 60), eps=0.0)) <= BOUND[torch.float32]


def test_zeros_infinities_and_nans_stay_in_their_matrix():
    shapes = [(70, 40), (30, 30), (64, 200), (50, 50)]
    offsets, rows = layout(shapes)
    src = flat_of(shapes)
    clean = muon(offsets, rows, own_state=False).orthogonalize(src.cuda())
    src[offsets[0]:offsets[1]] = 0
    src[offsets[1] + 5] = float("inf")
    src[offsets[3] + 7] = float("nan")
    out = muon(offsets, rows, own_state=False).orthogonalize(src.cuda())
    assert (out[:offsets[1]] == 0).all()
    assert torch.isnan(out[offsets[1]:offsets[2]]).any() and torch.isnan(out[offsets[3]:]).any()
    assert torch.equal(out[offsets[2]:offsets[3]], clean[offsets[2]:offsets[3]])


@pytest.mark.parametrize("nesterov", (True, False))
@pytest.mark.parametrize("grad_dtype,x_lp", [(torch.float32, None), (torch.float16, torch.float16), (torch.bfloat16, torch.bfloat16)])
def test_step(grad_dtype, x_lp, nesterov):
    shapes = LISTS["odd"]
    offsets, rows = layout(shapes)
    N, f = int(offsets[-1]), np.float32
    x, m = flat_of(shapes, seed=1, scale=0.02), flat_of(shapes, seed=2, scale=1e-3)
    scale, lr, wd, beta = (1.0 if grad_dtype == torch.float32 else 1 / 64), 3e-3, 0.1, 0.9
    opt = muon(offsets, rows, momentum=beta, weight_decay=wd, nesterov=nesterov, grad_scale=scale, x_lp_dtype=x_lp)
    opt.load_state(dict(x=x, m=m))
    for t in range(2):
        g = (flat_of(shapes, seed=10 + t, scale=1e-3) / scale).to(grad_dtype)
        before = opt.t["x"].clone()
        opt.step(g.cuda(), lr)
        gs = g.float() * f(scale)
        b, omb = float(f(beta)), float(f(1) - f(beta))
        for (r, c), i, j in zip(shapes, offsets[:-1], offsets[1:]):
            if not r:
                assert torch.equal(opt.t["m"][i:j].cpu(), m[i:j]) and torch.equal(opt.t["x"][i:j].cpu(), x[i:j])
                continue
            m[i:j] = b * m[i:j] + omb * gs[i:j]
            u = b * m[i:j] + omb * gs[i:j] if nesterov else m[i:j]
            assert torch.equal(opt.t["m"][i:j].cpu(), m[i:j])
            moved = opt.t["x"][i:j].double().cpu() - before[i:j].double().cpu() * (1 - lr * wd)
            want = -lr * 0.2 * max(r, c) ** 0.5 * definition(u.view(r, c)).reshape(-1)
            # (x is rounded three times, once in its product with 1 - lr wd, which is itself rounded)
            slack = 4 * 2.0 ** -24 * before[i:j].double().cpu().norm().item()
            assert (moved - want).norm() <= BOUND[torch.float32] * want.norm() + slack
            if x_lp is not None:
                assert torch.equal(opt.x_lp[i:j], opt.t["x"][i:j].to(x_lp))
    opt.close()


def test_step_on_a_momentum_formed_elsewhere():
    shapes = LISTS["block"]
    offsets, rows = layout(shapes)
    x, m = flat_of(shapes, seed=1, scale=0.02), flat_of(shapes, seed=2, scale=1e-3)
    opt = muon(offsets, rows, weight_decay=0.0, layer_scale=[2.0] * len(rows))
    opt.load_state(dict(x=x, m=m))
    opt.step(None, 0.25)
    assert torch.equal(opt.t["m"].cpu(), m)
    for (r, c), i, j in zip(shapes, offsets[:-1], offsets[1:]):
        want = x[i:j].double() - (0.5 * definition(m[i:j].view(r, c)).reshape(-1) if r else 0.0)
        assert off(opt.t["x"][i:j], want) <= BOUND[torch.float32]


def test_momentum_from_the_1_bit_exchange():
    """compress_local and server_reduce leave the global momentum in 1-bit form; its dense view is orthogonalised."""
    import paper_2104_06069_amd as ob
    from paper_2104_06069_amd.step import DeviceStep
    shapes = LISTS["block"]
    offsets, rows = layout(shapes)
    N = int(offsets[-1])
    ds = DeviceStep(offsets, 1, 0, packed_momentum=True, fused_apply=True, beta1=0.9, beta2=0.999, beta3=0.9, eta=1e-6, c_min=0.01,
                    c_max=0.3, r_min=0.5, r_max=4.0, r_threshold=0.1, weight_decay=0.0)
    g = torch.zeros(ds.n_pad, device="cuda")
    g[:N] = flat_of(shapes, seed=3, scale=1e-3).cuda()
    ds.begin_step()
    ds.compress_local(g)
    ds.server_reduce()
    opt = muon(offsets, rows, own_state=False)
    opt.t["x"], opt.t["m"] = ds.t["x"][:N], torch.empty(ds.n_pad, device="cuda")
    state = ob.make_state(**dict(ds.t, m=None, m_packed=ds.packed_all, m_scales=ds.server_scales))
    ob.ob_lamb_momentum_dense(ds.ctx, state, opt.t["m"], ds.stream)
    signs = torch.where(opt.t["m"][:N] > 0, 1.0, -1.0)
    assert torch.equal(signs, torch.where(0.1 * g[:N] >= 0, 1.0, -1.0))
    opt.step(None, 1e-2)
    for (r, c), i, j in zip(shapes, offsets[:-1], offsets[1:]):
        if r:
            want = -1e-2 * 0.2 * max(r, c) ** 0.5 * definition(opt.t["m"][i:j].view(r, c)).reshape(-1)
            assert off(opt.t["x"][i:j], want) <= BOUND[torch.float32]


def test_twice_the_same_on_another_stream_and_in_a_graph():
    shapes = LISTS["odd"] + [(300, 280)]
    offsets, rows = layout(shapes)
    for precision in (torch.float32, torch.float16):
        opt = muon(offsets, rows, precision=precision, own_state=False)
        src = flat_of(shapes).cuda()
        first = opt.orthogonalize(src)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            second = opt.orthogonalize(src)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(first, second)
        out = torch.zeros_like(src)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            opt.orthogonalize(src, out)
        for i in range(4):
            src.add_(torch.randn_like(src))
            out.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, opt.orthogonalize(src))


def test_refusals_of_the_python_class():
    from paper_2104_06069_amd import ObLambError
    opt = muon([0, 12], [3])
    g = torch.zeros(12, device="cuda")
    for bad in (lambda: opt.step(g[:11], 1.0), lambda: opt.step(g.double(), 1.0), lambda: opt.step(g.cpu(), 1.0),
                lambda: opt.orthogonalize(g, torch.zeros(24, device="cuda")[::2]),
                lambda: muon([0, 12], [3], own_state=False).step(g, 1.0)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: opt.step(g, float("nan")), lambda: muon([0, 12], [5]), lambda: muon([0, 12], [0]), lambda: muon([0, 12], [3], steps=0),
                lambda: muon([0, 12], [3], momentum=1.0), lambda: muon([0, 12], [3], coefficients=(1.0, 2.0)),
                lambda: muon([0, 12], [3, 4]), lambda: muon([0, 12], [3], precision=torch.bfloat16)):
        with pytest.raises(ObLambError):
            bad()


SMALL = [(64, 64), (0, 3), (63, 200), (512, 33), (1, 1), (1, 511), (9, 7), (0, 1), (64, 512), (20, 64), (130, 17)]


@pytest.mark.parametrize("precision", (torch.float32, torch.float16))
@pytest.mark.parametrize("kind", ("normal", "student_t3", "low_rank"))
def test_lists_of_small_matrices(kind, precision):
    """Lists whose matrices all have a side of at most 64 and one of at most 512 take a kernel of their own."""
    offsets, rows = layout(SMALL)
    src = flat_of(SMALL, kind, seed=4, scale=1e-3)
    for coefficients, steps in ((QUINTIC, 5), ((1.5, -0.5, 0.0) + QUINTIC, 3)):
        out = muon(offsets, rows, precision=precision, coefficients=coefficients, steps=steps,
                   own_state=False).orthogonalize(src.cuda(), torch.full((len(src),), 7.0, device="cuda"))
        for (r, c), a, b in zip(SMALL, offsets[:-1], offsets[1:]):
            if r:
                assert off(out[a:b].view(r, c), definition(src[a:b].view(r, c), steps, coefficients)) <= BOUND[torch.float32], (r, c)
            else:
                assert (out[a:b] == 7.0).all()


@pytest.mark.parametrize("nesterov", (True, False))
@pytest.mark.parametrize("grad_dtype,x_lp", [(torch.float32, None), (torch.float16, torch.float16), (torch.bfloat16, torch.bfloat16)])
def test_step_of_small_matrices(grad_dtype, x_lp, nesterov):
    offsets, rows = layout(SMALL)
    f = np.float32
    x, m = flat_of(SMALL, seed=1, scale=0.02), flat_of(SMALL, seed=2, scale=1e-3)
    scale, lr, wd, beta = (1.0 if grad_dtype == torch.float32 else 1 / 64), 3e-3, 0.1, 0.9
    opt = muon(offsets, rows, momentum=beta, weight_decay=wd, nesterov=nesterov, grad_scale=scale, x_lp_dtype=x_lp)
    opt.load_state(dict(x=x, m=m))
    for t in range(2):
        g = (flat_of(SMALL, seed=10 + t, scale=1e-3) / scale).to(grad_dtype)
        before = opt.t["x"].clone()
        opt.step(g.cuda(), lr)
        gs, b, omb = g.float() * f(scale), float(f(beta)), float(f(1) - f(beta))
        for (r, c), i, j in zip(SMALL, offsets[:-1], offsets[1:]):
            if not r:
                assert torch.equal(opt.t["m"][i:j].cpu(), m[i:j]) and torch.equal(opt.t["x"][i:j].cpu(), x[i:j])
                continue
            m[i:j] = b * m[i:j] + omb * gs[i:j]
            u = b * m[i:j] + omb * gs[i:j] if nesterov else m[i:j]
            assert torch.equal(opt.t["m"][i:j].cpu(), m[i:j])
            moved = opt.t["x"][i:j].double().cpu() - before[i:j].double().cpu() * (1 - lr * wd)
            want = -lr * 0.2 * max(r, c) ** 0.5 * definition(u.view(r, c)).reshape(-1)
            slack = 4 * 2.0 ** -24 * before[i:j].double().cpu().norm().item()
            assert (moved - want).norm() <= BOUND[torch.float32] * want.norm() + slack
            if x_lp is not None:
                assert torch.equal(opt.x_lp[i:j], opt.t["x"][i:j].to(x_lp))


def test_small_matrices_with_zeros_infinities_and_nans():
    offsets, rows = layout(SMALL)
    src = flat_of(SMALL)
    opt = muon(offsets, rows, own_state=False)
    clean = opt.orthogonalize(src.cuda())
    src[offsets[0]:offsets[1]] = 0
    src[offsets[2] + 5] = float("inf")
    src[offsets[6] + 7] = float("nan")
    out = opt.orthogonalize(src.cuda())
    assert (out[:offsets[1]] == 0).all()
    assert torch.isnan(out[offsets[2]:offsets[3]]).any() and torch.isnan(out[offsets[6]:offsets[7]]).any()
    for l in (3, 4, 5, 8, 9, 10):
        assert torch.equal(out[offsets[l]:offsets[l + 1]], clean[offsets[l]:offsets[l + 1]])


def test_groups_of_steps_that_follow_one_gram_matrix():
    """More steps than one Gram matrix serves, on matrices large enough that following it pays: 12 steps are groups of three."""
    shapes = [(512, 2048), (2048, 512)]
    offsets, rows = layout(shapes)
    src = flat_of(shapes * 1, "low_rank", seed=6)
    coefficients = QUINTIC * 4 + (1.875, -1.25, 0.375)
    opt = muon(offsets, rows, steps=12, coefficients=coefficients, own_state=False)
    out = opt.orthogonalize(src.cuda())
    for (r, c), a, b in zip(shapes, offsets[:-1], offsets[1:]):
        assert off(out[a:b].view(r, c), definition(src[a:b].view(r, c).cuda().cpu(), 12, coefficients)) <= 12 / 5 * BOUND[torch.float32]


@pytest.mark.parametrize("precision", (torch.float32, torch.float16))
def test_wide_and_square_matrices_in_one_list(precision):
    """Enough of the wide ones that they take a way of their own in precision float16."""
    shapes = [(1024, 1024), (0, 9), (1024, 4096), (4096, 1024), (1000, 1024)]
    offsets, rows = layout(shapes)
    src = flat_of(shapes, seed=9).cuda()
    out = muon(offsets, rows, precision=precision, own_state=False).orthogonalize(src)
    for (r, c), a, b in zip(shapes, offsets[:-1], offsets[1:]):
        if r:
            G = src[a:b].view(r, c).double()
            X = G.T if r > c else G
            X = X / (X.norm() + 1e-7)
            for _ in range(5):
                S = X @ X.T.contiguous()
                X = QUINTIC[0] * X + (QUINTIC[1] * S + QUINTIC[2] * S @ S) @ X
            want = (X.T if r > c else X).cpu()
            assert off(out[a:b].view(r, c), want) <= BOUND[precision]


@pytest.mark.parametrize("shape", [(60, 70), (200, 130)])
def test_matrices_beyond_32_bits(shape):
    """The second matrix begins more than 2^32 elements into the list."""
    gap, size = 2 ** 32 + 5, shape[0] * shape[1]
    offsets, rows = np.array([0, size, size + gap, 2 * size + gap], dtype=np.int64), [shape[0], 0, shape[0]]
    src = torch.zeros(2 * size + gap, dtype=torch.bfloat16, device="cuda")
    want = []
    for seed, a in ((11, 0), (12, size + gap)):
        part = flat_of([shape], seed=seed).to(torch.bfloat16)
        src[a:a + size] = part.cuda()
        want.append(definition(part.view(shape)))
    opt = muon(offsets, rows, own_state=False)
    out = opt.orthogonalize(src, torch.zeros_like(src))
    assert off(out[:size].view(shape), want[0]) <= BOUND[torch.float32] + ROUNDING[torch.bfloat16]
    assert off(out[size + gap:].view(shape), want[1]) <= BOUND[torch.float32] + ROUNDING[torch.bfloat16]
    assert not out[size:size + gap].any()
    opt.close()
