"""Every kind of tile of the matrix operators, at sizes whose last tiles are ragged, against the definition in 64 bits.
tests/test_matrix_plan.py checks, by the library's own rules, that the lists below reach every one of them.

Bounds.  Experts: as in tests/test_gpu_experts.py, depth 2^-23 of the products' magnitudes, and one rounding of the result.
Orthogonalised update, in the 2-norm over the matrix: precision float16 as in tests/test_gpu_muon.py, 5e-3.  precision float32 on
matrices of normal numbers with 30 rows and columns or more: a number of a working matrix is off by at most 2^-22 of it.  Such
errors spread over all singular directions alike, and a matrix of normal numbers has few with a singular value far below the
others', where they grow: each of 5 steps' three products (S, the polynomial, X) adds at most 3 * 2^-22 (the polynomial's
coefficients, up to 4.8, times singular values up to 1.2, next to a result of about 1, and less where they cancel): 1.1e-5."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
QUINTIC = (3.4445, -4.7750, 2.0315)
NORMAL, HALF = 15 * 3 * 2.0 ** -22, 5e-3
ROUNDING = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}

# groups, rows, k, n, aligned (sizes that are multiples of 8)
EXPERTS = [
    (2, 150, 72, 72, True), (16, 150, 72, 520, True), (2, 5001, 200, 200, True), (16, 5001, 520, 520, True), (16, 2999, 2056, 2056, True),
    (2, 150, 71, 71, False), (16, 150, 71, 2055, False), (2, 2999, 71, 1030, False), (16, 5001, 71, 521, False), (6, 3001, 1030, 1311, False),
]
# matrices (count, m, n), every second one lying the other way, and whether in 22 bits
LISTS = [
    ([(1, 100, 100)], True), ([(1, 100, 100)], False), ([(16, 330, 330)], True), ([(16, 330, 330)], False),
    ([(24, 570, 570)], True), ([(24, 570, 570)], False), ([(16, 650, 650)], True), ([(24, 330, 1100)], False), ([(24, 800, 800)], True), ([(24, 800, 800)], False),
    ([(1, 200, 705)], True), ([(6, 200, 705)], True), ([(16, 340, 830)], True), ([(24, 450, 1090)], True), ([(24, 570, 1090)], True), ([(24, 840, 1470)], True),
    ([(12, 840, 1590), (20, 840, 830)], True), ([(6, 840, 2700), (3, 840, 830)], False),
]
# lists whose wide and square matrices go through the steps apart
APART = LISTS[-2:]


def counts_of(groups, rows):
    """An uneven router's; one group has nothing to do, one a single row."""
    rng = np.random.default_rng(groups + rows)
    p = np.exp(rng.standard_normal(groups))
    if groups > 2:
        p[1] = 0.0
    c = rng.multinomial(rows - 1, p / p.sum())
    c[groups // 2] += 1
    return c.tolist()


def near(got, want, size, depth, what):
    err = (got.double() - want).abs()
    bound = depth * 2.0 ** -23 * size + ROUNDING[got.dtype] * want.abs() + (2.0 ** -25 if got.dtype == torch.float16 else 0.0)
    worst = (err - bound).max().item() if err.numel() else 0.0
    assert worst <= 0.0, f"{what}: {err.max().item():.3g} off, {worst:.3g} over its bound"


@pytest.mark.parametrize("case", EXPERTS)
@pytest.mark.parametrize("dtype", (torch.bfloat16, torch.float16))
@pytest.mark.parametrize("layout", ("kn", "nk"))
def test_experts(case, layout, dtype):
    from paper_2104_06069_amd.experts import ExpertLinear
    groups, rows, k, n, _ = case
    gen = torch.Generator(device="cuda").manual_seed(rows + n)
    normal = lambda *s: torch.randn(*s, generator=gen, device="cuda").to(dtype)  # noqa: E731
    op = ExpertLinear(groups, k, n, dtype=dtype, max_rows=rows, layout=layout)
    x, dy, w = normal(rows, k), normal(rows, n), normal(*op.w_shape)
    ends = np.concatenate([[0], np.cumsum(counts_of(groups, rows))])
    offsets = torch.tensor(ends, dtype=torch.int32, device="cuda")
    y, (dx, dw) = op.forward(x, w, offsets), op.backward(x, dy, w, offsets, dw_dtype=torch.float32)
    low = op.weight_grad(x, dy, offsets)
    start = torch.randn(op.w_shape, generator=gen, device="cuda")
    assert torch.equal(op.weight_grad(x, dy, offsets, out=start.clone(), accumulate=True), start + dw)
    assert torch.equal(low, dw.to(dtype))
    for g, (a, b) in enumerate(zip(ends[:-1].tolist(), ends[1:].tolist())):
        m = w[g].double() if layout == "kn" else w[g].double().T.contiguous()
        xg, dg, p = x[a:b].double(), dy[a:b].double(), dw[g] if layout == "kn" else dw[g].T
        near(y[a:b], xg @ m, xg.abs() @ m.abs(), k, f"y of group {g}")
        near(dx[a:b], dg @ m.T, dg.abs() @ m.abs().T, n, f"dx of group {g}")
        near(p, xg.T @ dg, xg.abs().T @ dg.abs(), b - a, f"dw of group {g}")
    op.close()


def shapes_of(list_):
    """With vectors of odd sizes between them."""
    shapes = []
    for count, m, n in list_:
        for i in range(count):
            shapes += [(n, m) if i % 2 else (m, n), (0, 2 * i + 1)]
    return shapes


def layout_of(shapes):
    sizes = [max(r, 1) * c for r, c in shapes]
    return np.concatenate([[0], np.cumsum(sizes)]).astype(np.int64), [r for r, _ in shapes]


def definition(G, steps=5):
    G = G.double()
    X = G.T.contiguous() if G.shape[0] > G.shape[1] else G
    X = X / (X.norm() + 1e-7)
    for _ in range(steps):
        S = X @ X.T.contiguous()
        X = QUINTIC[0] * X + (QUINTIC[1] * S + QUINTIC[2] * S @ S) @ X
    return X.T if G.shape[0] > G.shape[1] else X


def matrices(shapes, offsets, flat):
    return [(flat[a:b].view(r, c), a, b) for (r, c), a, b in zip(shapes, offsets[:-1].tolist(), offsets[1:].tolist()) if r]


@pytest.mark.parametrize("list_,fine", LISTS)
def test_orthogonalize(list_, fine):
    from paper_2104_06069_amd.muon import MuonStep
    shapes = shapes_of(list_)
    offsets, rows = layout_of(shapes)
    src = torch.randn(int(offsets[-1]), generator=torch.Generator(device="cuda").manual_seed(len(shapes)), device="cuda")
    opt = MuonStep(offsets, rows, precision=torch.float32 if fine else torch.float16, own_state=False)
    out = opt.orthogonalize(src, torch.full_like(src, 7.0))
    for G, a, b in matrices(shapes, offsets, src):
        want = definition(G)
        off = ((out[a:b].view(G.shape).double() - want).norm() / want.norm()).item()
        assert off <= (NORMAL if fine else HALF), (tuple(G.shape), a, off)
    for (r, _), a, b in zip(shapes, offsets[:-1], offsets[1:]):
        assert r or (out[a:b] == 7.0).all()
    opt.close()


@pytest.mark.parametrize("list_,fine", LISTS)
def test_step(list_, fine):
    """The last product ends in the update: each kind of tile, and matrices lying either way."""
    from paper_2104_06069_amd.muon import MuonStep
    shapes = shapes_of(list_)
    offsets, rows = layout_of(shapes)
    gen = torch.Generator(device="cuda").manual_seed(3)
    x, m, g = (torch.randn(int(offsets[-1]), generator=gen, device="cuda") * s for s in (0.02, 1e-3, 1e-3))
    opt = MuonStep(offsets, rows, momentum=0.9, weight_decay=0.1, precision=torch.float32 if fine else torch.float16, x_lp_dtype=torch.bfloat16)
    opt.load_state(dict(x=x, m=m))
    opt.step(g, 3e-3)
    beta, lr = np.float32(0.9), 3e-3
    new = m * float(beta) + g * float(1 - beta)
    for G, a, b in matrices(shapes, offsets, g):
        r, c = G.shape
        assert torch.equal(opt.t["m"][a:b], new[a:b])
        u = float(beta) * new[a:b].view(r, c).double() + float(1 - beta) * G.double()
        want = -lr * 0.2 * max(r, c) ** 0.5 * definition(u)
        moved = (opt.t["x"][a:b].double() - x[a:b].double() * (1 - lr * 0.1)).view(r, c)
        slack = 4 * 2.0 ** -24 * x[a:b].double().norm().item()      # (x is rounded three times)
        assert (moved - want).norm() <= (NORMAL if fine else HALF) * want.norm() + slack, (r, c)
        assert torch.equal(opt.x_lp[a:b], opt.t["x"][a:b].to(torch.bfloat16))
    for (r, _), a, b in zip(shapes, offsets[:-1].tolist(), offsets[1:].tolist()):
        assert r or (torch.equal(opt.t["x"][a:b], x[a:b]) and torch.equal(opt.t["m"][a:b], m[a:b]))
    opt.close()


@pytest.mark.parametrize("list_,fine", APART)
def test_low_rank_in_lists_whose_matrices_go_apart(list_, fine):
    """A sixteenth of the rank and 1% of noise: the small singular values have most to lose where one S serves several steps.  Bound in 22 bits
    as in tests/test_gpu_muon.py, 485 * 2^-22."""
    from paper_2104_06069_amd.muon import MuonStep
    shapes = shapes_of(list_)
    offsets, rows = layout_of(shapes)
    gen = torch.Generator(device="cuda").manual_seed(6)
    src = torch.zeros(int(offsets[-1]), device="cuda")
    for G, _, _ in matrices(shapes, offsets, src):
        r, c = G.shape
        k = min(r, c) // 16
        G.copy_(torch.randn(r, k, generator=gen, device="cuda") @ torch.randn(k, c, generator=gen, device="cuda") + 0.01 * torch.randn(r, c, generator=gen, device="cuda"))
    out = MuonStep(offsets, rows, precision=torch.float32 if fine else torch.float16, own_state=False).orthogonalize(src)
    for G, a, b in matrices(shapes, offsets, src):
        want = definition(G)
        assert (out[a:b].view(G.shape).double() - want).norm() <= (1.2e-4 if fine else HALF) * want.norm()


SMALL = [(64, 64), (0, 3), (63, 200), (512, 33), (64, 512), (30, 40), (40, 30)]


@pytest.mark.parametrize("shapes", [SMALL, [(128, 128), (0, 5), (128, 512), (512, 128), (65, 90)]])
def test_small_lists_of_normal_numbers(shapes):
    from paper_2104_06069_amd.muon import MuonStep
    offsets, rows = layout_of(shapes)
    src = torch.randn(int(offsets[-1]), generator=torch.Generator(device="cuda").manual_seed(8), device="cuda")
    out = MuonStep(offsets, rows, own_state=False).orthogonalize(src)
    for G, a, b in matrices(shapes, offsets, src):
        want = definition(G)
        assert (out[a:b].view(G.shape).double() - want).norm() <= NORMAL * want.norm(), tuple(G.shape)
