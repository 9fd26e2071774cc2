"""Ranges of the orthogonalised update's input.  Bound as in tests/test_gpu_muon.py: 485 * 2^-22 in the 2-norm over the matrix."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
BOUND = 1.2e-4
QUINTIC = (3.4445, -4.7750, 2.0315)


def muon(*args, **kw):
    from paper_2104_06069_amd.muon import MuonStep
    return MuonStep(*args, **kw)


def definition(G, eps, steps=5):
    """In 64 bits, with m <= n."""
    X = G.double() / (G.double().norm() + eps)
    for _ in range(steps):
        S = X @ X.T.contiguous()
        X = QUINTIC[0] * X + (QUINTIC[1] * S + QUINTIC[2] * S @ S) @ X
    return X


def normal(*shape, seed=0):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed))


@pytest.mark.parametrize("shape", [(40, 60), (100, 130), (520, 700)])
@pytest.mark.parametrize("scale", (1e-40, 1e-37, 1e-35, 3e37))
def test_norms_whose_inverse_is_no_binary32_number(shape, scale):
    """With eps = 0 every matrix but that of zeros has its direction.  (At 1e-40 the input's own numbers have 16 bits: the
    definition is that of the rounded ones.)"""
    src = (normal(*shape) * scale).float()
    assert torch.isfinite(src).all()
    out = muon([0, src.numel()], [shape[0]], eps=0.0, own_state=False).orthogonalize(src.reshape(-1).cuda()).view(shape).cpu()
    want = definition(src, 0.0)
    assert (out.double() - want).norm() <= BOUND * want.norm()


NORMAL = 15 * 3 * 2.0 ** -22      # of matrices of normal numbers (tests/test_gpu_matrix_tiles.py)


@pytest.mark.parametrize("shape", [(64, 200), (256, 320), (330, 1000)])
@pytest.mark.parametrize("small", (1e-4, 1e-5, 1e-6))
def test_rows_far_below_the_others(shape, small):
    """A number of a working matrix is held to 2^-22 of it, or where that is less to half of binary16's smallest number over the
    matrix's unit: 2^-33 for E and the polynomial's matrix, next to singular values of 1.  Row i of B X is off by that floor times
    |X|; E's floor reaches B times |2 c t| = |b| = 4.8, so by 6 * 2^-33 |X| a step, while a row far below the others grows by a = 3.44 a
    step, as much as |X| does at most.  In 5 steps 30 * 2^-33 over the row's share of the matrix's norm."""
    m, n = shape
    src = normal(*shape, seed=3)
    few = m // 8
    src[-few:] *= small
    out = muon([0, m * n], [m], own_state=False).orthogonalize(src.reshape(-1).cuda()).view(shape).cpu().double()
    want = definition(src, 1e-7)
    assert (out - want).norm() <= NORMAL * want.norm()
    off = (out - want).norm(dim=1) / want.norm(dim=1)
    share = src.double().norm(dim=1) / src.double().norm()
    print(f"rows {small:g} of the others, {m} x {n}: {off[-few:].max():.2g} off, the others {off[:-few].max():.2g}")
    assert (off <= NORMAL * m ** 0.5 + 30 * 2.0 ** -33 / share).all()


@pytest.mark.parametrize("shape", [(40, 60), (100, 130), (300, 520)])
@pytest.mark.parametrize("norm", (1e-9, 1.6e-12, 1e-14))
def test_norms_far_below_eps(shape, norm):
    """G / (|G| + eps) is then small as a whole: X's floor of 2^-37 an element is 2^-37 sqrt(m n) over its norm, of which later steps add
    1 / 3.44 each."""
    src = normal(*shape, seed=4)
    src *= norm / src.norm()
    out = muon([0, src.numel()], [shape[0]], own_state=False).orthogonalize(src.reshape(-1).cuda()).view(shape).cpu().double()
    want = definition(src, 1e-7)
    off = ((out - want).norm() / want.norm()).item()
    print(f"norm {norm:g} with eps 1e-7, {shape[0]} x {shape[1]}: {off:.2g} off")
    assert off <= NORMAL + 1.41 * 2.0 ** -37 * src.numel() ** 0.5 / (norm / (norm + 1e-7))
