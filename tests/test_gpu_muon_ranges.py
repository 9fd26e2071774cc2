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
