"""What the tests of a layer's operators share: 8-bit matrices from their definition, on the host in 64 bits."""
import torch

HALF = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}      # a rounding's largest relative error
LOWEST = {torch.bfloat16: 0.0, torch.float16: 2.0 ** -25, torch.float32: 0.0}                  # and below the normal numbers (bfloat16's and binary32's are not met)
E4M3, E5M2 = torch.float8_e4m3fn, torch.float8_e5m2
LARGEST = {E4M3: 448.0, E5M2: 57344.0}


def scales_of(most, fmt):
    """The smallest powers of two, from 2^-126 on, by which `most` is no more than the format's largest number; NaN for what is not finite."""
    most = most.double()
    s = torch.full_like(most, 2.0 ** -126)
    m, e = torch.frexp(torch.where(most.isfinite(), most, torch.ones_like(most)) / LARGEST[fmt])     # m 2^e, m from 1/2 up to 1
    s = torch.maximum(s, torch.pow(torch.tensor(2.0, dtype=torch.float64), (e - (m == 0.5).int()).double()))
    s[most == 0] = 2.0 ** -126
    s[~most.isfinite()] = float("nan")
    return s


def blocks_of(t, square=False):
    """Largest magnitude of each block (a NaN's block: NaN), [rows or blocks of them, blocks]"""
    a = torch.nn.functional.pad(t.double().abs(), (0, -t.shape[1] % 128, 0, -t.shape[0] % 128 if square else 0))
    a = a.view(a.shape[0] // 128, 128, -1, 128).amax((1, 3)) if square else a.view(a.shape[0], -1, 128).amax(2)
    return a


def spread(scales, shape, square=False):
    s = scales.repeat_interleave(128, 1)[:, :shape[1]]
    return s.repeat_interleave(128, 0)[:shape[0]] if square else s


def quantized(t, fmt, square=False):
    """-> (numbers as float64, scales as float64) of a host tensor"""
    scales = scales_of(blocks_of(t, square), fmt)
    q = (t.double() / spread(scales, t.shape, square)).float().to(fmt).double()      # (the quotient is a binary32 number, or far below the format's)
    return q, scales


def values(m):
    """A Matrix8's values, in 64 bits on the host"""
    return m.data.cpu().double() * spread(m.scales.cpu().double(), (m.rows, m.cols), m.square)


def padding_is_zero(m):
    rest = m.buffer[:m.rows * m.ld].view(m.rows, m.ld)[:, m.cols:]
    return bool((rest == 0).all())


def within(got, want, bound, what):
    got = got.double().cpu()
    assert got.shape == want.shape, what
    nan = want.isnan()
    assert torch.equal(got.isnan(), nan), f"{what}: NaNs elsewhere"
    err = (got - want).abs()
    same = got == want      # (infinities)
    worst = torch.where(nan | same, torch.zeros_like(err), err - bound)
    assert not worst.numel() or worst.max().item() <= 0.0, f"{what}: {err[~nan].max().item():.3g} off, {worst.max().item():.3g} over its bound"
