"""Matrices of 8-bit numbers with a scale for each block of 128 (include/ob_layer.h), as RMSNorm.forward8 and Linear8 make and read
them, and what the operators of a layer share of argument checks."""
import torch

from . import binding as ob

FORMATS = {torch.float8_e4m3fn: ob.OB_E4M3, torch.float8_e5m2: ob.OB_E5M2}


def adjacent(t):
    """Whether each row's elements follow each other and no row overlaps the next.  Of a single row only the distance to the next one
    is free."""
    rows, width = t.shape
    return rows == 0 or ((width < 2 or t.stride(1) == 1) and (rows < 2 or t.stride(0) >= width))


def rows_of(t, width, dtypes, device, what):
    """The distance between the rows of t [rows, width], once it is looked at."""
    if t.dim() != 2 or t.shape[1] != width or t.dtype not in dtypes or t.device != device:
        raise ValueError(f"{what}: a [rows, {width}] tensor of {' or '.join(map(str, dtypes))} on {device}, not {tuple(t.shape)} of {t.dtype} on {t.device}")
    if not adjacent(t):
        raise ValueError(f"{what}: rows of adjacent elements that do not overlap")
    return t.stride(0) if t.shape[0] > 1 else max(width, 1)


def format_of(dtype):
    if dtype not in FORMATS:
        raise ValueError(f"a format of 8 bits is torch.float8_e4m3fn or torch.float8_e5m2, not {dtype}")
    return FORMATS[dtype]


class Matrix8:
    """A matrix [rows, cols] in 8 bits.  `data` [rows, cols] holds the numbers, `scales` [rows, blocks of 128 columns] (`square`:
    [blocks of 128 rows, blocks of 128 columns]) the powers of two that they are multiplied by.  Both are views: the calls rely on the
    bytes between the rows, which are zeros, so that a matrix is made by them and not from tensors."""
    __slots__ = ("buffer", "rows", "cols", "dtype", "square", "ld", "ld_scales", "device")

    def __init__(self, rows, cols, dtype, device, square=False):
        self.rows, self.cols, self.dtype, self.square, self.device = rows, cols, dtype, square, device
        blocks = cols + 127 >> 7
        self.ld, self.ld_scales = blocks << 7, blocks + 3 & ~3
        self.buffer = torch.empty(rows * self.ld + (rows + 127 >> 7 if square else rows) * self.ld_scales, dtype=torch.uint8, device=device)

    @property
    def data(self):
        return self.buffer.view(self.dtype).as_strided((self.rows, self.cols), (self.ld, 1))

    @property
    def scales(self):
        high = (self.rows + 127) // 128 if self.square else self.rows
        return self.buffer.view(torch.float8_e8m0fnu).as_strided((high, (self.cols + 127) // 128), (self.ld_scales, 1), self.rows * self.ld)

    def address(self):
        """-> (address of the numbers, distance between rows, address of the scales, distance between theirs)"""
        at = self.buffer.data_ptr()
        return at, self.ld, at + self.rows * self.ld, self.ld_scales
