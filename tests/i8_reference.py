"""The 8-bit integer operators from their definitions, in 64 bits, with torch on any device."""
import math

import torch

PART = float.fromhex("0x1.020408p-7")                       # next to 1 / 127


def quantize(x):
    """(q, scale) of the rows of x: the scale is max|x| times the binary32 number next to 1 / 127, rounded to binary32, 2^-126 at least (the product is
    exact in binary64), q the integer next to x / scale, ties to even."""
    x = x.double()
    top = x.abs().amax(-1) if x.shape[-1] else x.new_zeros(x.shape[:-1])
    fine = torch.isfinite(x).all(-1)
    s = torch.where(fine, (top * PART).clamp(min=2.0 ** -126), torch.full_like(top, math.nan)).float()
    q = torch.round(torch.where(fine[..., None], x / s.double()[..., None], torch.zeros_like(x)))
    return q.to(torch.int8), s


def grouped_cols(rows, groups):
    return rows // 128 * 128 + 128 * groups


def first_col(offsets, g):
    return offsets[g] // 128 * 128 + 128 * g


def gather(x, index, rows):
    """Row index[r] of x, zeros where there is none."""
    if index is None:
        return x[:rows]
    index = index.long()
    there = (index >= 0) & (index < x.shape[0])
    return torch.where(there[:, None], x[torch.where(there, index, 0)], torch.zeros((), dtype=x.dtype, device=x.device))


def numbers(q, scale):
    return q.double() * scale.double()[:, None]


def product(a, b):
    """(q, scale) times (q, scale) transposed: exact but for the scales' products in binary64."""
    return (a[0].double() @ b[0].double().t()) * a[1].double()[:, None] * b[1].double()


STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}     # half a step, relative
LEAST = {torch.float32: 2.0 ** -150, torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}  # ... of the subnormal numbers


def bound(summed, want, dtype, alpha=1.0, beta=0.0, c=None):
    """How far a result of `dtype` may be from `want` = alpha * summed + beta * c.

    In binary32, each by 2^-24 of its result at most: the sum of integers as a binary32 number, its product with the one and with the other scale, that with alpha
    (exact for 1), the fused alpha * sum + beta * c.  Then the rounding to dtype.  1.01 covers the products of these errors and the 64-bit reference's."""
    u = 2.0 ** -24
    part = (3 + (alpha != 1.0)) * u * (alpha * summed).abs()
    if beta != 0.0:
        part = part + u * want.abs()
    if dtype is not torch.float32:
        part = part + STEP[dtype] * want.abs()
    return 1.01 * part + LEAST[dtype] + 2.0 ** -149


def check(got, want, limit):
    """got within limit of want; where want is beyond the type's numbers or NaN, got is the same."""
    got, over = got.double(), torch.finfo(got.dtype).max
    nan = torch.isnan(want)
    assert torch.equal(torch.isnan(got), nan), "NaN"
    far = (want.abs() > over) & ~nan
    off = torch.where(nan | far, torch.zeros_like(want), (got - want).abs())
    bad = off > limit.nan_to_num(0.0)
    assert not bad.any(), (int(bad.sum()), float(off[bad].max()), tuple(bad.nonzero()[0].tolist()), float(got[bad][0]), float(want[bad][0]))
