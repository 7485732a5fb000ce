"""Conversions to 8-bit integers in every form of their kernels, against the definition in 64 bits: rows of all lengths with the maxima of columns beside them or apart, on
rows with NaN, infinities and signalling NaN, and groups of very different lengths."""
import math

import pytest
import torch

import i8_reference as R
import paper_2508_03984_amd as oz
from test_gpu_i8 import FILL, TYPES, ends, gen, normal, target

pytestmark = pytest.mark.gpu

# batch, rows, cols.  Maxima of columns with the rows (4, 16, 64 and 256 threads to a row, which hold 1, 2, 4 and 8 times 8 numbers) ...
TOGETHER = [(6, 10000, 15), (6, 4000, 101), (6, 700, 501), (8, 700, 1000), (6, 521, 2100), (6, 600, 6001), (6, 530, 9001)]
# ... and apart from them (4, 16 and 64 threads to the columns of a part; the last one's rows are read twice)
APART = [(1, 20000, 30), (2, 9000, 100), (1, 3000, 257), (2, 1100, 1500), (1, 700, 3000), (1, 600, 6000), (1, 600, 9001), (2, 1100, 16400)]
# Offsets and columns
UNEVEN = [4, 900, 900, 1500, 2400, 2401, 3300]
GROUPED_TOGETHER = [(UNEVEN, 9), (UNEVEN, 77), (UNEVEN, 300), (UNEVEN, 1500), (UNEVEN, 2100), (UNEVEN, 6000), (UNEVEN, 9001), ([3, 395], 700)]
GROUPED_APART = [([0, 1000, 1001, 2999], 20), ([5, 1000, 1000, 3000], 100), ([0, 1200], 2100), ([0, 10, 1500], 6001)]
GROUPED_STRIPS = [(list(range(30)) + [5030] + list(range(5031, 5071)), 40), ([0, 0, 2300] + [2300 + i for i in range(1, 70)], 1001)]


def broken(x):
    """NaN, a signalling one and infinities here and there, a row of zeros."""
    rows, cols = x.shape
    bits = {torch.float32: (torch.int32, 0x7f800001), torch.bfloat16: (torch.int16, 0x7f81), torch.float16: (torch.int16, 0x7c01)}[x.dtype]
    x[rows // 3, cols - 1] = math.inf
    x[rows // 2, cols // 2] = math.nan
    x[rows // 2 + 1, 0] = -math.inf
    x[2] = 0
    signalling = torch.full((1,), bits[1], dtype=bits[0], device=x.device).view(x.dtype)
    x[rows - 1, cols // 3] = signalling
    return x


def same(got, want):
    """Scales, NaN for NaN, to the bit."""
    return torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(got.nan_to_num(3.0), want.nan_to_num(3.0))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("batch,rows,cols", TOGETHER + APART)
def test_batches(batch, rows, cols, dtype):
    x = broken(normal(gen(rows + cols), batch * rows, cols, dtype, cols + 3, 1))
    a, qa, sa = target(batch * rows, cols)
    t, qt, st = target(batch * cols, rows)
    oz.oz2_i8_quantize(batch, rows, cols, x, cols + 3, a, t)
    want, scale = R.quantize(x)
    assert same(a.scale, scale) and torch.equal(a.q, want)
    want, scale = R.quantize(x.reshape(batch, rows, cols).mT)
    assert same(t.scale, scale.flatten()) and torch.equal(t.q, want.flatten(0, 1))
    ends(qa, batch * rows, cols, 16)
    ends(qt, batch * cols, rows, 16)
    assert (sa[:, batch * rows:] == FILL).all() and (st[:, batch * cols:] == FILL).all()
    for both, alone, args in ((a, target(batch * rows, cols)[0], (0, None)), (t, target(batch * cols, rows)[0], (None, 0))):
        oz.oz2_i8_quantize(batch, rows, cols, x, cols + 3, *(None if v is None else alone for v in args))
        assert same(alone.scale, both.scale) and torch.equal(alone.q, both.q)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("offsets,cols", GROUPED_TOGETHER + GROUPED_APART + GROUPED_STRIPS, ids=lambda v: f"{len(v) - 1}_groups_{v[-1]}" if isinstance(v, list) else str(v))
def test_groups(offsets, cols, dtype):
    rows, groups, g = offsets[-1] + 9, len(offsets) - 1, gen(cols)
    tokens = rows // 3
    x = broken(normal(g, tokens, cols, dtype, cols + 1))
    index = torch.randint(-1, tokens + 1, (rows,), device="cuda", generator=g, dtype=torch.int32)     # (one before and one behind, too)
    off = torch.tensor(offsets, dtype=torch.int32, device="cuda")
    wide = oz.oz2_i8_grouped_cols(rows, groups)
    a, qa, sa = target(rows, cols)
    t, qt, st = target(cols, wide, groups)
    oz.oz2_i8_quantize_grouped(rows, cols, x, tokens, cols + 1, index, groups, off, a, t)
    full = R.gather(x, index, rows)
    want, scale = R.quantize(full)
    lo, hi = offsets[0], offsets[-1]
    assert torch.equal(a.q[lo:hi], want[lo:hi]) and same(a.scale[lo:hi], scale[lo:hi])
    ends(qa[lo:hi], hi - lo, cols, 16)
    for part in (slice(0, lo), slice(hi, None)):
        assert (qa[part] == FILL).all() and (sa[0, part] == FILL).all()
    expect = torch.full((cols, qt.shape[1]), FILL, dtype=torch.int8, device="cuda")
    for i in range(groups):
        first, n = R.first_col(offsets, i), offsets[i + 1] - offsets[i]
        want, scale = R.quantize(full[offsets[i]:offsets[i + 1]].t())
        expect[:, first:first + (n + 127) // 128 * 128] = 0
        expect[:, first:first + n] = want
        assert same(st[i, :cols], scale), i
    assert torch.equal(qt[:cols], expect) and (qt[cols:] == FILL).all() and (st[:, cols:] == FILL).all()
    alone, _, _ = target(cols, wide, groups)
    oz.oz2_i8_quantize_grouped(rows, cols, x, tokens, cols + 1, index, groups, off, None, alone)
    assert same(alone.scale, t.scale) and torch.equal(alone.q, t.q)
