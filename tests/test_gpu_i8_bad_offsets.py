"""Grouped calls in 8-bit integers with offsets that do not ascend or leave the rows, in every form that a call takes: unspecified results, in the memory that right offsets may
have written."""
import pytest
import torch

import paper_2508_03984_amd as oz
from test_gpu_i8 import gen, operand

pytestmark = pytest.mark.gpu

GUARD = 300                                                   # rows on both sides, more than a tile has
# rows, groups, n, k: few rows, tiles of 64 x 64, of 64 x 128, large ones, of more groups than a wavefront has lanes, ranges of k
ROWS = [(9, 5, 300, 500), (700, 5, 300, 500), (3000, 5, 2048, 400), (3000, 5, 5000, 640), (14000, 70, 1030, 400), (90, 4, 64, 8192)]
# rows, groups, m, n: the same without the first
SUMS = [(700, 5, 300, 500), (2000, 2, 2048, 1000), (4000, 5, 1024, 2048), (60000, 70, 1024, 1024), (30000, 3, 100, 100)]
# rows, groups, cols: in one launch, maxima of columns with the rows, apart from them, rows that are read twice
CONVERSIONS = [(700, 5, 500), (3300, 6, 300), (3300, 6, 6000), (3300, 3, 300), (3300, 3, 20000)]


def bad_offsets(rows, groups):
    most, least = 2 ** 31 - 1, -2 ** 31
    n = groups + 1
    mixed = [rows * i // groups + (-1) ** i * (rows // 3) for i in range(n)]
    return [list(range(rows, rows - n, -1)), [rows - rows * i // groups for i in range(n)], [most] * n, [least] * n, [(0, most)[i % 2] for i in range(n)],
            [(0, rows, rows // 2, -7, rows + 9)[i % 5] for i in range(n)], mixed, [least] + [0] * (n - 2) + [most]]


def guarded(rows, cols, wide, dtype):
    """A view of rows x cols in the middle of a buffer full of 7, and a check that only rows x `wide` of it have been written."""
    buf = torch.full((rows + 2 * GUARD, (wide + 15) // 16 * 16 + 32), 7, dtype=dtype, device="cuda")

    def kept():
        return bool((buf[:GUARD] == 7).all() and (buf[GUARD + rows:] == 7).all() and (buf[:, wide:] == 7).all())
    return buf[GUARD:GUARD + rows, :cols], kept


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,groups,n,k", ROWS)
def test_rows(rows, groups, n, k, dtype):
    g = gen(rows)
    a, b = operand(g, rows, k), operand(g, groups * n, k)
    for bad in bad_offsets(rows, groups):
        off = torch.tensor(bad, dtype=torch.int32, device="cuda")
        for beta in (0.0, 1.0):
            c, kept = guarded(rows, n, n, dtype)
            oz.oz2_i8_grouped_gemm(rows, n, k, groups, off, 1.0, a, b, beta, c, c.stride(0))
            torch.cuda.synchronize()
            assert kept(), bad


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,groups,m,n", SUMS)
def test_sums(rows, groups, m, n, dtype):
    g, wide = gen(rows), oz.oz2_i8_grouped_cols(rows, groups)
    a, b = operand(g, m, wide, groups), operand(g, n, wide, groups)
    for bad in bad_offsets(rows, groups):
        off = torch.tensor(bad, dtype=torch.int32, device="cuda")
        for beta in (0.0, 1.0):
            c, kept = guarded(groups * m, n, n, dtype)
            oz.oz2_i8_grouped_grad(m, n, rows, groups, off, 1.0, a, b, beta, c, c.stride(0))
            torch.cuda.synchronize()
            assert kept(), bad


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,groups,cols", CONVERSIONS)
def test_conversions(rows, groups, cols, dtype):
    g, wide = gen(rows), oz.oz2_i8_grouped_cols(rows, groups)
    x = torch.randn(rows, cols, device="cuda", generator=g).to(dtype)
    for bad in bad_offsets(rows, groups):
        off = torch.tensor(bad, dtype=torch.int32, device="cuda")
        q, kept = guarded(rows, cols, (cols + 15) // 16 * 16, torch.int8)
        qt, kept_t = guarded(cols, wide, wide, torch.int8)
        s, st = torch.full((rows + 20,), 7.0, device="cuda"), torch.full((groups + 2, cols + 20), 7.0, device="cuda")
        oz.oz2_i8_quantize_grouped(rows, cols, x, rows, cols, None, groups, off, oz.I8(q, s[10:rows + 10]), oz.I8(qt, st[1:groups + 1, 10:cols + 10]))
        torch.cuda.synchronize()
        assert kept() and kept_t(), bad
        assert (s[:10] == 7).all() and (s[rows + 10:] == 7).all()
        assert (st[0] == 7).all() and (st[-1] == 7).all() and (st[:, :10] == 7).all() and (st[:, cols + 10:] == 7).all()
