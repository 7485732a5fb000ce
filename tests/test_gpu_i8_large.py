"""Products in 8-bit integers by large tiles: whole and partial ones, groups that end anywhere, short groups among long ones."""
import math

import pytest
import torch

import i8_reference as R
import paper_2508_03984_amd as oz
from test_gpu_i8 import TYPES, gen, operand, output, outside_kept

pytestmark = pytest.mark.gpu


PRODUCTS = [(2048, 2048, 384), (2049, 2305, 385), (4095, 1030, 1000), (2300, 2060, 513), (1111, 4099, 640), (2048, 2050, 2047), (9000, 300, 500), (257, 16400, 700),
            (4300, 4400, 400), (4097, 4097, 515), (2048, 2048, 2048), (1024, 4099, 3333), (1536, 1000, 40000), (1537, 1001, 39999), (3000, 3100, 3001), (3841, 4093, 1920)]


def f32(x):
    return torch.tensor(x).double().item()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n,k", PRODUCTS)
def test_product(m, n, k, dtype):
    g = gen(m + n + k)
    a, b = operand(g, m, k), operand(g, n, k)
    a.scale[m // 2], b.scale[n - 1] = math.nan, math.nan
    summed = R.product((a.q, a.scale), (b.q, b.scale))
    for alpha, beta in ((1.0, 0.0), (0.37, 0.0), (-1.5, 0.75)):
        if dtype is torch.float16:
            alpha *= 2.0 ** -16
        c, buf, before = output(g, m, n, dtype)
        old = c.double()
        if beta == 0.0:
            c.fill_(math.nan)
        oz.oz2_i8_gemm(m, n, k, alpha, a, b, beta, c, c.stride(0))
        want = f32(alpha) * summed + beta * old
        R.check(c, want, R.bound(summed, want, dtype, alpha, beta))
        again = c.clone()
        if beta == 0.0:
            oz.oz2_i8_gemm(m, n, k, alpha, a, b, beta, c, c.stride(0))
            assert torch.equal(again.nan_to_num(3.0), c.nan_to_num(3.0))
        outside_kept(c, buf, before)


LONG = [[0, 256, 512, 2048], [5, 300, 301, 301, 1400, 2000, 2900], [0, 1, 2, 3, 5000], [0, 0, 0, 777, 777, 4000, 4001], [100, 2700], [0, 255, 511, 768, 1024 + 1, 1300, 2100, 2400, 2500]]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("offsets", LONG, ids=lambda o: f"{len(o) - 1}_groups_{o[-1]}")
@pytest.mark.parametrize("n,k", [(2048, 384), (1111, 1000), (2300, 513), (5000, 640), (7000, 400)])
def test_grouped(offsets, n, k, dtype):
    rows, groups, g = offsets[-1] + 7, len(offsets) - 1, gen(n + k)
    a, b = operand(g, rows, k), operand(g, groups * n, k)
    off = torch.tensor(offsets, dtype=torch.int32, device="cuda")
    for alpha, beta in ((1.0, 0.0), (0.37, 1.0)):
        if dtype is torch.float16:
            alpha *= 2.0 ** -16
        c, buf, before = output(g, rows, n, dtype)
        old = c.double()
        oz.oz2_i8_grouped_gemm(rows, n, k, groups, off, alpha, a, b, beta, c, c.stride(0))
        for i in range(groups):
            lo, hi = offsets[i], offsets[i + 1]
            if lo == hi:
                continue
            summed = R.product((a.q[lo:hi], a.scale[lo:hi]), (b.q[i * n:(i + 1) * n], b.scale[i * n:(i + 1) * n]))
            want = f32(alpha) * summed + beta * old[lo:hi]
            R.check(c[lo:hi], want, R.bound(summed, want, dtype, alpha, beta))
        assert torch.equal(c[:offsets[0]].double(), old[:offsets[0]]) and torch.equal(c[offsets[-1]:].double(), old[offsets[-1]:])
        outside_kept(c, buf, before)


SUMS = [(o, m, n) for o in LONG for m, n in ((1024, 2048), (1111, 1300), (257, 5000))]
SUMS += [([0, 100, 3000, 3256, 6000], 2304, 4099), ([7, 7, 5000, 5001, 9000], 2305, 2305), ([0, 257, 514, 4000, 4000, 4004], 4097, 2305), ([3, 2000, 2048], 4100, 4100)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("offsets,m,n", SUMS, ids=lambda o: f"{len(o) - 1}_groups_{o[-1]}" if isinstance(o, list) else str(o))
def test_grouped_grad(offsets, m, n, dtype):
    rows, groups, g = offsets[-1] + 7, len(offsets) - 1, gen(n + m)
    off = torch.tensor(offsets, dtype=torch.int32, device="cuda")
    wide = oz.oz2_i8_grouped_cols(rows, groups)
    a, b = operand(g, m, wide, groups), operand(g, n, wide, groups)
    for i in range(groups):
        first, count = R.first_col(offsets, i), offsets[i + 1] - offsets[i]
        for x in (a, b):
            x.q[:, first + count:first + (count + 127) // 128 * 128] = 0
    for alpha, beta in ((1.0, 0.0), (0.37, 1.0)):
        if dtype is torch.float16:
            alpha *= 2.0 ** -16
        c, buf, before = output(g, groups * m, n, dtype)
        old = c.double()
        oz.oz2_i8_grouped_grad(m, n, rows, groups, off, alpha, a, b, beta, c, c.stride(0))
        for i in range(groups):
            part = slice(R.first_col(offsets, i), R.first_col(offsets, i) + offsets[i + 1] - offsets[i])
            scale = (a.scale, b.scale) if groups == 1 else (a.scale[i], b.scale[i])
            summed = R.product((a.q[:, part], scale[0]), (b.q[:, part], scale[1]))
            want = f32(alpha) * summed + beta * old[i * m:(i + 1) * m]
            R.check(c[i * m:(i + 1) * m], want, R.bound(summed, want, dtype, alpha, beta))
        outside_kept(c, buf, before)
