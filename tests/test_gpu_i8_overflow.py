"""8-bit integer products whose results pass the largest number of their type, in every form of the kernels: infinities of the right sign there, and nowhere else."""
import pytest
import torch

import i8_reference as R
import paper_2508_03984_amd as oz
from test_gpu_i8 import TYPES, gen

pytestmark = pytest.mark.gpu

PRODUCTS = [(3, 200, 300), (100, 300, 777), (1024, 4096, 1024), (2100, 4100, 2000), (100, 100, 20000), (1536, 1000, 40000)]
# offsets, n, k: as in the products above, the last two in ranges of k and by large tiles
ROWS = [([2, 3, 3, 4], 70, 300), ([0, 5, 105, 300], 300, 513), ([0, 200, 1200, 2998], 2048, 400), ([3, 40, 40, 90], 64, 8192), ([5, 600, 601, 3000], 5000, 640)]
SUMS = [([3, 60, 60, 400], 70, 130), ([0, 1000, 2000], 2048, 1000), ([0, 3000, 8000], 26, 139), ([0, 1500, 1600, 1600, 2400, 4500], 1024, 2048)]


def edge(dtype):
    """Numbers of this magnitude and beyond are rounded to infinity: half a step above the largest one."""
    return {torch.float16: 2.0 ** 16 - 2.0 ** 4, torch.bfloat16: 2.0 ** 128 - 2.0 ** 119, torch.float32: 2.0 ** 128 - 2.0 ** 103}[dtype]


def check(got, summed, want, alpha=1.0, beta=0.0):
    """got is want to within its bound where the type has such a number, an infinity of want's sign beyond; within the error of the binary32 steps
    before the last rounding (R.bound) of the edge, either."""
    dtype, at = got.dtype, edge(got.dtype)
    near, limit = R.bound(summed, want, torch.float32, alpha, beta), R.bound(summed, want, dtype, alpha, beta)
    beyond, below, got = want.abs() > at + near, want.abs() < at - near, got.double()
    infinite = torch.isinf(got) & (torch.signbit(got) == torch.signbit(want))
    fine = torch.isfinite(got) & ((got - want).abs() <= limit)
    assert infinite[beyond].all() and fine[below].all() and (infinite | fine).all()


def operand(g, rows, k, scale, groups=1):
    m = oz.I8.empty(rows, k, groups)
    m.q.copy_(torch.randint(-128, 128, (rows, k), device="cuda", generator=g))
    m.scale.copy_((torch.rand(m.scale.shape, device="cuda", generator=g) + 0.5) * scale)
    return m


def scale_of(dtype, k):
    """For results whose deviation is near the edge: sums of k products of integers spread evenly over -128 .. 127 have 74^2 sqrt(k)."""
    return torch.finfo(dtype).max / (74.0 ** 2 * k ** 0.5)


def some_of_both(*parts):
    every = torch.cat([p.double().flatten() for p in parts])
    share = float(torch.isinf(every).double().mean())
    assert 0.1 < share < 0.7, share
    assert (every == float("inf")).any() and (every == -float("inf")).any()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n,k", PRODUCTS)
def test_products(m, n, k, dtype):
    g = gen(m + k)
    a, b = operand(g, m, k, 1.0), operand(g, n, k, scale_of(dtype, k))
    summed = R.product((a.q, a.scale), (b.q, b.scale))
    for beta in (0.0, 1.0):
        c = torch.randn(m, n, device="cuda", generator=g).mul_(50).to(dtype)
        old = c.double()
        oz.oz2_i8_gemm(m, n, k, 1.0, a, b, beta, c, n)
        check(c, summed, summed + beta * old, 1.0, beta)
        some_of_both(c)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("offsets,n,k", ROWS, ids=lambda v: f"to_{v[-1]}" if isinstance(v, list) else str(v))
def test_rows(offsets, n, k, dtype):
    rows, groups, g = offsets[-1] + 2, len(offsets) - 1, gen(n + k)
    a, b = operand(g, rows, k, 1.0), operand(g, groups * n, k, scale_of(dtype, k))
    off = torch.tensor(offsets, dtype=torch.int32, device="cuda")
    c = torch.zeros(rows, n, dtype=dtype, device="cuda")
    oz.oz2_i8_grouped_gemm(rows, n, k, groups, off, 1.0, a, b, 0.0, c, n)
    for i in range(groups):
        lo, hi = offsets[i], offsets[i + 1]
        summed = R.product((a.q[lo:hi], a.scale[lo:hi]), (b.q[i * n:(i + 1) * n], b.scale[i * n:(i + 1) * n]))
        check(c[lo:hi], summed, summed)
    some_of_both(c[offsets[0]:offsets[-1]])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("offsets,m,n", SUMS, ids=lambda v: f"to_{v[-1]}" if isinstance(v, list) else str(v))
def test_sums(offsets, m, n, dtype):
    rows, groups, g = offsets[-1] + 2, len(offsets) - 1, gen(m + n)
    wide = oz.oz2_i8_grouped_cols(rows, groups)
    a, b = operand(g, m, wide, 1.0, groups), operand(g, n, wide, scale_of(dtype, rows / groups), groups)
    off = torch.tensor(offsets, dtype=torch.int32, device="cuda")
    for i in range(groups):
        first, count = R.first_col(offsets, i), offsets[i + 1] - offsets[i]
        for x in (a, b):
            x.q[:, first + count:first + (count + 127) // 128 * 128] = 0
    c = torch.zeros(groups * m, n, dtype=dtype, device="cuda")
    oz.oz2_i8_grouped_grad(m, n, rows, groups, off, 1.0, a, b, 0.0, c, n)
    for i in range(groups):
        part = slice(R.first_col(offsets, i), R.first_col(offsets, i) + offsets[i + 1] - offsets[i])
        summed = R.product((a.q[:, part], a.scale[i]), (b.q[:, part], b.scale[i]))
        check(c[i * m:(i + 1) * m], summed, summed)
    some_of_both(c)
