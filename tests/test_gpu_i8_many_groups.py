"""Products by large tiles of more groups than a wavefront has lanes, with empty and short ones on both sides of the 64th, against the definition in 64 bits."""
import pytest
import torch

import i8_reference as R
import paper_2508_03984_amd as oz
from test_gpu_i8 import gen, operand, output, outside_kept

pytestmark = pytest.mark.gpu


def lengths(groups, mean):
    """Rows of the groups: about `mean`, some none, some one, some a few; the 63rd to 66th (from 0) and the last are of each kind in turn."""
    of = [mean + (37 * g) % 101 - 50 for g in range(groups)]
    for g in range(5, groups, 11):
        of[g] = (0, 1, 255, 256, 257)[g % 5]
    for g, n in ((62, 0), (63, 300), (64, 0), (65, 259), (66, 1)):
        if g < groups:
            of[g] = n
    return of


def offsets_of(groups, mean):
    off = [3]
    for n in lengths(groups, mean):
        off.append(off[-1] + n)
    return off


# groups, mean of their rows, n, k: by rows
ROWS = [(64, 200, 1030, 400), (65, 200, 1030, 400), (66, 210, 2048, 385), (128, 200, 1030, 400), (130, 230, 1030, 513), (1024, 180, 1030, 384)]
# groups, mean, m, n: over rows
SUMS = [(64, 960, 1024, 1024), (65, 960, 1024, 1024), (66, 960, 1100, 1000), (128, 960, 512, 700), (130, 960, 1024, 1024)]


@pytest.mark.parametrize("groups,mean,n,k", ROWS)
def test_rows(groups, mean, n, k):
    offsets = offsets_of(groups, mean)
    rows, g = offsets[-1] + 7, gen(groups)
    a, b = operand(g, rows, k), operand(g, groups * n, k)
    off = torch.tensor(offsets, dtype=torch.int32, device="cuda")
    for alpha, beta, dtype in ((1.0, 0.0, torch.bfloat16), (0.25, 1.0, torch.float32)):
        c, buf, before = output(g, rows, n, dtype)
        old = c.double()
        oz.oz2_i8_grouped_gemm(rows, n, k, groups, off, alpha, a, b, beta, c, c.stride(0))
        for i in range(groups) if groups <= 130 else list(range(0, groups, 17)) + [62, 63, 64, 65, 66, 1023]:
            lo, hi = offsets[i], offsets[i + 1]
            if lo < hi:
                summed = R.product((a.q[lo:hi], a.scale[lo:hi]), (b.q[i * n:(i + 1) * n], b.scale[i * n:(i + 1) * n]))
                want = alpha * summed + beta * old[lo:hi]
                R.check(c[lo:hi], want, R.bound(summed, want, dtype, alpha, beta))
        assert torch.equal(c[:offsets[0]].double(), old[:offsets[0]]) and torch.equal(c[offsets[-1]:].double(), old[offsets[-1]:])
        outside_kept(c, buf, before)


@pytest.mark.parametrize("groups,mean,m,n", SUMS)
def test_sums(groups, mean, m, n):
    offsets = offsets_of(groups, mean)
    rows, g = offsets[-1] + 7, gen(groups)
    off = torch.tensor(offsets, dtype=torch.int32, device="cuda")
    wide = oz.oz2_i8_grouped_cols(rows, groups)
    a, b = operand(g, m, wide, groups), operand(g, n, wide, groups)
    for i in range(groups):
        first, count = R.first_col(offsets, i), offsets[i + 1] - offsets[i]
        for x in (a, b):
            x.q[:, first + count:first + (count + 127) // 128 * 128] = 0
    for alpha, beta, dtype in ((1.0, 0.0, torch.bfloat16), (0.25, 1.0, torch.float32)):
        c, buf, before = output(g, groups * m, n, dtype)
        oz.oz2_i8_grouped_grad(m, n, rows, groups, off, alpha, a, b, beta, c, c.stride(0))
        for i in range(groups):
            part = slice(R.first_col(offsets, i), R.first_col(offsets, i) + offsets[i + 1] - offsets[i])
            mine = slice(i * m, (i + 1) * m)
            old = before[1 + i * m:1 + (i + 1) * m, 3:n + 3].double()
            summed = R.product((a.q[:, part], a.scale[i]), (b.q[:, part], b.scale[i]))
            want = alpha * summed + beta * old
            R.check(c[mine], want, R.bound(summed, want, dtype, alpha, beta))
        outside_kept(c, buf, before)
