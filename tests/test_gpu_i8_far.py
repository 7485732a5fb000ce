"""8-bit integer calls whose operands and results pass 2^32 bytes: rows far apart, of which some are checked."""
import pytest
import torch

import i8_reference as R
import paper_2508_03984_amd as oz
from test_gpu_i8 import gen

pytestmark = pytest.mark.gpu

ROWS, LD = 70000, 65536                                       # 4.6e9 bytes apart in the end
SAMPLE = [0, 1, 63, 32767, 32768, 65535, 65536, 65537, ROWS - 257, ROWS - 2, ROWS - 1]


@pytest.fixture(scope="module")
def memory():
    return torch.zeros(ROWS * LD, dtype=torch.int8, device="cuda")


def far(memory, g, k):
    q = memory.view(ROWS, LD)[:, :k]
    q.copy_(torch.randint(-127, 128, (ROWS, k), device="cuda", generator=g).to(torch.int8))
    return oz.I8(q, torch.rand(ROWS, device="cuda", generator=g) + 0.5)


def near(g, rows, k):
    m = oz.I8.empty(rows, k)
    m.q.copy_(torch.randint(-127, 128, (rows, k), device="cuda", generator=g).to(torch.int8))
    m.scale.copy_(torch.rand(rows, device="cuda", generator=g) + 0.5)
    return m


def part(m, rows):
    return m.q[rows], m.scale[rows]


@pytest.mark.parametrize("n,k", [(5, 300), (100, 300), (300, 520)])
def test_products(memory, n, k):
    g = gen(n)
    a, b, at = far(memory, g, k), near(g, n, k), torch.tensor(SAMPLE, device="cuda")
    big = torch.empty(ROWS, 20000, device="cuda")              # C, 5.6e9 bytes from end to end
    c = big[:, 19000:19000 + n]
    oz.oz2_i8_gemm(ROWS, n, k, 1.0, a, b, 0.0, c, big.stride(0))
    want = R.product(part(a, at), (b.q, b.scale))
    R.check(c[at], want, R.bound(want, want, torch.float32))
    turned = torch.empty(n, ROWS, device="cuda")               # the far one as B
    oz.oz2_i8_gemm(n, ROWS, k, 1.0, b, a, 0.0, turned, ROWS)
    R.check(turned[:, at].t(), want, R.bound(want, want, torch.float32))
    off = torch.tensor([0, 30000, 30000, ROWS], dtype=torch.int32, device="cuda")
    w = near(g, 3 * n, k)
    oz.oz2_i8_grouped_gemm(ROWS, n, k, 3, off, 1.0, a, w, 0.0, c, big.stride(0))
    for rows, e in (([r for r in SAMPLE if r < 30000], 0), ([r for r in SAMPLE if r >= 30000], 2)):
        at = torch.tensor(rows, device="cuda")
        want = R.product(part(a, at), (w.q[e * n:(e + 1) * n], w.scale[e * n:(e + 1) * n]))
        R.check(c[at], want, R.bound(want, want, torch.float32))


def test_experts_far_apart(memory):
    """One token for each of 70 experts of 1000 rows, and the gradient of weights whose rows are tokens, both far apart."""
    g, k, n = gen(7), 200, 1000
    b, a = far(memory, g, k), near(g, 70, k)
    off = torch.arange(71, dtype=torch.int32, device="cuda")
    c = torch.empty(70, n, device="cuda")
    oz.oz2_i8_grouped_gemm(70, n, k, 70, off, 1.0, a, b, 0.0, c, n)
    for e in (0, 1, 35, 65, 66, 69):
        want = R.product((a.q[e:e + 1], a.scale[e:e + 1]), (b.q[e * n:(e + 1) * n], b.scale[e * n:(e + 1) * n]))
        R.check(c[e:e + 1], want, R.bound(want, want, torch.float32))
    m, rows = 70000, 60000                                     # the columns of a row are tokens
    off = torch.tensor([0, 100, rows], dtype=torch.int32, device="cuda")
    wide = oz.oz2_i8_grouped_cols(rows, 2)
    assert wide <= LD
    a, b = oz.I8(memory.view(ROWS, LD)[:, :wide], torch.ones(2, m, device="cuda")), oz.I8.empty(3, wide, 2)
    a.q.zero_()
    b.q.zero_()
    b.scale.fill_(0.5)
    at = torch.tensor(SAMPLE, device="cuda")
    for lo, hi in ((0, 100), (128, 128 + rows - 100)):         # (columns of the two groups)
        a.q[at, lo:hi] = torch.randint(-127, 128, (len(SAMPLE), hi - lo), device="cuda", generator=g).to(torch.int8)
        b.q[:, lo:hi] = torch.randint(-127, 128, (3, hi - lo), device="cuda", generator=g).to(torch.int8)
    c = torch.empty(2 * m, 3, device="cuda")
    oz.oz2_i8_grouped_grad(m, 3, rows, 2, off, 1.0, a, b, 0.0, c, 3)
    for e, (lo, hi) in enumerate(((0, 100), (128, 128 + rows - 100))):
        want = R.product((a.q[at, lo:hi], a.scale[e][at]), (b.q[:, lo:hi], b.scale[e]))
        R.check(c[e * m + at], want, R.bound(want, want, torch.float32))


def test_quantize(memory):
    g, cols, ldx = gen(9), 300, 40000                          # X: 5.6e9 bytes from end to end
    big = torch.empty(ROWS, ldx, dtype=torch.bfloat16, device="cuda")
    x = big[:, 39000:39000 + cols]
    x.copy_(torch.randn(ROWS, cols, device="cuda", generator=g))
    a = oz.I8(memory.view(ROWS, LD)[:, :cols], torch.empty(ROWS, device="cuda"))
    t = oz.I8.empty(cols, ROWS)
    oz.oz2_i8_quantize(1, ROWS, cols, x, ldx, a, t)
    for m, y in ((a, x), (t, x.t())):
        want, scale = R.quantize(y)
        assert torch.equal(m.scale, scale) and torch.equal(m.q, want)
    del big
