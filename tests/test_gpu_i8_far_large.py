"""8-bit integer products by large tiles whose operands and results pass 2^32 bytes: rows far apart, of which some are checked."""
import pytest
import torch

import i8_reference as R
import paper_2508_03984_amd as oz
from test_gpu_i8 import gen
from test_gpu_i8_far import LD, ROWS, SAMPLE, far, memory, near, part  # noqa: F401

pytestmark = pytest.mark.gpu

N, K, LDC = 1024, 640, 20000                                  # of the products; C's rows are 5.6e9 bytes from end to end
M, TOKENS, LDW = 70000, 3000, 10000                           # of the gradient: two groups of tokens, results as far apart


def test_products(memory):  # noqa: F811
    g = gen(11)
    a, b, at = far(memory, g, K), near(g, N, K), torch.tensor(SAMPLE, device="cuda")
    want = R.product(part(a, at), (b.q, b.scale))
    big = torch.empty(ROWS, LDC, device="cuda")
    c = big[:, LDC - N - 3:LDC - 3]
    oz.oz2_i8_gemm(ROWS, N, K, 1.0, a, b, 0.0, c, LDC)
    R.check(c[at], want, R.bound(want, want, torch.float32))
    old = c[at].double()
    oz.oz2_i8_gemm(ROWS, N, K, 1.0, a, b, 1.0, c, LDC)         # added to C
    R.check(c[at], want + old, R.bound(want, want + old, torch.float32, 1.0, 1.0))
    turned = torch.empty(N, ROWS, device="cuda")               # the far one as B
    oz.oz2_i8_gemm(N, ROWS, K, 1.0, b, a, 0.0, turned, ROWS)
    R.check(turned[:, at].t(), want, R.bound(want, want, torch.float32))


def test_gradient(memory):  # noqa: F811
    g, off = gen(12), torch.tensor([0, 1000, TOKENS], dtype=torch.int32, device="cuda")
    wide = oz.oz2_i8_grouped_cols(TOKENS, 2)
    spans = ((0, 1000), (7 * 128 + 128, 7 * 128 + 128 + 2000))  # columns of the two groups
    a, b = oz.I8(memory.view(ROWS, LD)[:, :wide], torch.rand(2, M, device="cuda", generator=g) + 0.5), near(g, N, wide)
    b = oz.I8(b.q, torch.rand(2, N, device="cuda", generator=g) + 0.5)
    a.q.zero_()
    at = torch.tensor(SAMPLE, device="cuda")
    for lo, hi in spans:
        a.q[at, lo:hi] = torch.randint(-127, 128, (len(SAMPLE), hi - lo), device="cuda", generator=g).to(torch.int8)
        b.q[:, hi:(hi + 127) // 128 * 128] = 0
    for dtype in (torch.float32, torch.bfloat16):
        ld = LDW * (4 // dtype.itemsize)
        big = torch.empty(2 * M, ld, dtype=dtype, device="cuda")
        c = big[:, ld - N - 3:ld - 3]
        oz.oz2_i8_grouped_grad(M, N, TOKENS, 2, off, 1.0, a, b, 0.0, c, ld)
        for e, (lo, hi) in enumerate(spans):
            want = R.product((a.q[at, lo:hi], a.scale[e][at]), (b.q[:, lo:hi], b.scale[e]))
            R.check(c[e * M + at], want, R.bound(want, want, dtype))
        del big, c
    a.q.zero_()
    for lo, hi in spans:
        a.q[at, lo:hi] = torch.randint(-127, 128, (len(SAMPLE), hi - lo), device="cuda", generator=g).to(torch.int8)
    out = torch.empty(2 * N, 2 * M, device="cuda")[:, M:]      # the far one as B, behind other columns
    oz.oz2_i8_grouped_grad(N, M, TOKENS, 2, off, 1.0, b, a, 0.0, out, 2 * M)
    for e, (lo, hi) in enumerate(spans):
        want = R.product((b.q[:, lo:hi], b.scale[e]), (a.q[at, lo:hi], a.scale[e][at]))
        R.check(out[e * N:(e + 1) * N][:, at], want, R.bound(want, want, torch.float32))
