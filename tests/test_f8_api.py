"""Host side of the 8-bit floating-point products: refusals, and which form a product takes."""
import ctypes as C
import os

import pytest

import paper_2508_03984_amd as oz
from paper_2508_03984_amd.binding import _F8Struct


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(oz.lib_path()):
        from paper_2508_03984_amd.build import build_library
        build_library()
    return oz.load()


OK, INVALID, UNSUPPORTED = 0, 1, 2
P = 1 << 20                                                   # an address that nothing reads


def f8(q=P, ld=256, scale=P, ld_scale=4, block_rows=1):
    return C.byref(_F8Struct(q, ld, scale, ld_scale, block_rows))


BAD = [(dict(q=None), INVALID), (dict(scale=None), INVALID), (dict(q=P + 8), INVALID), (dict(scale=P + 2), INVALID), (dict(ld=200), INVALID),
       (dict(ld=192), INVALID), (dict(ld=264), INVALID), (dict(ld_scale=0), INVALID), (dict(ld_scale=6), INVALID), (dict(block_rows=2), INVALID),
       (dict(block_rows=0), INVALID), (dict(ld=(1 << 23) + 16), UNSUPPORTED), (dict(ld_scale=(1 << 23) + 4), UNSUPPORTED)]


@pytest.mark.parametrize("bad,status", BAD)
def test_matrices_that_are_refused(lib, bad, status):
    assert lib.oz2_f8_gemm(70, 70, 200, 1.0, f8(**bad), f8(), 0.0, P, 70, 0, None) == status
    assert lib.oz2_f8_gemm(70, 70, 200, 1.0, f8(), f8(**bad), 0.0, P, 70, 0, None) == status
    assert lib.oz2_f8_gated(70, 70, 200, 0, f8(**bad), f8(), P, 70, None, 0, 0, None) == status
    assert lib.oz2_f8_gated(70, 70, 200, 0, f8(), f8(**bad), P, 70, None, 0, 0, None) == status
    assert lib.oz2_f8_quantize(70, 200, P, 200, 0, f8(**bad), None, None) == status
    assert lib.oz2_f8_quantize(200, 70, P, 70, 0, None, f8(**bad), None) == status
    assert lib.oz2_f8_gated_grad(200, 200, 0, P, 456, P, 200, 0, None, f8(**bad), None) == status


def test_arguments_that_are_refused(lib):
    gemm = lambda m=70, n=70, k=200, A=f8(), B=f8(), c=P, ldc=70, t=0: lib.oz2_f8_gemm(m, n, k, 1.0, A, B, 0.0, c, ldc, t, None)  # noqa: E731
    assert gemm(m=-1) == gemm(n=-1) == gemm(k=-1) == gemm(A=None) == gemm(B=None) == gemm(c=None) == gemm(ldc=69) == gemm(t=3) == gemm(t=-1) == INVALID
    assert gemm(c=P + 1) == gemm(c=P + 2, t=2) == INVALID
    assert gemm(k=(1 << 20) + 1, A=f8(ld=1 << 21, ld_scale=1 << 14), B=f8(ld=1 << 21, ld_scale=1 << 14)) == UNSUPPORTED
    assert gemm(m=(1 << 30) + 1) == gemm(n=(1 << 30) + 1, ldc=1 << 31) == UNSUPPORTED
    assert gemm(m=0) == gemm(n=0) == gemm(m=0, A=None, c=None) == OK
    gated = lambda m=70, f=70, k=200, act=0, X=f8(), W=f8(), h=P, ldh=70, z=None, ldz=0, t=0: lib.oz2_f8_gated(  # noqa: E731
        m, f, k, act, X, W, h, ldh, z, ldz, t, None)
    assert gated(act=2) == gated(act=-1) == gated(h=None) == gated(ldh=69) == gated(z=P, ldz=197) == gated(z=P + 1, ldz=198) == gated(t=3) == INVALID
    assert gated(m=0) == gated(f=0) == OK
    quant = lambda r=70, c=200, x=P, ldx=200, t=0, a=f8(), b=None: lib.oz2_f8_quantize(r, c, x, ldx, t, a, b, None)  # noqa: E731
    assert quant(r=-1) == quant(c=-1) == quant(x=None) == quant(ldx=199) == quant(t=5) == quant(a=None) == quant(x=P + 1) == INVALID
    assert quant(b=f8(block_rows=128)) == INVALID             # two forms, two sizes of blocks
    assert quant(r=0) == quant(c=0) == OK
    grad = lambda m=70, f=70, act=0, z=P, ldz=198, h=P, ldh=70, t=0, d=f8(), dt=None: lib.oz2_f8_gated_grad(m, f, act, z, ldz, h, ldh, t, d, dt, None)  # noqa: E731
    assert grad(d=None) == grad(z=None) == grad(h=None) == grad(ldz=197) == grad(ldh=69) == grad(act=7) == grad(d=f8(block_rows=128)) == INVALID
    assert grad(d=f8(ld=192)) == grad(m=300, d=None, dt=f8()) == INVALID
    assert grad(m=0) == grad(f=0) == OK


def test_the_binding_refuses_what_the_structs_cannot_show():
    torch = pytest.importorskip("torch")
    q = torch.zeros(4, 32, dtype=torch.uint8).view(torch.float8_e4m3fn)
    s = torch.zeros(4, 4, dtype=torch.uint8).view(torch.float8_e8m0fnu)
    for args in ((q.view(torch.uint8), s[:, :1], 1), (q, s[:, :1].view(torch.uint8), 1), (q, s[:, :2], 1), (q, s[:, :1], 128), (q, s[:, :1], 3),
                 (q.t(), s[:, :1], 1), (q[:, 16:20], s[:, :1], 1), (q, s[:, :1], 1)):
        with pytest.raises(ValueError):                       # the last one: right, but not on a device
            oz.F8(*args)


def test_workspace_only_for_few_tiles_and_long_contractions(lib):
    need = oz.oz2_f8_workspace_bytes
    assert need(1, 8192, 8192) == need(16384, 16384, 16384) == need(128, 128, 512) == need(0, 5, 5) == need(-1, 5, 5) == 0
    for gated in (False, True):
        assert need(150, 140, 20000, gated) > 0
        for m, n, k in ((65, 17, 3000), (1500, 1111, 3001), (1536, 1000, 40000), (200, 1, 1 << 20)):
            wide = (n + 15) // 16 * 16 * (2 if gated else 1)
            assert need(m, n, k, gated) in [r * m * wide * 4 for r in (0, *range(2, 17))]


def test_launches_that_would_be_too_large_are_refused(lib):
    wide = f8(ld=1 << 20, ld_scale=1 << 13)
    assert lib.oz2_f8_gemm(1 << 30, 1 << 20, 200, 1.0, f8(), f8(), 0.0, P, 1 << 20, 0, None) == UNSUPPORTED
    assert lib.oz2_f8_gemm(1, 1 << 30, 200, 1.0, f8(), f8(), 0.0, P, 1 << 30, 0, None) == UNSUPPORTED
    assert lib.oz2_f8_quantize(1 << 30, 200, P, 200, 0, f8(), None, None) == UNSUPPORTED
    assert lib.oz2_f8_gated_grad(1 << 30, 1 << 19, 0, P, 1 << 20, P, 1 << 19, 0, wide, None, None) == UNSUPPORTED


PLAN = r"""
#include "%s"
#include <cstdio>
using namespace oz2;
int main() {
    long m, n, k; int gated;
    while (scanf("%%ld %%ld %%ld %%d", &m, &n, &k, &gated) == 4) {
        const F8Plan p = f8_plan(m, n, k, gated), q = f8_plan_one_range(m, n, k, gated);
        printf("%%d %%d %%d %%zu %%d %%d\n", (int)p.form, p.ranges, p.kb_each, p.plane_bytes, (int)q.form, q.kb_each);
    }
}
"""


def test_plans_fit_what_the_kernels_assume(tmp_path):
    """For many sizes: ranges are whole groups of 4 blocks, none empty, all blocks covered; the form for few rows has few rows; large tiles are
    whole and have three blocks in every range; planes only for several ranges."""
    import random
    import subprocess
    src, exe = tmp_path / "plan.cpp", tmp_path / "plan"
    src.write_text(PLAN % os.path.join(os.path.dirname(oz.lib_path()), "csrc", "oz2_f8.hpp"))
    subprocess.check_call(["g++", "-O1", "-std=c++17", str(src), "-o", str(exe)])
    rng = random.Random(3)
    size = lambda hi: int(2 ** rng.uniform(0, hi))  # noqa: E731
    cases = [(size(15), size(15), size(20), rng.randrange(2)) for _ in range(4000)]
    cases += [(m, n, k, g) for m in (1, 64, 65, 255, 256, 257) for n in (1, 127, 128, 129, 256, 60000) for k in (0, 1, 128, 257, 385, 512, 1 << 20) for g in (0, 1)]
    out = subprocess.run([str(exe)], input="\n".join("%d %d %d %d" % c for c in cases), capture_output=True, text=True, check=True).stdout.split("\n")
    forms = set()
    for (m, n, k, gated), line in zip(cases, out):
        form, ranges, each, planes, form1, each1 = map(int, line.split())
        blocks, wide = -(-k // 128), n * (2 if gated else 1)
        forms.add((form, ranges > 1))
        assert 1 <= ranges <= 16 and (ranges - 1) * each < max(blocks, 1) <= ranges * max(each, 1)
        assert ranges == 1 or each % 4 == 0
        assert planes == (0 if ranges == 1 else ranges * m * (-(-n // 16) * 16) * (2 if gated else 1) * 4)
        assert form != 0 or (m <= 64 and ranges == 1)
        assert form != 3 or (m >= 256 and wide >= 256 and blocks - (ranges - 1) * each >= 3)
        assert form1 == form and each1 == max(blocks, 1) and (form1 != 3 or blocks >= 3)
    assert forms == {(0, False), (1, False), (1, True), (2, False), (2, True), (3, False), (3, True)}
