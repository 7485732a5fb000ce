"""Host side of the 8-bit integer products: refusals, and what the reference of their tests and the layout of groups rest on."""
import ctypes as C
import os
import random

import pytest

import paper_2508_03984_amd as oz
from paper_2508_03984_amd.binding import _I8Struct


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(oz.lib_path()):
        from paper_2508_03984_amd.build import build_library
        build_library()
    return oz.load()


OK, INVALID, UNSUPPORTED = 0, 1, 2
P = 1 << 20                                                   # an address that nothing reads


def i8(q=P, ld=1024, scale=P, ld_scale=1024):
    return C.byref(_I8Struct(q, ld, scale, ld_scale))


BAD = [(dict(q=None), INVALID), (dict(scale=None), INVALID), (dict(q=P + 8), INVALID), (dict(scale=P + 2), INVALID), (dict(ld=192), INVALID),
       (dict(ld=1032), INVALID), (dict(ld=(1 << 23) + 16), UNSUPPORTED)]


@pytest.mark.parametrize("bad,status", BAD)
def test_matrices_that_are_refused(lib, bad, status):
    assert lib.oz2_i8_gemm(70, 70, 200, 1.0, i8(**bad), i8(), 0.0, P, 70, 0, None) == status
    assert lib.oz2_i8_gemm(70, 70, 200, 1.0, i8(), i8(**bad), 0.0, P, 70, 0, None) == status
    assert lib.oz2_i8_grouped_gemm(70, 70, 200, 3, P, 1.0, i8(**bad), i8(), 0.0, P, 70, 0, None) == status
    assert lib.oz2_i8_grouped_gemm(70, 70, 200, 3, P, 1.0, i8(), i8(**bad), 0.0, P, 70, 0, None) == status
    assert lib.oz2_i8_grouped_grad(70, 70, 200, 3, P, 1.0, i8(**bad), i8(), 0.0, P, 70, 0, None) == status
    assert lib.oz2_i8_grouped_grad(70, 70, 200, 3, P, 1.0, i8(), i8(**bad), 0.0, P, 70, 0, None) == status
    assert lib.oz2_i8_quantize(1, 70, 200, P, 200, 0, i8(**bad), None, None) == status
    assert lib.oz2_i8_quantize(1, 200, 70, P, 70, 0, None, i8(**bad), None) == status
    assert lib.oz2_i8_quantize_grouped(70, 200, P, 70, 200, 0, None, 3, P, i8(**bad), None, None) == status
    assert lib.oz2_i8_quantize_grouped(200, 70, P, 200, 70, 0, None, 3, P, None, i8(**bad), None) == status


def test_arguments_that_are_refused(lib):
    gemm = lambda m=70, n=70, k=200, A=i8(), B=i8(), c=P, ldc=70, t=0: lib.oz2_i8_gemm(m, n, k, 1.0, A, B, 0.0, c, ldc, t, None)  # noqa: E731
    assert gemm(m=-1) == gemm(n=-1) == gemm(k=-1) == gemm(A=None) == gemm(B=None) == gemm(c=None) == gemm(ldc=69) == gemm(t=3) == gemm(t=-1) == INVALID
    assert gemm(c=P + 1) == gemm(c=P + 2, t=2) == INVALID
    assert gemm(k=131072, A=i8(ld=1 << 20), B=i8(ld=1 << 20)) == gemm(m=(1 << 30) + 1) == gemm(n=(1 << 30) + 1, ldc=1 << 31) == UNSUPPORTED
    assert gemm(m=1 << 30, n=1 << 30, ldc=1 << 30) == UNSUPPORTED
    assert gemm(m=0) == gemm(n=0) == gemm(m=0, A=None, c=None) == OK

    quant = lambda b=1, r=70, c=200, x=P, ldx=200, t=0, a=i8(), d=None: lib.oz2_i8_quantize(b, r, c, x, ldx, t, a, d, None)  # noqa: E731
    assert quant(b=-1) == quant(r=-1) == quant(c=-1) == quant(x=None) == quant(ldx=199) == quant(t=5) == quant(a=None) == quant(x=P + 1) == INVALID
    assert quant(b=1 << 20, r=1 << 20) == quant(b=1 << 40, r=1 << 40) == quant(b=1 << 62, r=4) == UNSUPPORTED
    assert quant(b=0) == quant(r=0) == quant(c=0) == OK

    group = lambda r=70, c=200, x=P, xr=70, ldx=200, t=0, i=None, g=3, o=P, a=i8(), d=None: lib.oz2_i8_quantize_grouped(  # noqa: E731
        r, c, x, xr, ldx, t, i, g, o, a, d, None)
    assert group(r=-1) == group(c=-1) == group(x=None) == group(ldx=199) == group(t=5) == group(a=None) == group(g=0) == group(o=None) == INVALID
    assert group(xr=69) == group(xr=0, i=P) == group(i=P + 2) == group(o=P + 1) == group(xr=-1, i=P) == INVALID
    assert group(d=i8(ld=256 + 112)) == group(d=i8(ld_scale=199)) == group(r=1000, xr=1000, d=i8(ld=1024 + 240)) == INVALID
    assert group(g=4097) == group(r=(1 << 30) + 1, xr=1 << 40) == UNSUPPORTED
    assert group(r=0) == group(c=0) == OK

    grouped = lambda r=70, n=70, k=200, g=3, o=P, A=i8(), B=i8(), c=P, ldc=70, t=0: lib.oz2_i8_grouped_gemm(  # noqa: E731
        r, n, k, g, o, 1.0, A, B, 0.0, c, ldc, t, None)
    grad = lambda r=200, n=70, k=70, g=3, o=P, A=i8(), B=i8(), c=P, ldc=70, t=0: lib.oz2_i8_grouped_grad(  # noqa: E731
        k, n, r, g, o, 1.0, A, B, 0.0, c, ldc, t, None)
    for call in (grouped, grad):
        assert call(r=-1) == call(n=-1) == call(k=-1) == call(g=0) == call(g=-1) == call(o=None) == call(o=P + 2) == INVALID
        assert call(A=None) == call(B=None) == call(c=None) == call(ldc=69) == call(t=3) == call(c=P + 1) == INVALID
        assert call(g=4097) == call(r=(1 << 30) + 1) == UNSUPPORTED
        assert call(n=0) == OK
    assert grouped(r=0) == grad(k=0) == OK
    assert grouped(k=131072, A=i8(ld=1 << 20), B=i8(ld=1 << 20)) == grouped(g=4096, n=1 << 20, ldc=1 << 20) == UNSUPPORTED
    assert grad(g=4096, k=1 << 20, A=i8(ld=1 << 20)) == UNSUPPORTED
    assert grad(A=i8(ld_scale=69)) == grad(B=i8(ld_scale=69)) == grad(A=i8(ld=496)) == INVALID


def test_groups_that_lie_side_by_side_never_meet(lib):
    rng = random.Random(1)
    for _ in range(300):
        groups = rng.randint(1, 20)
        cuts = sorted(rng.choices(range(rng.choice((1, 5, 300, 5000)) + 1), k=groups + 1))
        rows = cuts[-1] + rng.choice((0, 0, rng.randint(0, 300)))
        wide, end = lib.oz2_i8_grouped_cols(rows, groups), 0
        assert wide == oz.oz2_i8_grouped_cols(rows, groups) == rows // 128 * 128 + 128 * groups
        for g in range(groups):
            first = cuts[g] // 128 * 128 + 128 * g
            assert first >= end
            end = first + (cuts[g + 1] - cuts[g] + 127) // 128 * 128
        assert end <= wide
    assert oz.oz2_i8_grouped_cols(-1, 3) == oz.oz2_i8_grouped_cols(5, 0) == oz.oz2_i8_grouped_cols(5, 4097) == oz.oz2_i8_grouped_cols((1 << 30) + 1, 1) == 0


def test_the_binding_refuses_what_the_structs_cannot_show():
    torch = pytest.importorskip("torch")
    q, s = torch.zeros(4, 32, dtype=torch.int8), torch.zeros(4)
    for args in ((q.to(torch.uint8), s), (q, s.double()), (q, s[:3]), (q, torch.zeros(2, 3)), (q.t(), torch.zeros(32)), (q[:, 20:], s),
                 (q, torch.zeros(8)[::2]), (q, torch.zeros(4, 2).t()), (q, torch.zeros(1, 1, 4)), (q, s)):
        with pytest.raises(ValueError):                       # the last one: right, but not on a device
            oz.I8(*args)


def test_the_reference_rounds_the_scale_once():
    torch = pytest.importorskip("torch")
    import i8_reference as R
    import numpy as np
    top = torch.randn(100000).abs()
    q, s = R.quantize(top[:, None])
    assert np.array_equal(s.numpy(), np.maximum(top.numpy() * (np.float32(1) / np.float32(127)), np.float32(2.0 ** -126)))
    assert set(q.flatten().tolist()) == {127}
