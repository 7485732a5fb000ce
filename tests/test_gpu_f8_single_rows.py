"""Matrices of one row, or of one row of scales, whose tensors have any stride between rows that do not exist."""
import numpy as np
import pytest

import f8_reference as R

torch = pytest.importorskip("torch")
import paper_2508_03984_amd as oz  # noqa: E402
from test_gpu_f8 import close, host, random_f8  # noqa: E402

pytestmark = pytest.mark.gpu


def cut(values, width, dtype):
    """The rows of `values` as the beginnings of rows of `width` bytes."""
    big = torch.zeros((values.shape[0], width), dtype=torch.uint8, device="cuda")
    big[:, : values.shape[1]] = torch.from_numpy(values).cuda()
    return big.view(dtype)[:, : values.shape[1]]


@pytest.mark.parametrize("k,width", [(20, 40), (20, 33), (300, 307), (300, 304)])
def test_one_row(k, width):
    rng = np.random.default_rng(k + width)
    q, s = R.quantize(rng.standard_normal((1, k)), 1)
    A = oz.F8(cut(q, width, torch.float8_e4m3fn), cut(s, 7, torch.float8_e8m0fnu), 1)
    B, b = random_f8(rng, 50, k, 128)
    a = R.numbers(q, s, 1)
    for m, n, X, Y, x, y in ((1, 50, A, B, a, b), (50, 1, B, A, b, a)):
        C = torch.empty(m, n, device="cuda")
        oz.oz2_f8_gemm(m, n, k, 1.0, X, Y, 0.0, C, n)
        close(host(C), x @ y.T, np.abs(x) @ np.abs(y).T, "f32")
    x = torch.from_numpy(rng.standard_normal((1, k))).float().cuda()
    oz.oz2_f8_quantize(1, k, x, k, A, None)
    want_q, want_s = R.quantize(host(x), 1)
    assert np.array_equal(host(A.q), want_q) and np.array_equal(host(A.scale), want_s)


def test_one_row_of_scales():
    rng = np.random.default_rng(3)
    q, s = R.quantize(rng.standard_normal((100, 300)), 128)
    B = oz.F8(cut(q, 304, torch.float8_e4m3fn), cut(s, 5, torch.float8_e8m0fnu), 128)
    A, a = random_f8(rng, 70, 300, 1)
    b = R.numbers(q, s, 128)
    C = torch.empty(70, 100, device="cuda")
    oz.oz2_f8_gemm(70, 100, 300, 1.0, A, B, 0.0, C, 100)
    close(host(C), a @ b.T, np.abs(a) @ np.abs(b).T, "f32")
