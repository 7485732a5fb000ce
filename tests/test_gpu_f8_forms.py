"""Products in 8-bit floating point and the gated block at sizes that take each form of the kernels: tiles with two and with four stages, tiles of
64 x 128, large tiles moved inwards at the edges, all of them with K ranges, and with everything that can be asked of the results.  Tolerances
are those of test_gpu_f8.py."""
import numpy as np
import pytest

import f8_reference as R

torch = pytest.importorskip("torch")
import paper_2508_03984_amd as oz  # noqa: E402
from test_gpu_f8 import CUT, DTYPES, EPS, TINY, check_quantize, close, gated_case, host, random_f8, test_gated_grad as check_gated_grad  # noqa: E402

pytestmark = pytest.mark.gpu

# (m, n, k): form and K ranges that the sizes lead to
PRODUCTS = [
    (500, 300, 777),                                          # 64 x 64, four stages
    (3585, 3601, 129), (2050, 2100, 400), (2600, 2500, 385),  # 64 x 64, two stages
    (2000, 2000, 1500),                                       # 64 x 128
    (3100, 2900, 600), (257, 40000, 500),                     # 256 x 256
    (300, 200, 5000), (80, 80, 40000),                        # 64 x 64 in ranges
    (700, 600, 30000),                                        # 64 x 128 in ranges
    (1300, 1300, 30000), (1536, 1000, 40000),                 # 256 x 256 in ranges
]


@pytest.mark.parametrize("m,n,k", PRODUCTS)
def test_products(m, n, k):
    rng = np.random.default_rng(m + k)
    (A, a), (B, b) = random_f8(rng, m, k, 1, 1, 0.3), random_f8(rng, n, k, 128, 0, 0.3)
    want, mags = a @ b.T, np.abs(a) @ np.abs(b).T
    for dtype, ldc in (("bf16", n), ("f16", n + 3), ("f32", n + 1)):
        C = torch.full((m, ldc), 7.0, dtype=DTYPES[dtype], device="cuda")
        oz.oz2_f8_gemm(m, n, k, 1.0, A, B, 0.0, C, ldc)
        close(host(C[:, :n]), want, mags, dtype, dtype)
        assert (C[:, n:] == 7.0).all()
        again = torch.full((m, ldc), 7.0, dtype=DTYPES[dtype], device="cuda")
        oz.oz2_f8_gemm(m, n, k, 1.0, A, B, 0.0, again, ldc)
        assert torch.equal(C, again)
        before = torch.from_numpy(rng.standard_normal((m, n))).to("cuda", DTYPES[dtype])
        C = before.clone()
        oz.oz2_f8_gemm(m, n, k, 0.5, A, B, -1.5, C, n)
        expect = 0.5 * want - 1.5 * host(before)
        err = np.abs(host(C) - expect)
        assert (err <= CUT * mags + EPS[dtype] * (np.abs(expect) + CUT * mags) + 2.0 ** -22 * (mags + 2 * np.abs(host(before))) + TINY[dtype]).all()


GATED = [(500, 200, 777), (500, 5000, 130), (1100, 1000, 1500), (2900, 1500, 500), (1500, 1001, 385), (150, 130, 20000), (600, 700, 20000)]


@pytest.mark.parametrize("m,f,k", GATED)
def test_gated(m, f, k):
    rng = np.random.default_rng(m + k)
    X, x, W, w = gated_case(rng, m, f, k)
    up = R.up(f)
    g, u = x @ w[:f].T, x @ w[up:].T
    mg, mu = np.abs(x) @ np.abs(w[:f]).T, np.abs(x) @ np.abs(w[up:]).T
    eg, eu = CUT * mg, CUT * mu
    for act, dtype in ((0, "bf16"), (1, "f16"), (0, "f32")):
        H = torch.full((m, f + 1), 7.0, dtype=DTYPES[dtype], device="cuda")
        Z = torch.full((m, up + f), 7.0, dtype=DTYPES[dtype], device="cuda")
        oz.oz2_f8_gated(m, f, k, act, X, W, H, f + 1, Z, up + f)
        h = R.act(g, act)[0]
        want = h * u
        bound = 1.13 * eg * (np.abs(u) + eu) + (np.abs(h) + 1.13 * eg) * eu + 2.0 ** -20 * np.abs(want)
        err = np.abs(host(H[:, :f]) - want)
        assert (err <= bound + EPS[dtype] * (np.abs(want) + bound) + TINY[dtype]).all()
        assert (H[:, f:] == 7.0).all() and (Z[:, f:up] == 7.0).all()
        close(host(Z[:, :f]), g, mg, dtype)
        close(host(Z[:, up:]), u, mu, dtype)
        only = torch.empty(m, f, dtype=DTYPES[dtype], device="cuda")
        oz.oz2_f8_gated(m, f, k, act, X, W, only, f)
        assert torch.equal(only, H[:, :f])


def test_every_tile_of_a_large_product_with_odd_blocks():
    """Many tiles per compute unit with an odd number of blocks each, so that the stages change their roles from tile to tile, and an exact
    result: small whole numbers, whose sums no part of the matrix cores rounds."""
    rng = np.random.default_rng(3)
    m, n, k = 6000, 5900, 128 * 5 + 40
    a, b = rng.integers(-2, 3, (m, k)).astype(np.float64), rng.integers(-2, 3, (n, k)).astype(np.float64)
    A, B = oz.F8.empty(m, k), oz.F8.empty(n, k, 128)
    oz.oz2_f8_quantize(m, k, torch.from_numpy(a).float().cuda(), k, A, None)
    oz.oz2_f8_quantize(n, k, torch.from_numpy(b).float().cuda(), k, B, None)
    C = torch.empty(m, n, device="cuda")
    oz.oz2_f8_gemm(m, n, k, 1.0, A, B, 0.0, C, n)
    want = torch.from_numpy(a).cuda() @ torch.from_numpy(b).cuda().t()
    assert torch.equal(C.double(), want)


@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_that_end_anywhere(dtype, block_rows):
    """Every number of numbers in the last piece of a row, and in rows shorter than a piece."""
    rng = np.random.default_rng(17)
    for cols in [*range(1, 26), *range(121, 146), 255, 257]:
        for rows in (1, 5, 131):
            x = np.clip(rng.standard_normal((rows, cols)) * np.exp(2 * rng.standard_normal((rows, cols))), -6e4, 6e4)
            check_quantize(x, dtype, block_rows, spare_x=1, offset=cols % 2)


@pytest.mark.parametrize("f", [3, 7, 8, 9, 15, 121, 127, 129, 135, 136])
def test_gated_grad_of_rows_that_end_anywhere(f):
    check_gated_grad(5, f, "bf16", f % 2)
    check_gated_grad(129, f, "f32", f // 2 % 2)


@pytest.mark.parametrize("m,n,k", [(6, 70, 300), (130, 71, 300), (257, 40000, 500), (3600, 3585, 400), (300, 201, 5000)])
def test_adding_to_c(m, n, k):
    """Rows of C that begin anywhere, in every form, with what is beside C left as it is."""
    rng = np.random.default_rng(m + n)
    (A, a), (B, b) = random_f8(rng, m, k, 1, 0, 0.3), random_f8(rng, n, k, 128, 0, 0.3)
    want, mags = a @ b.T, np.abs(a) @ np.abs(b).T
    for dtype, ldc in (("bf16", n + 1), ("f16", n + 2), ("f32", n + 3)):
        before = torch.from_numpy(rng.standard_normal((m, ldc))).to("cuda", DTYPES[dtype])
        before[:, n:] = float("nan")
        C = before.clone()
        oz.oz2_f8_gemm(m, n, k, 2.0, A, B, 0.25, C, ldc)
        was = host(before[:, :n])
        expect = 2.0 * want + 0.25 * was
        err = np.abs(host(C[:, :n]) - expect)
        assert (err <= 2 * CUT * mags + EPS[dtype] * (np.abs(expect) + 2 * CUT * mags) + 2.0 ** -22 * (2 * mags + np.abs(was)) + TINY[dtype]).all()
        assert C[:, n:].isnan().all()


@pytest.mark.parametrize("rows,cols", [(2050, 4097), (1930, 4100), (1300, 200)])
def test_quantize_as_it_is_by_rows_and_by_tiles(rows, cols):
    """Matrices on both sides of the size from which tiles convert what is not transposed."""
    rng = np.random.default_rng(rows)
    X = torch.from_numpy(rng.standard_normal((rows, cols)) * np.exp(2 * rng.standard_normal((rows, cols)))).clamp(-6e4, 6e4).to("cuda", torch.bfloat16)
    a = oz.F8.empty(rows, cols)
    oz.oz2_f8_quantize(rows, cols, X, cols, a, None)
    q, scale = R.quantize(host(X), 1)
    assert np.array_equal(host(a.scale), scale) and np.array_equal(host(a.q), q)
