"""Products in 8-bit floating point against their definitions in 64 bits.

Tolerances.  Quantisation: none, the scales are powers of two and the one rounding is defined.  Products: the matrix cores cut each
product at 2^-13 of the largest of 8, of which 7 can lose something, so an entry is off by less than 7 * 2^-13 sum |a||b|, taken as
2^-10 sum |a||b| with the binary32 additions; over a whole matrix of independent entries the cuts, each less than
2^-13 of a product of about 3 standard deviations, average to less than 2^-12.5 of the norm.  Rounding to the type adds 2^-8 (bfloat16),
2^-11 (half precision; 2^-25 near its subnormals), 2^-24 (single precision)."""
import numpy as np
import pytest

import f8_reference as R

torch = pytest.importorskip("torch")
import paper_2508_03984_amd as oz  # noqa: E402

pytestmark = pytest.mark.gpu
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
EPS = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}
TINY = {"bf16": 0.0, "f16": 2.0 ** -25, "f32": 0.0}
CUT, CUT_NORM = 2.0 ** -10, 2.0 ** -12.5


def host(t):
    return t.detach().cpu().double().numpy() if t.dtype.itemsize > 1 else t.detach().cpu().view(torch.uint8).numpy()


def matrix(q, scale, block_rows, spare=0, filler=0x7f):
    """An oz.F8 of the bytes, in rows with `spare` * 16 more bytes; what lies between the rows is NaN."""
    rows, cols = q.shape
    ld, lds = R.up(cols) // 8 * 8 if spare else -(-cols // 16) * 16, -(-scale.shape[1] // 4) * 4
    ld += spare * 16
    big = torch.full((rows, ld), filler, dtype=torch.uint8)
    sc = torch.full((scale.shape[0], lds), 255 if filler else 0, dtype=torch.uint8)
    big[:, :cols] = torch.from_numpy(q)
    sc[:, : scale.shape[1]] = torch.from_numpy(scale)
    big, sc = big.cuda().view(torch.float8_e4m3fn), sc.cuda().view(torch.float8_e8m0fnu)
    return oz.F8(big[:, :cols], sc[:, : scale.shape[1]], block_rows)


def random_f8(rng, rows, k, block_rows, spare=0, spread=1.0):
    """(oz.F8, its numbers in 64 bits)."""
    x = rng.standard_normal((rows, k)) * np.exp(spread * rng.standard_normal((rows, 1)))
    q, s = R.quantize(x, block_rows)
    return matrix(q, s, block_rows, spare), R.numbers(q, s, block_rows)


def close(got, want, mags, name, what=""):
    """got within the tolerances of want, whose sums have the magnitudes mags."""
    err = np.abs(got - want)
    assert np.isfinite(got).all(), what
    bound = CUT * mags + EPS[name] * (np.abs(want) + CUT * mags) + TINY[name]
    assert (err <= bound).all(), (what, float((err - bound).max()))
    if got.size >= 64:
        norm = np.linalg.norm(want)
        assert np.linalg.norm(err) <= (CUT_NORM + EPS[name]) * norm + TINY[name] * np.sqrt(got.size), (what, np.linalg.norm(err) / norm)


# ------------------------------------------------------------------ quantisation
def check_quantize(x, dtype, block_rows, spare_x=0, offset=0):
    rows, cols = x.shape
    store = torch.zeros(rows * (cols + spare_x) + offset, dtype=DTYPES[dtype], device="cuda")
    X = store[offset:].view(rows, cols + spare_x)[:, :cols]
    X.copy_(torch.from_numpy(x))
    seen = host(X)
    for as_is, transposed in ((1, 1), (1, 0), (0, 1)):
        a, t = oz.F8.empty(rows, cols, block_rows), oz.F8.empty(cols, rows, block_rows)
        for out in (a, t):
            for part in (out.q, out.scale):
                torch.empty(0, dtype=torch.uint8, device="cuda").set_(part.untyped_storage()).fill_(0xa5)
        oz.oz2_f8_quantize(rows, cols, X, cols + spare_x, a if as_is else None, t if transposed else None)
        torch.cuda.synchronize()
        for out, asked, of in ((a, as_is, seen), (t, transposed, seen.T)):
            q, s = host(out.q), host(out.scale)
            if not asked:
                assert (q == 0xa5).all() and (s == 0xa5).all()
                continue
            want_q, want_s = R.quantize(of, block_rows)
            assert np.array_equal(s, want_s)
            nan = (want_q & 127) == 127
            assert np.array_equal((q & 127) == 127, nan) and np.array_equal(q[~nan], want_q[~nan])
            whole = torch.as_strided(out.q.view(torch.uint8), (out.q.shape[0], out.q.stride(0)), (out.q.stride(0), 1)).cpu().numpy()
            kept = -(-out.q.shape[1] // 16) * 16
            assert (whole[:, out.q.shape[1]: kept] == 0).all() and (whole[:, kept:] == 0xa5).all()


@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 16), (2, 17), (128, 128), (127, 129), (129, 300), (37, 1111), (1, 4096), (300, 5)])
def test_quantize(rows, cols, dtype, block_rows):
    rng = np.random.default_rng(rows * 7 + cols)
    x = rng.standard_normal((rows, cols)) * np.exp(2 * rng.standard_normal((rows, cols)))
    x = np.clip(x, -6e4, 6e4)
    x[rows // 2] = 0
    check_quantize(x, dtype, block_rows)
    check_quantize(x, dtype, block_rows, spare_x=8)
    check_quantize(x, dtype, block_rows, spare_x=3, offset=1)


@pytest.mark.parametrize("block_rows", [1, 128])
def test_quantize_special_numbers(block_rows):
    nan, inf, big = np.nan, np.inf, float(np.finfo(np.float32).max)
    rows = [[0.0, -0.0], [448.0, 1.0], [448.0000305, 1.0], [nan, 3.0], [inf, -inf], [-inf, 0.5], [nan, nan], [big, -big], [2.0 ** -149, 0],
            [2.0 ** -126, -2.0 ** -130], [2.0 ** -118, 1.75 * 2.0 ** -118], [449.0, 17.0], [17.0, 19.0], [1.0625, 448], [-1.1875, 448], [2.0 ** -10, 448], [3 * 2.0 ** -10, 448]]
    x = np.zeros((len(rows), 130))
    x[:, 3:5], x[:, 129] = rows, np.array(rows)[:, 0]
    check_quantize(x.astype(np.float32).astype(np.float64), "f32", block_rows)
    for i in range(len(rows)):                                # each row alone: in blocks of 128 rows it has its own scale then
        check_quantize(x[i: i + 1].astype(np.float32).astype(np.float64), "f32", block_rows)


# ------------------------------------------------------------------ products
PRODUCTS = [(1, 1, 1), (1, 16, 128), (3, 17, 130), (16, 40, 512), (17, 100, 640), (33, 130, 1111), (64, 64, 777), (65, 64, 777), (128, 128, 128),
            (129, 127, 255), (200, 333, 1024), (256, 256, 2100), (300, 200, 5000), (2, 5000, 300), (3000, 5, 200), (3600, 3584, 300), (3585, 3601, 129)]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("m,n,k", PRODUCTS)
def test_product(m, n, k, dtype):
    rng = np.random.default_rng(m + n + k)
    for b_rows, spare, a_rows in ((128, 0, 1), (1, 1, 128)):
        (A, a), (B, b) = random_f8(rng, m, k, a_rows, spare, 0.3), random_f8(rng, n, k, b_rows, spare, 0.3)
        want, mags = a @ b.T, np.abs(a) @ np.abs(b).T
        for ldc in (n, n + 5) if spare else (-(-n // 16) * 16,):
            C = torch.full((m, ldc), 7.0, dtype=DTYPES[dtype], device="cuda")
            oz.oz2_f8_gemm(m, n, k, 1.0, A, B, 0.0, C, ldc)
            close(host(C[:, :n]), want, mags, dtype, (b_rows, ldc))
            assert (C[:, n:] == 7.0).all()


@pytest.mark.parametrize("m,n,k", [(5, 50, 300), (130, 70, 300), (130, 70, 9000), (3600, 3584, 128)])
def test_product_alpha_beta(m, n, k):
    rng = np.random.default_rng(5)
    (A, a), (B, b) = random_f8(rng, m, k, 1), random_f8(rng, n, k, 128)
    for dtype in DTYPES:
        before = torch.from_numpy(rng.standard_normal((m, n))).to("cuda", DTYPES[dtype])
        C = before.clone()
        oz.oz2_f8_gemm(m, n, k, -0.5, A, B, 2.0, C, n)
        want, mags = -0.5 * (a @ b.T) + 2 * host(before), 0.5 * np.abs(a) @ np.abs(b).T
        err = np.abs(host(C) - want)
        # binary32 on the way: 2^-23 of either term
        assert (err <= CUT * mags + EPS[dtype] * (np.abs(want) + CUT * mags) + 2.0 ** -22 * (mags + 2 * np.abs(host(before))) + TINY[dtype]).all()
        C = torch.full((m, n), float("nan"), dtype=DTYPES[dtype], device="cuda")
        oz.oz2_f8_gemm(m, n, k, 1.0, A, B, 0.0, C, n)
        assert torch.isfinite(C).all()
    C = torch.ones(m, n, device="cuda")
    oz.oz2_f8_gemm(m, n, 0, 1.0, A, B, 3.0, C, n)
    assert (C == 3).all()
    oz.oz2_f8_gemm(m, n, 0, 1.0, None, None, 0.0, C, n)
    assert (C == 0).all()


@pytest.mark.parametrize("m,n", [(7, 90), (150, 90), (3600, 3584)])
def test_product_nan_goes_where_it_belongs(m, n):
    rng = np.random.default_rng(6)
    k = 390
    x, w = rng.standard_normal((m, k)), rng.standard_normal((n, k))
    x[2, 100], w[5, 389] = np.nan, np.nan
    (qa, sa), (qb, sb) = R.quantize(x, 1), R.quantize(w, 1)
    sa[4, 3] = 255
    C = torch.empty(m, n, device="cuda")
    oz.oz2_f8_gemm(m, n, k, 1.0, matrix(qa, sa, 1), matrix(qb, sb, 1), 0.0, C, n)
    nan = np.zeros((m, n), bool)
    nan[[2, 4]] = nan[:, 5] = True
    assert np.array_equal(np.isnan(host(C)), nan)


@pytest.mark.parametrize("m,n", [(7, 90), (150, 90)])
def test_product_scales_at_the_ends(m, n):
    """Scales of 2^-126 and 2^127 against their opposites: the products are ordinary numbers."""
    rng = np.random.default_rng(7)
    k = 256
    (qa, sa), (qb, sb) = R.quantize(rng.standard_normal((m, k)), 1), R.quantize(rng.standard_normal((n, k)), 128)
    sa[:, 0], sb[:, 0], sa[:, 1], sb[:, 1] = 1, 254, 254, 1
    a, b = R.numbers(qa, sa, 1), R.numbers(qb, sb, 128)
    C = torch.empty(m, n, device="cuda")
    oz.oz2_f8_gemm(m, n, k, 1.0, matrix(qa, sa, 1), matrix(qb, sb, 128), 0.0, C, n)
    close(host(C), a @ b.T, np.abs(a) @ np.abs(b).T, "f32")


def test_product_of_rows_beyond_4_gib():
    """Rows of A further than 2^32 bytes from its start, in a tile and, as B, in the form for few tokens."""
    rng = np.random.default_rng(8)
    rows, ld, k = 66000, 65536 + 16, 200
    q = torch.zeros((rows, ld), dtype=torch.uint8, device="cuda")
    qa, sa = R.quantize(rng.standard_normal((rows, k)), 1)
    q[:, :k] = torch.from_numpy(qa).cuda()
    scale = torch.zeros((rows, 4), dtype=torch.uint8, device="cuda")
    scale[:, :2] = torch.from_numpy(sa).cuda()
    A, a = oz.F8(q.view(torch.float8_e4m3fn)[:, :k], scale.view(torch.float8_e8m0fnu)[:, :2], 1), R.numbers(qa, sa, 1)
    for n in (48, 80):
        B, b = random_f8(rng, n, k, 1)
        want, mags = a @ b.T, np.abs(a) @ np.abs(b).T
        C = torch.empty(rows, n, device="cuda")
        oz.oz2_f8_gemm(rows, n, k, 1.0, A, B, 0.0, C, n)
        close(host(C), want, mags, "f32")
        C = torch.empty(n, rows, device="cuda")
        oz.oz2_f8_gemm(n, rows, k, 1.0, B, A, 0.0, C, rows)
        close(host(C), want.T, mags.T, "f32")


def test_product_k_ranges_and_workspaces():
    """A long contraction and few tiles: planes of K ranges in the library's workspace, in a caller's, and one range where there is no room."""
    rng = np.random.default_rng(9)
    m, n, k = 150, 140, 20000
    (A, a), (B, b) = random_f8(rng, m, k, 1), random_f8(rng, n, k, 128)
    want, mags = a @ b.T, np.abs(a) @ np.abs(b).T
    need = oz.oz2_f8_workspace_bytes(m, n, k)
    assert need > 0
    ctx = oz.Context()

    def product():
        C = torch.empty(m, n, device="cuda")
        oz.oz2_ctx_f8_gemm(ctx, m, n, k, 1.0, A, B, 0.0, C, n)
        torch.cuda.synchronize()
        close(host(C), want, mags, "f32")
        return C
    own = product()
    assert torch.equal(own, product())
    buf = torch.empty(need, dtype=torch.uint8, device="cuda")
    oz.oz2_ctx_set_workspace(ctx, buf)
    assert torch.equal(own, product())
    small = torch.full((4096,), 9, dtype=torch.uint8, device="cuda")
    oz.oz2_ctx_set_workspace(ctx, small)
    product()
    assert (small == 9).all()
    oz.oz2_ctx_set_workspace(ctx, None)
    oz.oz2_ctx_set_workspace_limit(ctx, 1024)
    product()
    ctx.destroy()


# ------------------------------------------------------------------ gated block
GATED = [(1, 1, 1), (1, 128, 128), (4, 200, 700), (16, 129, 512), (40, 100, 1111), (64, 256, 256), (65, 127, 300), (130, 300, 520), (200, 128, 9000), (2000, 1800, 300)]


def gated_case(rng, m, f, k):
    X, x = random_f8(rng, m, k, 1, 0, 0.2)
    w = rng.standard_normal((R.up(f) + f, k)) * k ** -0.5
    q, s = R.quantize(w, 128)
    q[f: R.up(f)] = 0x7f                                      # rows between the weights are not read
    return X, x, matrix(q, s, 128), R.numbers(q, s, 128)


@pytest.mark.parametrize("act", [0, 1])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("m,f,k", GATED)
def test_gated(m, f, k, dtype, act):
    rng = np.random.default_rng(m + f + k)
    X, x, W, w = gated_case(rng, m, f, k)
    up = R.up(f)
    g, u = x @ w[:f].T, x @ w[up:].T
    mg, mu = np.abs(x) @ np.abs(w[:f]).T, np.abs(x) @ np.abs(w[up:]).T
    for with_z in (True, False):
        H = torch.full((m, f + 3), 7.0, dtype=DTYPES[dtype], device="cuda")
        Z = torch.full((m, up + f), 7.0, dtype=DTYPES[dtype], device="cuda") if with_z else None
        oz.oz2_f8_gated(m, f, k, act, X, W, H, f + 3, Z, up + f)
        h, slope = R.act(g, act)
        # h = act(g) u: slopes are below 1.13, both sums have the error of a product, the activation 2^-20
        eg, eu = CUT * mg, CUT * mu
        bound = 1.13 * eg * (np.abs(u) + eu) + (np.abs(h) + 1.13 * eg) * eu + 2.0 ** -20 * np.abs(h * u)
        want = h * u
        err = np.abs(host(H[:, :f]) - want)
        assert (err <= bound + EPS[dtype] * (np.abs(want) + bound) + TINY[dtype]).all()
        if m * f >= 64:
            assert np.linalg.norm(err) <= (4 * CUT_NORM + EPS[dtype]) * np.linalg.norm(want) + TINY[dtype] * np.sqrt(m * f)
        assert (H[:, f:] == 7.0).all()
        if with_z:
            close(host(Z[:, :f]), g, mg, dtype)
            close(host(Z[:, up:]), u, mu, dtype)
            assert (Z[:, f:up] == 7.0).all()


def test_gated_k_ranges_need_no_workspace():
    rng = np.random.default_rng(11)
    m, f, k = 150, 130, 20000
    X, x, W, w = gated_case(rng, m, f, k)
    assert oz.oz2_f8_workspace_bytes(m, f, k, True) > 0
    want = R.act(x @ w[:f].T, 0)[0] * (x @ w[R.up(f):].T)
    ctx = oz.Context()
    oz.oz2_ctx_set_workspace(ctx, torch.empty(256, dtype=torch.uint8, device="cuda"))
    H = torch.empty(m, f, device="cuda")
    oz.oz2_ctx_f8_gated(ctx, m, f, k, 0, X, W, H, f)
    assert np.linalg.norm(host(H) - want) <= 4 * CUT_NORM * np.linalg.norm(want)
    ctx.destroy()


# ------------------------------------------------------------------ its gradient
def grad_case(rng, m, f, dtype):
    up = R.up(f)
    z = torch.from_numpy(rng.standard_normal((m, up + f)) * 2).to(DTYPES[dtype])
    z[:, f:up] = float("nan")                                 # not read
    dh = torch.from_numpy(rng.standard_normal((m, f)) * np.exp(rng.standard_normal((m, 1)))).to(DTYPES[dtype])
    dh[m // 2] = 0
    return z, dh


@pytest.mark.parametrize("act", [0, 1])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("m,f", [(1, 1), (5, 16), (128, 128), (130, 100), (77, 300), (300, 257)])
def test_gated_grad(m, f, dtype, act):
    rng = np.random.default_rng(m + f)
    up = R.up(f)
    z, dh = grad_case(rng, m, f, dtype)
    g, u, h = host(z[:, :f]), host(z[:, up:]), host(dh)
    a, slope = R.act(g, act)
    want = np.zeros((m, up + f))
    want[:, :f], want[:, up:] = h * u * slope, h * a
    for d_asked, dt_asked, spare in ((1, 1, 0), (1, 0, 1), (0, 1, 3)):
        D, DT = oz.F8.empty(m, up + f), oz.F8.empty(up + f, m)
        Z = torch.full((m, up + f + spare), float("nan"), dtype=DTYPES[dtype], device="cuda")
        Z[:, : up + f] = z.cuda()
        H = torch.zeros((m, f + spare), dtype=DTYPES[dtype], device="cuda")
        H[:, :f] = dh.cuda()
        oz.oz2_f8_gated_grad(m, f, act, Z, up + f + spare, H, f + spare, D if d_asked else None, DT if dt_asked else None)
        for out, asked, of in ((D, d_asked, want), (DT, dt_asked, want.T)):
            if not asked:
                continue
            got = R.numbers(host(out.q), host(out.scale), 1)
            exact = R.numbers(*R.quantize(of, 1), 1)
            # binary32 on the way: a number beside a tie, or a maximum beside 448 2^s, may go the other way: off by a half unit of E4M3
            # (2^-4, or 2^-10 of the scale, which may be the next one) and a little
            top = np.abs(R.blocks(of, 1)).max(axis=(1, 3))
            coarse = np.repeat(top / 448, 128, 1)[:, : of.shape[1]] * 4 * 2.0 ** -10
            assert (np.abs(got - of) <= 2.0 ** -4 * 1.001 * np.abs(of) + coarse * 1.001).all()
            assert (got != exact).mean() <= max(1e-3, 2 / got.size)
            assert (host(out.q)[of == 0] & 127 == 0).all()


def test_gated_grad_against_differences():
    """The sum of dH * H along a direction in Z, by central differences of the forward formula, against the gradient in 8 bits: independent
    roundings of up to 2^-4 over 2 m f products average out to less than 2^-4 / sqrt(3) of the norm, and five standard deviations of that
    over the directions."""
    rng = np.random.default_rng(12)
    m, f = 60, 200
    up = R.up(f)
    for act in (0, 1):
        z, dh = grad_case(rng, m, f, "f32")
        D = oz.F8.empty(m, up + f)
        oz.oz2_f8_gated_grad(m, f, act, z.cuda(), up + f, dh.cuda(), f, D, None)
        d = R.numbers(host(D.q), host(D.scale), 1)
        z, dh = host(z), host(dh)
        loss = lambda g, u: (dh * R.act(g, act)[0] * u).sum()  # noqa: E731
        for _ in range(8):
            vg, vu, e = rng.standard_normal((m, f)), rng.standard_normal((m, f)), 1e-5
            g, u = z[:, :f], z[:, up:]
            slope = (loss(g + e * vg, u + e * vu) - loss(g - e * vg, u - e * vu)) / (2 * e)
            got = (d[:, :f] * vg).sum() + (d[:, up:] * vu).sum()
            assert abs(got - slope) <= 5 * 2.0 ** -4 / np.sqrt(3) * np.linalg.norm(d)


def test_whole_gradient():
    """dX and dW of the block from the quantised gradient, against their formulas on the quantised factors."""
    rng = np.random.default_rng(13)
    m, f, k = 150, 200, 300
    up = R.up(f)
    z, dh = grad_case(rng, m, f, "bf16")
    x, w = rng.standard_normal((m, k)), rng.standard_normal((up + f, k)) * k ** -0.5
    w[f:up] = 0
    Xt, xt = (lambda q: (matrix(*q, 1), R.numbers(*q, 1)))(R.quantize(x.T, 1))
    Wt, wt = (lambda q: (matrix(*q, 128), R.numbers(*q, 128)))(R.quantize(w.T, 128))
    D, DT = oz.F8.empty(m, up + f), oz.F8.empty(up + f, m)
    oz.oz2_f8_gated_grad(m, f, 0, z.cuda(), up + f, dh.cuda(), f, D, DT)
    dx, dw = torch.empty(m, k, device="cuda"), torch.empty(up + f, k, device="cuda")
    oz.oz2_f8_gemm(m, k, up + f, 1.0, D, Wt, 0.0, dx, k)
    oz.oz2_f8_gemm(up + f, k, m, 1.0, DT, Xt, 0.0, dw, k)
    d, dt = R.numbers(host(D.q), host(D.scale), 1), R.numbers(host(DT.q), host(DT.scale), 1)
    close(host(dx), d @ wt.T, np.abs(d) @ np.abs(wt).T, "f32")
    close(host(dw), dt @ xt.T, np.abs(dt) @ np.abs(xt).T, "f32")
    assert (dw[f:up] == 0).all()


# ------------------------------------------------------------------ streams and graphs
def test_streams_and_repetition():
    rng = np.random.default_rng(14)
    m, n, k = 150, 140, 20000
    (A, a), (B, b) = random_f8(rng, m, k, 1), random_f8(rng, n, k, 128)
    want = torch.empty(m, n, device="cuda")
    oz.oz2_f8_gemm(m, n, k, 1.0, A, B, 0.0, want, n)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = torch.empty(m, n, device="cuda")
    for _ in range(20):
        got.fill_(1.0)
        side.wait_stream(torch.cuda.current_stream())
        oz.oz2_f8_gemm(m, n, k, 1.0, A, B, 0.0, got, n, stream=side)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(got, want)


def test_graph_replays():
    """A token's way through the block, recorded once and replayed on new inputs, with other work between the replays."""
    rng = np.random.default_rng(15)
    m, f, k = 3, 200, 300
    X, _, W, _ = gated_case(rng, m, f, k)
    Down, _ = random_f8(rng, k, f, 128)
    x = torch.zeros(m, k, dtype=torch.bfloat16, device="cuda")
    xq, hq = oz.F8.empty(m, k), oz.F8.empty(m, f)
    h, y = torch.empty(m, f, dtype=torch.bfloat16, device="cuda"), torch.empty(m, k, dtype=torch.bfloat16, device="cuda")

    def step():
        oz.oz2_f8_quantize(m, k, x, k, xq, None)
        oz.oz2_f8_gated(m, f, k, 0, xq, W, h, f)
        oz.oz2_f8_quantize(m, f, h, f, hq, None)
        oz.oz2_f8_gemm(m, k, f, 1.0, hq, Down, 0.0, y, k)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(4):
        x.copy_(torch.from_numpy(rng.standard_normal((m, k))))
        graph.replay()
        torch.cuda.synchronize()
        got = y.clone()
        y.zero_(), h.zero_()
        step()
        assert torch.equal(got, y) and torch.isfinite(y).all() and y.abs().sum() > 0
