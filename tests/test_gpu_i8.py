"""Products in 8-bit integers, alone and grouped by expert, and the conversions to them, against their definitions in 64 bits."""
import math

import pytest
import torch

import i8_reference as R
import paper_2508_03984_amd as oz

pytestmark = pytest.mark.gpu

TYPES = [torch.bfloat16, torch.float16, torch.float32]
FILL = 77                                                     # what lies where nothing may be written


def gen(seed):
    return torch.Generator("cuda").manual_seed(seed)


def normal(g, rows, cols, dtype, ld=None, before=0):
    """rows x cols numbers at a place of a larger buffer: `before` numbers behind its beginning, rows ld apart, NaN between them."""
    ld = ld or cols
    buf = torch.full((before + max(rows, 1) * ld,), math.nan, dtype=dtype, device="cuda")
    x = torch.as_strided(buf, (rows, cols), (ld, 1), before)
    x.copy_(torch.randn(rows, cols, device="cuda", generator=g) * torch.exp(2 * torch.randn(rows, 1, device="cuda", generator=g)))
    return x


def target(rows, cols, groups=1, ld=None):
    """A matrix to be written, in memory full of FILL with 2 rows more than it has."""
    ld = ld or (cols + 15) // 16 * 16 + 16
    q = torch.full((rows + 2, ld), FILL, dtype=torch.int8, device="cuda")
    s = torch.full((groups, rows + 2), float(FILL), device="cuda")
    m = oz.I8(q[:rows, :cols], s[0, :rows] if groups == 1 else s[:, :rows])
    return m, q, s


def ends(q, rows, cols, whole):
    """Bytes behind the rows: cleared to a multiple of `whole`, further ones as they were."""
    up = (cols + whole - 1) // whole * whole
    assert (q[:rows, cols:up] == 0).all() and (q[:rows, up:] == FILL).all() and (q[rows:] == FILL).all()


SIZES = [(1, 1), (1, 7), (3, 8), (2, 15), (5, 129), (130, 500), (7, 513), (64, 777), (129, 1111), (3, 2049), (260, 130), (2, 5000), (5, 8200), (3, 16384), (2, 16390),
         (1, 40001), (1000, 33)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", SIZES)
def test_quantize(rows, cols, dtype):
    x = normal(gen(rows * cols), rows, cols, dtype, cols + 3, 1)
    if rows > 2:
        x[rows // 2] = 0
    a, qa, sa = target(rows, cols)
    t, qt, st = target(cols, rows)
    oz.oz2_i8_quantize(1, rows, cols, x, cols + 3, a, t)
    want, scale = R.quantize(x)
    assert torch.equal(a.scale, scale) and torch.equal(a.q, want)
    want, scale = R.quantize(x.t())
    assert torch.equal(t.scale, scale) and torch.equal(t.q, want)
    ends(qa, rows, cols, 16)
    ends(qt, cols, rows, 16)
    assert (sa[:, rows:] == FILL).all() and (st[:, cols:] == FILL).all()
    alone, _, _ = target(rows, cols)
    oz.oz2_i8_quantize(1, rows, cols, x, cols + 3, alone, None)
    assert torch.equal(alone.q, a.q) and torch.equal(alone.scale, a.scale)
    alone, _, _ = target(cols, rows)
    oz.oz2_i8_quantize(1, rows, cols, x, cols + 3, None, alone)
    assert torch.equal(alone.q, t.q) and torch.equal(alone.scale, t.scale)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("batch,rows,cols", [(2, 1, 1), (3, 5, 17), (7, 130, 70), (70, 3, 9), (2, 257, 600), (65, 129, 130)])
def test_quantize_a_batch(batch, rows, cols, dtype):
    x = normal(gen(batch), batch * rows, cols, dtype)
    a, qa, _ = target(batch * rows, cols)
    t, qt, st = target(batch * cols, rows)
    oz.oz2_i8_quantize(batch, rows, cols, x, cols, a, t)
    want, scale = R.quantize(x)
    assert torch.equal(a.scale, scale) and torch.equal(a.q, want)
    want, scale = R.quantize(x.reshape(batch, rows, cols).mT)
    assert torch.equal(t.scale, scale.flatten()) and torch.equal(t.q, want.flatten(0, 1))
    ends(qa, batch * rows, cols, 16)
    ends(qt, batch * cols, rows, 16)
    assert (st[:, batch * cols:] == FILL).all()


@pytest.mark.parametrize("by", [1.0, 2.0 ** -100, 2.0 ** -126, 2.0 ** 120, 1 / 3, 1.7e-38, 1e-42])
def test_quantize_at_the_middle_of_two_integers(by):
    """Quotients that are halves of odd numbers, and the numbers next to them: a scale of `by` (a power of two: the halves are met exactly)."""
    n = torch.arange(-126, 127, device="cuda").float()
    half = (n + 0.5) * by
    rows = [half, torch.nextafter(half, half + math.inf), torch.nextafter(half, half - math.inf)]
    x = torch.stack([torch.cat((r, torch.tensor([127.0 * by, 0.0, -0.0], device="cuda"))) for r in rows])
    a, _, _ = target(*x.shape)
    t, _, _ = target(x.shape[0], x.shape[1])
    oz.oz2_i8_quantize(1, *x.shape, x, x.shape[1], a, None)
    turned = x.t().contiguous()
    oz.oz2_i8_quantize(1, *turned.shape, turned, turned.shape[1], None, t)
    want, scale = R.quantize(x)
    for m in (a, t):
        assert torch.equal(m.scale, scale) and torch.equal(m.q, want)


def test_quantize_of_random_bits():
    """Every binary32 number can come; so all quotients of these have to be rounded as the definition says."""
    g = gen(5)
    bits = torch.randint(-2 ** 31, 2 ** 31, (300, 4000), device="cuda", generator=g, dtype=torch.int64).int()
    x = bits.view(torch.float32)
    x = torch.where(torch.isfinite(x), x, torch.zeros_like(x))
    near = torch.randn(300, 4000, device="cuda", generator=g)              # (of random bits few are near the largest)
    for y in (x, near, near * 2.0 ** -130, near * 1e38):
        a, _, _ = target(*y.shape)
        oz.oz2_i8_quantize(1, *y.shape, y, y.shape[1], a, None)
        want, scale = R.quantize(y)                           # (the last ones pass the type's range here and there: NaN)
        assert torch.equal(a.scale.view(torch.int32), scale.view(torch.int32)) and torch.equal(a.q, want)


@pytest.mark.parametrize("dtype", TYPES)
def test_quantize_nan_and_infinities(dtype):
    x = normal(gen(1), 300, 700, dtype)
    x[3, 5], x[100, 699], x[200, 0], x[201] = math.nan, math.inf, -math.inf, math.nan
    a, _, _ = target(300, 700)
    t, _, _ = target(700, 300)
    oz.oz2_i8_quantize(1, 300, 700, x, 700, a, t)
    for m, y in ((a, x), (t, x.t())):
        want, scale = R.quantize(y)
        assert torch.equal(torch.isnan(m.scale), torch.isnan(scale)) and torch.equal(m.scale.nan_to_num(), scale.nan_to_num()) and torch.equal(m.q, want)
    assert torch.isnan(t.scale).all() and not torch.isnan(a.scale[4])


# ------------------------------------------------------------------ groups
GROUPS = [[0, 1], [0, 0], [0, 5, 5, 6], [0, 128, 256], [3, 100, 131, 131, 400], [0, 127, 128, 129, 300, 1000], [0] + [i * i for i in range(1, 30)] + [841] * 40 + [900],
          list(range(0, 141)), [0, 64, 1500]]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("offsets", GROUPS, ids=lambda o: f"{len(o) - 1}_groups_{o[-1]}")
@pytest.mark.parametrize("cols", [5, 300, 2100])
def test_quantize_grouped(offsets, cols, dtype):
    rows, groups, g = offsets[-1] + 9, len(offsets) - 1, gen(cols)
    tokens = max(rows // 3, 1)
    x = normal(g, tokens, cols, dtype, cols + 1)
    index = torch.randint(-1, tokens + 1, (rows,), device="cuda", generator=g, dtype=torch.int32)     # (one before and one behind, too)
    index[::17] = torch.tensor([-2 ** 31], device="cuda").int()
    index[5::19] = 2 ** 31 - 1
    off = torch.tensor(offsets, dtype=torch.int32, device="cuda")
    wide = oz.oz2_i8_grouped_cols(rows, groups)
    assert wide == R.grouped_cols(rows, groups)
    a, qa, sa = target(rows, cols)
    t, qt, st = target(cols, wide, groups)
    oz.oz2_i8_quantize_grouped(rows, cols, x, tokens, cols + 1, index, groups, off, a, t)
    full = R.gather(x, index, rows)
    want, scale = R.quantize(full)
    lo, hi = offsets[0], offsets[-1]
    assert torch.equal(a.q[lo:hi], want[lo:hi]) and torch.equal(a.scale[lo:hi], scale[lo:hi])
    for part in (slice(0, lo), slice(hi, None)):
        assert (qa[part] == FILL).all() and (sa[0, part] == FILL).all()
    expect = torch.full((cols, qt.shape[1]), FILL, dtype=torch.int8, device="cuda")
    for i in range(groups):
        first, n = R.first_col(offsets, i), offsets[i + 1] - offsets[i]
        want, scale = R.quantize(full[offsets[i]:offsets[i + 1]].t())
        expect[:, first:first + (n + 127) // 128 * 128] = 0
        expect[:, first:first + n] = want
        assert torch.equal(st[i if groups > 1 else 0, :cols], scale), i
    assert torch.equal(qt[:cols], expect) and (qt[cols:] == FILL).all() and (st[:, cols:] == FILL).all()
    b, _, _ = target(rows, cols)
    rest, _, _ = target(cols, wide, groups)
    own = full.contiguous()
    oz.oz2_i8_quantize_grouped(rows, cols, own, rows, cols, None, groups, off, b, rest)
    assert torch.equal(b.q[lo:hi], a.q[lo:hi]) and torch.equal(rest.scale, t.scale) and torch.equal(rest.q, t.q)


# ------------------------------------------------------------------ products
def operand(g, rows, k, groups=1, ld=None):
    """A matrix in 8-bit integers whose rows are followed by bytes that may not count."""
    ld = ld or (k + 15) // 16 * 16 + 16
    q = torch.randint(-128, 128, (rows + 1, ld), device="cuda", generator=g, dtype=torch.int64).to(torch.int8)
    s = torch.exp(3 * torch.randn(groups, rows, device="cuda", generator=g))
    return oz.I8(q[:rows, :k], s[0] if groups == 1 else s)


def output(g, rows, cols, dtype):
    """C in a larger buffer, and a copy of that."""
    buf = torch.randn(rows + 2, cols + 5, device="cuda", generator=g).mul_(50).to(dtype)
    return buf[1:rows + 1, 3:cols + 3], buf, buf.clone()


def outside_kept(c, buf, before):
    c.copy_(before[1:c.shape[0] + 1, 3:c.shape[1] + 3])
    assert torch.equal(buf, before)


PRODUCTS = [(1, 1, 1), (1, 16, 16), (2, 3, 130), (5, 17, 31), (16, 64, 128), (17, 100, 100), (33, 65, 257), (64, 64, 640), (65, 63, 129), (100, 300, 777), (128, 128, 1024),
            (130, 515, 200), (256, 256, 384), (257, 300, 1000), (300, 1000, 129), (512, 512, 512), (1, 700, 3000), (4, 1024, 5000), (40, 200, 9000), (600, 520, 2000)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n,k", PRODUCTS)
def test_product(m, n, k, dtype):
    g = gen(m + n + k)
    a, b = operand(g, m, k), operand(g, n, k)
    summed = R.product((a.q, a.scale), (b.q, b.scale))
    for alpha, beta in ((1.0, 0.0), (0.37, 0.0), (-1.5, 0.75)):
        if dtype is torch.float16:
            alpha *= 2.0 ** -16
        c, buf, before = output(g, m, n, dtype)
        if beta == 0.0:
            c.fill_(math.nan)                                 # not read
        old = c.double()
        oz.oz2_i8_gemm(m, n, k, alpha, a, b, beta, c, c.stride(0))
        alpha32 = torch.tensor(alpha).double().item()
        want = alpha32 * summed + (beta * old if beta else 0.0)
        R.check(c, want, R.bound(summed, want, dtype, alpha, beta, old))
        outside_kept(c, buf, before)


def test_sums_at_the_end_of_32_bits():
    k = 131071
    a, b = oz.I8.empty(3, k), oz.I8.empty(130, k)
    a.q.fill_(-128)
    b.q.fill_(-128)
    b.q[7] = 127
    a.scale.fill_(1.0)
    b.scale.fill_(1.0)
    c = torch.empty(3, 130, device="cuda")
    oz.oz2_i8_gemm(3, 130, k, 1.0, a, b, 0.0, c, 130)
    want = torch.full((3, 130), 16384.0 * k, device="cuda", dtype=torch.float64)
    want[:, 7] = -128.0 * 127 * k
    assert torch.equal(c, want.float())                       # (both are rounded once, and the scales are 1)


@pytest.mark.parametrize("m,n", [(3, 200), (100, 70), (300, 300)])
def test_nan_scales_reach_their_row_and_column_only(m, n):
    g = gen(3)
    a, b = operand(g, m, 300), operand(g, n, 300)
    a.scale[1], b.scale[n - 1] = math.nan, math.nan
    c = torch.zeros(m, n, device="cuda")
    oz.oz2_i8_gemm(m, n, 300, 1.0, a, b, 0.0, c, n)
    nan = torch.isnan(c)
    assert nan[1].all() and nan[:, n - 1].all() and int(nan.sum()) == m + n - 1


@pytest.mark.parametrize("dtype", TYPES)
def test_products_of_nothing(dtype):
    c, buf, before = output(gen(2), 70, 90, dtype)
    for alpha in (2.0, math.inf, math.nan):
        c.copy_(before[1:71, 3:93])
        oz.oz2_i8_gemm(70, 90, 0, alpha, None, None, 0.5, c, c.stride(0))
        assert torch.equal(c, (before[1:71, 3:93].float() * 0.5).to(dtype))
    off = torch.tensor([0, 10, 60], dtype=torch.int32, device="cuda")
    c.copy_(before[1:71, 3:93])
    oz.oz2_i8_grouped_gemm(70, 90, 0, 2, off, math.inf, None, None, 0.5, c, c.stride(0))
    assert torch.equal(c[:60], (before[1:61, 3:93].float() * 0.5).to(dtype)) and torch.equal(c[60:], before[61:71, 3:93])
    c.copy_(before[1:71, 3:93])
    oz.oz2_i8_grouped_grad(35, 90, 0, 2, torch.zeros(3, dtype=torch.int32, device="cuda"), math.inf, None, None, 0.5, c, c.stride(0))
    assert torch.equal(c, (before[1:71, 3:93].float() * 0.5).to(dtype))
    c.fill_(math.nan)
    oz.oz2_i8_grouped_grad(35, 90, 0, 2, torch.zeros(3, dtype=torch.int32, device="cuda"), 1.0, None, None, 0.0, c, c.stride(0))
    assert (c == 0).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("offsets", GROUPS, ids=lambda o: f"{len(o) - 1}_groups_{o[-1]}")
@pytest.mark.parametrize("n,k", [(1, 1), (70, 130), (300, 257), (129, 1000)])
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
        alpha32 = torch.tensor(alpha).double().item()
        for i in range(groups):
            lo, hi = offsets[i], offsets[i + 1]
            if lo == hi:
                continue
            summed = R.product((a.q[lo:hi], a.scale[lo:hi]), (b.q[i * n:(i + 1) * n], b.scale[i * n:(i + 1) * n]))
            want = alpha32 * summed + beta * old[lo:hi]
            R.check(c[lo:hi], want, R.bound(summed, want, dtype, alpha, beta, old[lo:hi]))
        assert torch.equal(c[:offsets[0]].double(), old[:offsets[0]]) and torch.equal(c[offsets[-1]:].double(), old[offsets[-1]:])
        outside_kept(c, buf, before)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("offsets", GROUPS, ids=lambda o: f"{len(o) - 1}_groups_{o[-1]}")
@pytest.mark.parametrize("m,n", [(1, 1), (70, 130), (129, 300)])
def test_grouped_grad(offsets, m, n, dtype):
    rows, groups, g = offsets[-1] + 7, len(offsets) - 1, gen(n + m)
    off = torch.tensor(offsets, dtype=torch.int32, device="cuda")
    wide = oz.oz2_i8_grouped_cols(rows, groups)
    a, b = operand(g, m, wide, groups), operand(g, n, wide, groups)
    for i in range(groups):                                   # zeros from the end of a group to the next multiple of 128, anything beyond
        first, count = R.first_col(offsets, i), offsets[i + 1] - offsets[i]
        for x in (a, b):
            x.q[:, first + count:first + (count + 127) // 128 * 128] = 0
    for alpha, beta in ((1.0, 0.0), (0.37, 1.0)):
        if dtype is torch.float16:
            alpha *= 2.0 ** -14
        c, buf, before = output(g, groups * m, n, dtype)
        old = c.double()
        oz.oz2_i8_grouped_grad(m, n, rows, groups, off, alpha, a, b, beta, c, c.stride(0))
        alpha32 = torch.tensor(alpha).double().item()
        for i in range(groups):
            part = slice(R.first_col(offsets, i), R.first_col(offsets, i) + offsets[i + 1] - offsets[i])
            scale = (a.scale, b.scale) if groups == 1 else (a.scale[i], b.scale[i])
            summed = R.product((a.q[:, part], scale[0]), (b.q[:, part], scale[1]))
            want = alpha32 * summed + beta * old[i * m:(i + 1) * m]
            R.check(c[i * m:(i + 1) * m], want, R.bound(summed, want, dtype, alpha, beta))
        outside_kept(c, buf, before)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("offsets", [list(range(40)) + [500], [0, 700] + list(range(701, 760)), [0] * 100 + [1] * 20 + [9], [4, 4, 4, 90, 90]], ids=["end", "start", "few", "one"])
@pytest.mark.parametrize("n,k", [(16, 2048), (130, 515), (1000, 4100), (5, 70000)])
def test_grouped_with_most_rows_in_one_group(offsets, n, k, dtype):
    rows, groups, g = offsets[-1] + 3, len(offsets) - 1, gen(n + k)
    a, b = operand(g, rows, k), operand(g, groups * n, k)
    off = torch.tensor(offsets, dtype=torch.int32, device="cuda")
    c, buf, before = output(g, rows, n, dtype)
    old, alpha = c.double(), 2.0 ** -20
    oz.oz2_i8_grouped_gemm(rows, n, k, groups, off, alpha, a, b, 0.0, c, c.stride(0))
    for i in range(groups):
        lo, hi = offsets[i], offsets[i + 1]
        if lo < hi:
            summed = R.product((a.q[lo:hi], a.scale[lo:hi]), (b.q[i * n:(i + 1) * n], b.scale[i * n:(i + 1) * n]))
            R.check(c[lo:hi], alpha * summed, R.bound(summed, alpha * summed, dtype, alpha))
    assert torch.equal(c[:offsets[0]].double(), old[:offsets[0]]) and torch.equal(c[offsets[-1]:].double(), old[offsets[-1]:])
    outside_kept(c, buf, before)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n,k", [(100, 100, 20000), (54, 205, 13245), (3, 16, 40000), (512, 500, 4100), (1300, 1000, 30001), (200, 1, 131071)])
def test_product_in_ranges_of_k(m, n, k, dtype):
    g = gen(k)
    a, b = operand(g, m, k), operand(g, n, k)
    summed = R.product((a.q, a.scale), (b.q, b.scale))
    need = oz.oz2_i8_workspace_bytes(m, n, k)
    assert need > 0
    own, small = oz.Context(), oz.Context()
    room = torch.empty(1 << 12, dtype=torch.uint8, device="cuda")
    oz.oz2_ctx_set_workspace(small, room)       # no room for planes: one range
    for alpha, beta in ((2.0 ** -20, 0.0), (-2.0 ** -19, 0.75)):
        results = []
        for ctx in (None, own, small):
            gen_c = gen(7)
            c, buf, before = output(gen_c, m, n, dtype)
            old = c.double()
            oz.oz2_ctx_i8_gemm(ctx, m, n, k, alpha, a, b, beta, c, c.stride(0))
            want = alpha * summed + beta * old
            R.check(c, want, R.bound(summed, want, dtype, alpha, beta))
            results.append(c.clone())
            outside_kept(c, buf, before)
        assert torch.equal(results[0], results[1]) and torch.equal(results[0], results[2])  # (integer sums are exact in any order)


def in_contexts(call):
    """The call in the default context, in one of its own and in one without room for planes: the same bits."""
    own, small, room = oz.Context(), oz.Context(), torch.empty(1 << 12, dtype=torch.uint8, device="cuda")
    oz.oz2_ctx_set_workspace(small, room)
    got = [call(ctx) for ctx in (None, own, small)]
    assert torch.equal(got[0].view(torch.uint8), got[1].view(torch.uint8)) and torch.equal(got[0].view(torch.uint8), got[2].view(torch.uint8))
    return got[0]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("offsets,n,k", [([3, 40, 40, 90], 64, 8192), ([0, 200, 200, 200, 201], 130, 9001), ([0, 0, 64], 33, 40000)])
def test_grouped_in_ranges_of_k(offsets, n, k, dtype):
    rows, groups, g = offsets[-1] + 5, len(offsets) - 1, gen(k)
    assert oz.oz2_i8_grouped_workspace_bytes(rows, n, k, groups) > 0
    a, b = operand(g, rows, k), operand(g, groups * n, k)
    off = torch.tensor(offsets, dtype=torch.int32, device="cuda")
    old = torch.randn(rows, n, device="cuda", generator=g).mul_(50).to(dtype)
    for alpha, beta in ((2.0 ** -20, 0.0), (-2.0 ** -19, 0.75)):
        def call(ctx):
            c = old.clone()
            oz.oz2_ctx_i8_grouped_gemm(ctx, rows, n, k, groups, off, alpha, a, b, beta, c, n)
            return c
        c = in_contexts(call)
        for i in range(groups):
            lo, hi = offsets[i], offsets[i + 1]
            if lo < hi:
                summed = R.product((a.q[lo:hi], a.scale[lo:hi]), (b.q[i * n:(i + 1) * n], b.scale[i * n:(i + 1) * n]))
                want = alpha * summed + beta * old[lo:hi].double()
                R.check(c[lo:hi], want, R.bound(summed, want, dtype, alpha, beta))
        assert torch.equal(c[:offsets[0]], old[:offsets[0]]) and torch.equal(c[offsets[-1]:], old[offsets[-1]:])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("offsets,m,n", [([0, 3000, 8000], 26, 139), ([5, 5, 4000, 4001, 4001, 9000], 100, 100), ([0, 30000], 64, 65), ([7, 140000, 140100], 20, 30),
                                         ([5, 5, 24000, 24001, 24001, 50000], 100, 100)])
def test_grouped_grad_in_ranges(offsets, m, n, dtype):
    rows, groups, g = offsets[-1] + 5, len(offsets) - 1, gen(m)
    if offsets[-1] != 9000:                                   # (whose groups are as fast without)
        assert oz.oz2_i8_grouped_workspace_bytes(rows, n, m, groups, True) > 0
    wide = oz.oz2_i8_grouped_cols(rows, groups)
    a, b = operand(g, m, wide, groups), operand(g, n, wide, groups)
    off = torch.tensor(offsets, dtype=torch.int32, device="cuda")
    for i in range(groups):
        first, count = R.first_col(offsets, i), offsets[i + 1] - offsets[i]
        for x in (a, b):
            x.q[:, first + count:first + (count + 127) // 128 * 128] = 0
            if count == 0:
                x.scale[i] = float("nan")                     # (the scales of nothing are not read)
    old = torch.randn(groups * m, n, device="cuda", generator=g).mul_(50).to(dtype)
    for alpha, beta in ((2.0 ** -20, 0.0), (-2.0 ** -19, 0.75)):
        def call(ctx):
            c = old.clone()
            oz.oz2_ctx_i8_grouped_grad(ctx, m, n, rows, groups, off, alpha, a, b, beta, c, n)
            return c
        c = in_contexts(call)
        for i in range(groups):
            part = slice(R.first_col(offsets, i), R.first_col(offsets, i) + offsets[i + 1] - offsets[i])
            own, mine = c[i * m:(i + 1) * m], old[i * m:(i + 1) * m].double()
            if offsets[i + 1] - offsets[i] > 131071:
                assert torch.isnan(own).all()
            elif offsets[i + 1] == offsets[i]:
                assert torch.equal(own, (beta * mine).to(dtype))
            else:
                scale = (a.scale, b.scale) if groups == 1 else (a.scale[i], b.scale[i])
                summed = R.product((a.q[:, part], scale[0]), (b.q[:, part], scale[1]))
                want = alpha * summed + beta * mine
                R.check(own, want, R.bound(summed, want, dtype, alpha, beta))
