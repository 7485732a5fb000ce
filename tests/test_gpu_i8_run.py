"""8-bit integer products as a program runs them: captured and replayed, on streams and contexts of their own, a run of them together."""
import pytest
import torch

import i8_reference as R
import paper_2508_03984_amd as oz
from test_gpu_i8 import gen, operand

pytestmark = pytest.mark.gpu


def captured(call):
    call()                                                    # allocates
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    return graph


@pytest.mark.parametrize("rows,n,k,groups", [(40, 96, 200, 7), (900, 300, 520, 6), (3000, 1100, 700, 3)])
def test_a_run_of_them_replayed(rows, n, k, groups):
    """Tokens to experts, through their products, back through their gradients; new tokens and other routes before each replay."""
    g = gen(rows)
    x, index, off = (torch.zeros(rows, k, device="cuda", dtype=torch.bfloat16), torch.zeros(rows, dtype=torch.int32, device="cuda"),
                     torch.zeros(groups + 1, dtype=torch.int32, device="cuda"))
    wide = oz.oz2_i8_grouped_cols(rows, groups)
    w = torch.randn(groups * n, k, device="cuda", generator=g)
    w8, wt8 = oz.I8.empty(groups * n, k), oz.I8.empty(groups * k, n)
    x8, xt8, y8, yt8 = oz.I8.empty(rows, k), oz.I8.empty(k, wide, groups), oz.I8.empty(rows, n), oz.I8.empty(n, wide, groups)
    y, dx, dw = (torch.zeros(*s, device="cuda", dtype=torch.float32) for s in ((rows, n), (rows, k), (groups * n, k)))

    def step():
        oz.oz2_i8_quantize(groups, n, k, w, k, w8, wt8)
        oz.oz2_i8_quantize_grouped(rows, k, x, rows, k, index, groups, off, x8, xt8)
        oz.oz2_i8_grouped_gemm(rows, n, k, groups, off, 1.0, x8, w8, 0.0, y, n)
        oz.oz2_i8_quantize_grouped(rows, n, y, rows, n, None, groups, off, y8, yt8)
        oz.oz2_i8_grouped_gemm(rows, k, n, groups, off, 1.0, y8, wt8, 0.0, dx, k)
        oz.oz2_i8_grouped_grad(n, k, rows, groups, off, 1.0, yt8, xt8, 0.0, dw, k)

    graph = captured(step)
    for turn in range(4):
        x.copy_(torch.randn(rows, k, device="cuda", generator=g))
        index.copy_(torch.randint(-1, rows, (rows,), device="cuda", generator=g))
        cuts = torch.sort(torch.randint(0, rows + 1, (groups + 1,), device="cuda", generator=g)).values
        off.copy_(cuts)
        w.normal_(generator=g)
        for t in (y, dx, dw):
            t.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (y, dx, dw)]
        for t in (y, dx, dw):
            t.fill_(7.0)
        step()
        assert all(torch.equal(a, b) for a, b in zip(got, (y, dx, dw)))
        bounds, full = cuts.tolist(), R.gather(x, index, rows)
        for i in range(groups):
            part = slice(bounds[i], bounds[i + 1])
            a, b = R.quantize(full[part]), R.quantize(w[i * n:(i + 1) * n])
            summed = R.product(a, b)
            R.check(y[part], summed, R.bound(summed, summed, torch.float32))
            ya, bt = R.quantize(y[part]), R.quantize(w[i * n:(i + 1) * n].t())
            summed = R.product(ya, bt)
            R.check(dx[part], summed, R.bound(summed, summed, torch.float32))
            if bounds[i] < bounds[i + 1]:
                summed = R.product(R.quantize(y[part].t()), R.quantize(full[part].t()))
                R.check(dw[i * n:(i + 1) * n], summed, R.bound(summed, summed, torch.float32))
            else:
                assert (dw[i * n:(i + 1) * n] == 0).all()
        for t in (y, dx):
            assert (t[:bounds[0]] == 7.0).all() and (t[bounds[-1]:] == 7.0).all()


def test_graphs_of_one_context_keep_their_planes():
    """What a graph replays into is there whatever calls came after the capture, of this format or of 8-bit floating point."""
    g, ctx = gen(1), oz.oz2_create()
    m, n, k = 150, 140, 20000
    a, b = operand(g, m, k), operand(g, n, k)
    c = torch.empty(m, n, device="cuda")
    assert oz.oz2_i8_workspace_bytes(m, n, k) > 0

    def product():
        oz.oz2_ctx_i8_gemm(ctx, m, n, k, 1.0, a, b, 0.0, c, n)

    graph = captured(product)
    product()
    want = c.clone()
    M, N, K = 1536, 1000, 40000
    assert oz.oz2_i8_workspace_bytes(M, N, K) > 8 * oz.oz2_i8_workspace_bytes(m, n, k)
    big_a, big_b, big = operand(g, M, K), operand(g, N, K), torch.empty(M, N, device="cuda")
    f8 = oz.F8.empty(M, K, 1)
    f8.q.view(torch.uint8).zero_()
    f8.scale.view(torch.uint8).fill_(127)
    for _ in range(3):
        oz.oz2_ctx_i8_gemm(ctx, M, N, K, 1.0, big_a, big_b, 0.0, big, N)
        oz.oz2_ctx_f8_gemm(ctx, 1000, 900, K, 1.0, f8, f8, 0.0, big, N)
        torch.cuda.synchronize()
        c.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(c, want)
    oz.oz2_destroy(ctx)


def test_calls_on_two_streams_with_contexts_of_their_own():
    g = gen(2)
    m, n, k = 300, 200, 16000
    sides = []
    for _ in range(2):
        a, b = operand(g, m, k), operand(g, n, k)
        sides.append((torch.cuda.Stream(), oz.oz2_create(), a, b, torch.zeros(m, n, device="cuda"), R.product((a.q, a.scale), (b.q, b.scale))))
    torch.cuda.synchronize()
    for _ in range(20):
        for stream, ctx, a, b, c, _ in sides:
            oz.oz2_ctx_i8_gemm(ctx, m, n, k, 1.0, a, b, 0.0, c, n, stream=stream)
    torch.cuda.synchronize()
    for _, ctx, _, _, c, want in sides:
        R.check(c, want, R.bound(want, want, torch.float32))
        oz.oz2_destroy(ctx)


def test_offsets_that_do_not_ascend_stay_inside():
    """Unspecified results, but in the memory that right offsets may have written."""
    rows, n, k, groups, g = 700, 300, 500, 5, gen(3)
    a, b = operand(g, rows, k), operand(g, groups * n, k)
    wide = oz.oz2_i8_grouped_cols(rows, groups)
    at, bt = operand(g, n, wide, groups), operand(g, k, wide, groups)
    x = torch.randn(rows, k, device="cuda", generator=g)
    for bad in ([0, 600, 100, 650, 20, 700], [-5, -3, 900, 10, 2 ** 31 - 1, -2 ** 31], [700, 600, 500, 400, 300, 0], [2 ** 31 - 1] * 6, [-2 ** 31] * 6, [0, 2 ** 31 - 1, 0, 2 ** 31 - 1, 0, 700]):
        off = torch.tensor(bad, dtype=torch.int32, device="cuda")
        c = torch.full((rows + 4, n + 2), 7.0, device="cuda")
        oz.oz2_i8_grouped_gemm(rows, n, k, groups, off, 1.0, a, b, 0.0, c[2:], n + 2)
        d = torch.full((groups * n + 4, k + 2), 7.0, device="cuda")
        oz.oz2_i8_grouped_grad(n, k, rows, groups, off, 1.0, at, bt, 0.0, d[2:], k + 2)
        q = torch.full((rows + 4, 528), 7, dtype=torch.int8, device="cuda")
        qt = torch.full((k + 4, wide + 16), 7, dtype=torch.int8, device="cuda")
        oz.oz2_i8_quantize_grouped(rows, k, x, rows, k, None, groups, off, oz.I8(q[2:rows + 2, :k], torch.zeros(rows, device="cuda")),
                                   oz.I8(qt[2:k + 2, :wide], torch.zeros(groups, k, device="cuda")))
        torch.cuda.synchronize()
        assert (c[:2] == 7).all() and (c[rows + 2:] == 7).all() and (c[:, n:] == 7).all()
        assert (d[:2] == 7).all() and (d[groups * n + 2:] == 7).all() and (d[:, k:] == 7).all()
        assert (q[:2] == 7).all() and (q[rows + 2:] == 7).all() and (q[:, 512:] == 7).all()
        assert (qt[:2] == 7).all() and (qt[k + 2:] == 7).all() and (qt[:, wide:] == 7).all()
