"""Captured graphs and the memory of a context: what a graph replays into is there whatever calls came after the capture."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
import paper_2508_03984_amd as oz  # noqa: E402
from test_gpu_f8 import random_f8  # noqa: E402

pytestmark = pytest.mark.gpu


def captured(call):
    call()                                                    # allocates
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    return graph


def test_graphs_of_one_context():
    rng = np.random.default_rng(1)
    ctx = oz.oz2_create()
    m, n, k = 150, 140, 20000
    (A, _), (B, _) = random_f8(rng, m, k, 1), random_f8(rng, n, k, 128)
    assert oz.oz2_f8_workspace_bytes(m, n, k) > 0
    C = torch.empty(m, n, device="cuda")
    d = 300
    P, Q = (torch.from_numpy(rng.standard_normal((d, d))).cuda() for _ in range(2))
    R = torch.empty(d, d, dtype=torch.float64, device="cuda")

    def product():
        oz.oz2_ctx_f8_gemm(ctx, m, n, k, 1.0, A, B, 0.0, C, n)

    def dgemm():
        oz.oz2_ctx_dgemm(ctx, oz.OZ2_OP_N, oz.OZ2_OP_N, 0, d, d, d, 1.0, P, d, Q, d, 0.0, R, d, 15)
    of_product, of_dgemm = captured(product), captured(dgemm)
    product(), dgemm()
    want, want_d = C.clone(), R.clone()
    M, N, K = 1536, 1000, 40000
    assert oz.oz2_f8_workspace_bytes(M, N, K) > 8 * oz.oz2_f8_workspace_bytes(m, n, k)
    (A2, _), (B2, _) = random_f8(rng, M, K, 1), random_f8(rng, N, K, 1)
    C2 = torch.empty(M, N, device="cuda")
    for _ in range(3):
        oz.oz2_ctx_f8_gemm(ctx, M, N, K, 1.0, A2, B2, 0.0, C2, N)          # larger planes
        torch.cuda.synchronize()
        fill = torch.full((16 << 20,), 3.0, device="cuda")                 # whatever was freed may be given away again
        C.zero_(), R.zero_()
        of_dgemm.replay(), of_product.replay()
        torch.cuda.synchronize()
        assert torch.equal(C, want) and torch.equal(R, want_d)
        assert (fill == 3.0).all()
    first = C2.clone()
    D = 2000
    X = torch.from_numpy(rng.standard_normal((D, D))).cuda()
    Y = torch.empty(D, D, dtype=torch.float64, device="cuda")
    oz.oz2_ctx_dgemm(ctx, oz.OZ2_OP_N, oz.OZ2_OP_N, 0, D, D, D, 1.0, X, D, X, D, 0.0, Y, D, 15)    # a larger workspace, which ends the graph of the small one
    oz.oz2_ctx_f8_gemm(ctx, M, N, K, 1.0, A2, B2, 0.0, C2, N)
    for _ in range(3):
        C.zero_()
        of_product.replay()
        torch.cuda.synchronize()
        assert torch.equal(C, want)
    assert torch.equal(C2, first)
    del of_product, of_dgemm
    oz.oz2_destroy(ctx)


def test_stages_of_a_product_outlive_planes():
    rng = np.random.default_rng(2)
    ctx = oz.Context()
    m, n, k = 150, 140, 20000
    (A, _), (B, _) = random_f8(rng, m, k, 1), random_f8(rng, n, k, 128)
    C, d = torch.empty(m, n, device="cuda"), 200
    P = torch.from_numpy(rng.standard_normal((d, d))).cuda()
    R = torch.empty(d, d, dtype=torch.float64, device="cuda")
    oz.oz2_ctx_dgemm(ctx, oz.OZ2_OP_N, oz.OZ2_OP_N, 0, d, d, d, 1.0, P, d, P, d, 0.0, R, d, 15)
    before = [oz.stage_tensor(s, ctx=ctx).clone() for s in range(4)]
    oz.oz2_ctx_f8_gemm(ctx, m, n, k, 1.0, A, B, 0.0, C, n)
    assert all(torch.equal(x, oz.stage_tensor(s, ctx=ctx)) for s, x in enumerate(before))
    ctx.destroy()
